// Attention over a cache of histories held in int8 (layout and definition: silvertorch.h).
//
// A block's logits are formed transposed: the matrix instruction takes 16 keys as its rows and 16 query rows as its
// columns, so that a lane holds one query row's logits of four neighbouring tokens, the softmax state of a row is one register of
// its lane, and the weights are, as they lie, the columns of the second product (values as rows).  Nothing goes through
// the LDS on the way; the values are stored in the order of slots that this gives.
//
// Integers are exact as 16-bit floats.  A query row is scaled by a power of two so that its largest magnitude is near
// 2^14 (exact but for values 2^-38 of that), the key scale of the block and the softmax scale multiply the logits in fp32.
// Weights are exp2(x - m + 8) with m a maximum that follows the row's largest logit at a distance of at most 7, so that the sums are
// seldom rescaled: 11 significant bits from 2^15 down to 2^-14 (a 16-bit float's denormals come below 2^-22 of the row's
// largest weight).  Outputs are divided by the fp32 sum of the weights as rounded, so that a row that one token dominates is
// not off by that token's rounding; lse and the blocks' weights go by the sum of the unrounded ones, formed where they are asked for.
#pragma once
#include "st_kv_device.h"

namespace st {

struct KvAttendArgs {
    KvCacheView c;
    KvBatchView b;
    const void* q;
    int64_t q_stride;
    int32_t bf16, group, causal;
    float scale_log2;   // softmax scale * log2(e)
    const uint64_t* mask;
    int32_t mask_words, n_sel;
    const int32_t* blocks;  // selected ones, or null
    void* out;
    float* lse;
    int32_t exact;       // lse or the blocks' weights are asked for
    int32_t chunk, splits, tiles, tile_rows, dies;
    uint32_t pairs;      // of sequences and heads
    int32_t rows_pad;    // rows of a unit and head in the workspace
    float* part_o;       // [unit, head, split, rows_pad, d]
    float4* part_ml;     // [unit, head, split, rows_pad]: maximum, sum of rounded weights, sum of weights, what part_o is in units of
    float2* block_ml;    // [unit, head, entries, rows_pad]: maximum so far, sum of the block's weights; or null
    int64_t entries;     // blocks, or selected ones
    float2* row_ml;      // [unit, head, rows_pad]: final maximum and sum, written where block_ml is
    const float* mass_in;
    float decay;
    float* mass_out;     // [n_seq, n_heads, max_blocks] or null
};

__device__ inline float kv_weight(float2 block, float2 row)
{
    return row.y != 0.0f && block.y != 0.0f ? block.y * __builtin_amdgcn_exp2f(block.x - row.x) / row.y : 0.0f;
}
// Whether the workgroup that has all rows and blocks of a sequence and head writes its blocks' weights too.
__device__ inline bool kv_whole(const KvAttendArgs& a, int n_list) { return a.tiles == 1 && a.tile_rows == 16 && n_list <= a.chunk; }

// Few rows: outputs are sums of up to 2^20 values times 2^15, so that a wavefront that meets value scales above the first of these keeps
// them in units of the second from there on.
constexpr float kKvLarge = 0x1p40f, kKvUnit = 0x1p64f;

constexpr float kKvLift = 8.0f;   // weights are 2^8 times themselves,
constexpr float kKvSlack = 7.0f;  // and the maximum they go by may lie 7 (in powers of two) below the largest logit

// Maxima of this size and more: x * ks - m in one rounding can be above what the rounded products' distance to m allows, by half
// the spacing of numbers near m, and pass a 16-bit float's range.  Such rows subtract m from the rounded products, which is exact
// near the largest ones.  (What looking for them costs: 131.3 us against 130.7 for 500 candidates to each of 16 histories, 294
// against 292 for 2047 tokens under a mask, nothing for single tokens.)
__device__ inline bool kv_far(float m) { return fabsf(m) >= 0x1p18f && m != -__builtin_inff(); }

// A query row goes into the product times *up, a power of two that brings its largest magnitude near 2^14, with the sign
// of the softmax scale; *factor times the product and a key scale is then the logit, in powers of two.
__device__ inline void kv_query_unit(float top, float scale_log2, float* up, float* factor)
{
    const int e = top > 0.0f ? min(max(ilogbf(top), -100), 127) : 0;
    *up = ldexpf(scale_log2 < 0.0f ? -1.0f : 1.0f, 13 - e);
    *factor = fabsf(scale_log2) * ldexpf(1.0f, e - 13);
}

// A row of a unit and head: its token and its head of queries.
struct KvRow {
    int64_t tok;
    int q_head, i;  // i: token of the unit
};
__device__ inline KvRow kv_row(int row, int64_t tok_unit, int head, int group)
{
    KvRow r;
    r.i = (int)((uint32_t)row / (uint32_t)group);
    r.tok = tok_unit + r.i;
    r.q_head = head * group + row - r.i * group;
    return r;
}

// What a tile of rows of a unit (a sequence, or a token whose blocks were selected) and a head reads.
struct KvTile {
    int seq;
    int rows;       // of the unit
    int n_blocks;   // blocks that any row of the tile sees
    int n_list;     // entries to go through: blocks, or what was selected
    int64_t tok_unit, tok_first, tok_last;  // first token of the unit; first and last token of the tile
    int past, len, group;  // a row of token i of the unit sees positions below len - past + i (causal) or len
    bool causal;
    __device__ int limit(int i) const { return max(0, causal ? len - past + i : len); }
    __device__ int token(int row) const { return (int)((uint32_t)row / (uint32_t)group); }  // of the unit
};

// Which part of the work a workgroup does.  The first splits of all rows come first, so that the last workgroups to start
// are those with what long sequences have left.  Parts of one sequence and head that read the same blocks (tiles of rows, tokens
// whose blocks were selected) follow one another on one of the chip's 8 dies, whose L2 serves them: workgroups are handed to
// the dies in turn.
struct KvPlace {
    int seq, head, unit, tile, split;  // unit < 0: none
};
template <bool kSelected>
__device__ inline KvPlace kv_place(const KvAttendArgs& a)
{
    const uint32_t per = (uint32_t)a.tiles * (kSelected ? a.b.max_tok : 1);
    const uint32_t k = blockIdx.x / a.dies;
    uint32_t key = k / per;  // split and pair
    const uint32_t item = k - key * per;
    key = key * a.dies + (blockIdx.x - k * a.dies);
    KvPlace p;
    p.split = key / a.pairs;
    const uint32_t pair = key - p.split * a.pairs;
    p.seq = pair / a.c.n_heads;
    p.head = pair - p.seq * a.c.n_heads;
    p.unit = p.split < a.splits ? p.seq : -1;
    const int i = item / a.tiles;
    p.tile = item - i * a.tiles;
    if (kSelected && p.unit >= 0) {
        int first, count;
        kv_tokens(a.b, p.seq, &first, &count);
        p.unit = i < count ? first + i : -1;
    }
    return p;
}

template <bool kSelected>
__device__ inline KvTile kv_tile(const KvAttendArgs& a, int seq, int unit, int row0, int tile_rows)
{
    KvTile t;
    t.seq = seq;
    const KvSeq q = kv_seq(a.b, t.seq);
    const bool mine = !kSelected || (unit >= q.first && unit < q.first + q.count);
    t.rows = kSelected ? a.group : q.count * a.group;
    t.group = a.group;
    t.causal = a.causal != 0;
    t.len = mine ? q.len : 0;
    // (a unit of one token: that token is its token 0)
    t.past = kSelected ? q.count - 1 - (unit - q.first) : q.count - 1;
    t.tok_unit = kSelected ? unit : q.first;
    const int i_first = t.token(row0), i_last = t.token(max(0, min(row0 + tile_rows, t.rows) - 1));
    t.tok_first = t.tok_unit + i_first;
    t.tok_last = t.tok_unit + i_last;
    t.n_blocks = row0 < t.rows ? (t.limit(i_last) + kKvBlock - 1) / kKvBlock : 0;
    t.n_list = kSelected ? a.n_sel : t.n_blocks;
    return t;
}

// kWaves wavefronts share the blocks of 16 rows and join what they found in the LDS (one: nothing to join, for calls that
// fill the chip with rows alone).  Bound by HBM where rows are few: 64 histories of 2144 to 8192 tokens, 8 heads of 128 with 4 query
// heads each: 143 us, 4.8 TB/s (5.4 with histories of one length; a plain pass over memory reads 6.3), two of 262144 and 163840 tokens 86
// us, 5.1 TB/s.  With a tile to every few tokens it is bound by turning integers into floats, once to a tile.  Selected blocks: 16
// tokens, 8 heads, 64 blocks each, 25 us, 5.4 TB/s; 800 tokens, 4 heads, 8 blocks each, 45 us, 410 MB out of the L2 (9 TB/s),
// 93 MB behind it.
template <int D, bool kSelected, int kWaves>
__global__ __launch_bounds__(kWaves * 64, kWaves == 1 && D <= 128 ? 3 : 2) void kv_attend_kernel(KvAttendArgs a)
{
    constexpr int kSteps = D / 32, kWide = D / 64, kCh = D / 16;
    constexpr bool kHalf = D % 64 != 0;
    // Values of a block are loaded before its keys' products, the next block's keys right behind these.  d = 256 has registers for
    // half of that: its second half of the values takes the place of keys that were used (left to the compiler, the
    // values' loads ended up one behind the other, each with a wait: 193 us against 107 for 8 x 16000 tokens, 4 heads, 64 rows).
    constexpr bool kBoth = D <= 128;
    constexpr int kFirst = kBoth ? kCh : kCh / 2;
    __shared__ float s_o[kWaves][16][D + 4];
    __shared__ float4 s_ml[kWaves][16];
    __shared__ float2 s_fin[16];
    const int lane = threadIdx.x & 63, w = kWaves == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const KvPlace at = kv_place<kSelected>(a);
    if (at.unit < 0) return;
    const int split = at.split, head = at.head, unit = at.unit, row0 = at.tile * 16, jb = split * a.chunk;
    const int64_t uh = (int64_t)unit * a.c.n_heads + head, heads_all = (int64_t)a.c.n_heads * a.group;
    const bool bf16 = a.bf16 != 0;
    // A workgroup's life is short, so what it reads first is asked for at once: the first blocks (pages, or the
    // list of what was selected), the queries, the length.
    const int32_t* list = kSelected ? a.blocks + uh * a.n_sel : a.b.tables + (int64_t)at.seq * a.b.max_blocks;
    const int first_entry = list[min(jb + kWaves * lane + w, (kSelected ? a.n_sel : a.b.max_blocks) - 1)];
    const int row = row0 + n;
    bool valid;
    KvRow of;
    uint4 raw[kSteps];
    {
        int first = unit, rows = a.group;
        if (!kSelected) kv_tokens(a.b, at.seq, &first, &rows), rows *= a.group;
        if (row0 >= rows) return;
        valid = row < rows;
        of = kv_row(valid ? row : row0, first, head, a.group);
        const uint16_t* src = (const uint16_t*)a.q + of.tok * a.q_stride + of.q_head * D;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int ch = k < 2 * kWide ? k / 2 * 64 + g * 16 + k % 2 * 8 : kWide * 64 + g * 8;
            raw[k] = *(const uint4*)(src + ch);
        }
    }
    const KvTile t = kv_tile<kSelected>(a, at.seq, unit, row0, 16);
    const int lim = valid ? t.limit(of.i) : 0, lim_all = t.limit(t.token(row0));
    const int je = min(jb + a.chunk, t.n_list);
    if (split > 0 && jb >= je) return;

    // queries: eight channels of each 32 to a lane, in the order in which it holds those of a key
    half8 q[kSteps];
    float factor;
    {
        float f[kSteps][8];
        float top = 0.0f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            eight_floats(raw[k], bf16, f[k]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[k][j] = valid ? f[k][j] : 0.0f;
                top = fmaxf(top, fabsf(f[k][j]));
            }
        }
        float up;
        kv_query_unit(max_over_16_32(top), a.scale_log2, &up, &factor);
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) q[k][j] = (_Float16)(f[k][j] * up);
    }

    float m = -__builtin_inff(), l = 0.0f, l_exact = 0.0f;
    uint64_t far = 0;    // rows of large logits (kv_far)
    float o_unit = 1.0f;
    float4v o[kCh];
#pragma unroll
    for (int c = 0; c < kCh; ++c) o[c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    for (int j0 = jb; j0 < je; j0 += 64 * kWaves) {
        // up to 64 blocks of this wavefront: page and scales, one to a lane
        const int j = j0 + kWaves * lane + w;
        int block = -1, page = -1;
        if (j < je) {
            const int entry = j0 == jb ? first_entry : list[j];
            block = kSelected ? entry : j;
            if (block >= 0 && block < t.n_blocks) page = kSelected ? kv_page(a.c, a.b, t.seq, block) : kv_page_of(a.c, entry);
        }
        uint64_t any = ~0ull;
        if (a.mask && page >= 0) {  // a block that no row of the tile sees is not read
            any = 0;
            for (int64_t i = t.tok_first; i <= t.tok_last; ++i) any |= a.mask[i * a.mask_words + block];
            if (any == 0) page = -1;
        }
        if (a.block_ml && j < je && page < 0)
            for (int r = 0; r < 16; ++r) a.block_ml[(uh * a.entries + j) * a.rows_pad + row0 + r] = make_float2(0.0f, 0.0f);
        const int64_t ph_l = (int64_t)max(page, 0) * a.c.n_heads + head;
        const float ks_l = page >= 0 ? a.c.k_scale[ph_l] : 0.0f;
        float vs_l = page >= 0 ? a.c.v_scale[ph_l] : 0.0f;
        uint64_t todo = ballot(page >= 0);
        if (todo == 0) continue;
        if (o_unit == 1.0f && ballot(vs_l > kKvLarge) != 0) {
            o_unit = kKvUnit;
#pragma unroll
            for (int c = 0; c < kCh; ++c) o[c] *= 1.0f / kKvUnit;
        }
        vs_l *= 1.0f / o_unit;
        int it = __builtin_ctzll(todo);
        const uint32_t key_at = n * D + g * 16, val_at = n * kKvBlock + g * 16;
        uint4 kw[4][kWide ? kWide : 1];
        uint2 kh[4];
        auto load_keys = [&](int from) {
            const int64_t at_page = (int64_t)(int)lane_value((uint32_t)page, from) * a.c.n_heads + head;
            const int8_t* kp = a.c.k + at_page * (D * kKvBlock);
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
                for (int c = 0; c < kWide; ++c) kw[tt][c] = *(const uint4*)(kp + tt * 16 * D + c * 64 + key_at);
                if (kHalf) kh[tt] = *(const uint2*)(kp + tt * 16 * D + kWide * 64 + (key_at - g * 8));
            }
        };
        // a block's word of the mask: rows of one token have what was read above
        uint64_t word = ~0ull;
        auto load_word = [&](int from) {
            if (kSelected) word = (uint64_t)lane_value((uint32_t)(any >> 32), from) << 32 | lane_value((uint32_t)any, from);
            else if (a.mask) word = a.mask[of.tok * a.mask_words + j0 + kWaves * from + w];
        };
        if (kBoth) load_keys(it);
        load_word(it);
        while (todo) {
            const int cur = it;
            todo &= todo - 1;
            it = todo ? __builtin_ctzll(todo) : -1;
            const int b = (int)lane_value((uint32_t)block, cur);
            const int64_t ph = (int64_t)(int)lane_value((uint32_t)page, cur) * a.c.n_heads + head;
            const int8_t* vp = a.c.v + ph * (D * kKvBlock);
            uint4 vw[kCh];
            auto load_values = [&](int from, int to) {
#pragma unroll
                for (int c = from; c < to; ++c) vw[c] = *(const uint4*)(vp + c * 16 * kKvBlock + val_at);
            };
            if (!kBoth) load_keys(cur);
            load_values(0, kFirst);
            uint64_t see = ~0ull;
            const bool part = a.mask || (b + 1) * kKvBlock > lim_all;
            if (part) {
                const int left = lim - b * kKvBlock;
                see = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0ull;
                see &= word;
            }
            float4v x[4];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                x[tt] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < kWide; ++c) {
                    x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(kw[tt][c].x, kw[tt][c].y), q[2 * c], x[tt], 0, 0, 0);
                    x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(kw[tt][c].z, kw[tt][c].w), q[2 * c + 1], x[tt], 0, 0, 0);
                }
                if (kHalf) x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(kh[tt].x, kh[tt].y), q[kSteps - 1], x[tt], 0, 0, 0);
                if (!kBoth) {
                    __builtin_amdgcn_sched_barrier(0);
                    load_values(kFirst + tt * (kCh - kFirst) / 4, kFirst + (tt + 1) * (kCh - kFirst) / 4);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (it >= 0) {
                if (kBoth) load_keys(it);
                load_word(it);
            }
            // (a scale or a factor of zero gives logits of next to nothing, and -inf stays what it is)
            float ks = fmaxf(__uint_as_float(lane_value(__float_as_uint(ks_l), cur)) * factor, 1e-37f);
            const float vs = __uint_as_float(lane_value(__float_as_uint(vs_l), cur));
            if (part) {
                const uint64_t mine = see >> (g * 4);
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[tt][r] = kv_seen(x[tt][r], (uint32_t)(mine >> (tt / 2 * 32)), tt % 2 * 16 + r);
            }
            float top = x[0][0];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, x[tt][r]);
            top = max_over_16_32(top) * ks;
            // (as branches of their own: one for both, as in the kernel for many rows, 148 us against 143 for the 64 histories above)
            if (ballot(top - m > kKvSlack) != 0) {
                const float m_new = top - m > kKvSlack ? top : m;
                const float alpha = m_new == m ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= alpha;
                l_exact *= alpha;
#pragma unroll
                for (int c = 0; c < kCh; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[c][r] *= alpha;
                far = ballot(kv_far(m));
            }
            float base = m == -__builtin_inff() ? 0.0f : kKvLift - m;
            if (far) {
                const float from = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[tt][r] = __fmul_rn(x[tt][r], ks) - from;
                ks = 1.0f;
                base = kKvLift;
            }
            half8 p[2];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[tt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tt][r], ks, base));
                    p[tt / 2][tt % 2 * 4 + r] = (_Float16)x[tt][r];
                }
            l = add_halves(p[0], add_halves(p[1], l));
            if (a.exact) {
                float sum = 0.0f;
#pragma unroll
                for (int tt = 0; tt < 4; ++tt) sum += (x[tt][0] + x[tt][1]) + (x[tt][2] + x[tt][3]);
                l_exact += sum;
                if (a.block_ml) {
                    const float all = sum_over_16_32(sum);
                    if (g == 0) a.block_ml[(uh * a.entries + j0 + kWaves * cur + w) * a.rows_pad + row] = make_float2(m, all);
                }
            }
#pragma unroll
            for (int c = 0; c < kCh; ++c) {
                float4v y = {0.0f, 0.0f, 0.0f, 0.0f};
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(vw[c].x, vw[c].y), p[0], y, 0, 0, 0);
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(vw[c].z, vw[c].w), p[1], y, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[c][r] = __builtin_fmaf(y[r], vs, o[c][r]);
            }
        }
    }
    l = sum_over_16_32(l);
    l_exact = sum_over_16_32(l_exact);

    // the wavefronts' states into one
    if (g == 0) s_ml[w][n] = make_float4(m, l, l_exact, o_unit);
#pragma unroll
    for (int c = 0; c < kCh; ++c) *(float4v*)&s_o[w][n][c * 16 + g * 4] = o[c];
    __syncthreads();
    const int64_t part = (uh * a.splits + split) * a.rows_pad + row0;
    for (int i = threadIdx.x; i < 16 * (D / 4); i += kWaves * 64) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float top = -__builtin_inff(), y_unit = 1.0f;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            top = fmaxf(top, s_ml[k][r].x);
            y_unit = fmaxf(y_unit, s_ml[k][r].w);
        }
        float sum = 0.0f, exact = 0.0f;
        float4v y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float4 ml = s_ml[k][r];
            const float f = ml.y > 0.0f || ml.y != ml.y ? __builtin_amdgcn_exp2f(ml.x - top) : 0.0f;
            const float4v v = *(const float4v*)&s_o[k][r][c];
            const float fv = ml.w == y_unit ? f : f * (1.0f / kKvUnit);
            sum += ml.y * f;
            exact += ml.z * f;
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] += v[u] * fv;
        }
        if (row0 + r >= t.rows) continue;
        if (t.n_list > a.chunk) {
            *(float4v*)(a.part_o + (part + r) * D + c) = y;
            if (c == 0) a.part_ml[part + r] = make_float4(top, sum, exact, y_unit);
            continue;
        }
        const KvRow to = kv_row(row0 + r, t.tok_unit, head, a.group);
        const int64_t place = to.tok * heads_all + to.q_head;
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        uint32_t h[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) h[u] = to_16_bits(y[u] * inv * y_unit, bf16);
        *(uint2*)((uint16_t*)a.out + place * D + c) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
        if (c == 0) {
            if (a.lse) a.lse[place] = exact == 0.0f ? -__builtin_inff() : (top - kKvLift + log2f(exact)) * 0.69314718056f;
            if (a.row_ml) a.row_ml[uh * a.rows_pad + row0 + r] = make_float2(top, exact);
            s_fin[r] = make_float2(top, exact);
        }
    }
    if (kSelected || !a.mass_out || !kv_whole(a, t.n_list)) return;
    __syncthreads();
    const int nb = a.b.max_blocks, held = (t.len + kKvBlock - 1) / kKvBlock;
    const int64_t to = uh * nb;
    for (int b = threadIdx.x; b < nb; b += kWaves * 64) {
        float sum = 0.0f;
        if (b < t.n_list) {
            const float2* block = a.block_ml + (uh * a.entries + b) * a.rows_pad;
            for (int r = 0; r < t.rows; ++r) sum += kv_weight(block[r], s_fin[r]);
        }
        a.mass_out[to + b] = b < held ? (a.mass_in ? a.mass_in[to + b] * a.decay : 0.0f) + sum : 0.0f;
    }
}

// Joins the splits of a row: kWaves wavefronts to a row, each lane a quarter of four channels' sums over every
// (kWaves * 256 / D)-th split.  Bound by latency: 64 rows of 64 splits 4.8 us, 30705 rows of 2 splits 19 us (loads asked for
// before the length was known changed nothing).
template <int D, bool kSelected, int kWaves>
__global__ __launch_bounds__(kKvThreads) void kv_join_kernel(KvAttendArgs a)
{
    constexpr int kLanes = D / 4, kTeam = kWaves * 64, kParts = kTeam / kLanes;  // (D = 96: 24 lanes, 16 of 256 idle)
    constexpr int kRows = kKvThreads / kTeam;
    __shared__ float4v s_y[kRows][kParts][kLanes];
    __shared__ float2 s_top[kRows][kWaves];
    __shared__ float2 s_sum[kRows][kParts];
    const int team = threadIdx.x / kTeam, me = threadIdx.x % kTeam, lane = me & 63;
    const int64_t heads_all = (int64_t)a.c.n_heads * a.group;
    const int64_t place = (int64_t)blockIdx.x * kRows + team;
    const bool there = place < a.b.n_tok * heads_all;
    const int tok = there ? (int)(place / heads_all) : 0, qh = there ? (int)(place % heads_all) : 0, head = qh / a.group;
    const int s = kv_seq_of(a.b, tok);
    const KvSeq q = kv_seq(a.b, s);
    bool mine = there && tok >= q.first && tok < q.first + q.count;
    const int unit = kSelected ? tok : s;
    const int row = !mine ? 0 : kSelected ? qh % a.group : (tok - q.first) * a.group + qh % a.group;
    const KvTile t = kv_tile<kSelected>(a, s, unit, row / a.tile_rows * a.tile_rows, a.tile_rows);
    const int64_t uh = (int64_t)unit * a.c.n_heads + head, stride = a.rows_pad;
    mine = mine && t.n_list > a.chunk;  // (a row in one split has its output already)
    const int splits = mine ? (t.n_list + a.chunk - 1) / a.chunk : 0;
    const int64_t part = uh * a.splits * stride + row;
    float top = -__builtin_inff(), y_unit = 0.0f;  // the largest maximum, and the largest unit of the parts' outputs
    for (int i = me; i < splits; i += kTeam) {
        const float4 ml = a.part_ml[part + i * stride];
        top = fmaxf(top, ml.x);
        y_unit = fmaxf(y_unit, ml.w);
    }
    for (int k = 8; k > 0; k >>= 1) {
        top = fmaxf(top, __shfl_xor(top, k));
        y_unit = fmaxf(y_unit, __shfl_xor(y_unit, k));
    }
    top = max_over_16_32(top);
    y_unit = max_over_16_32(y_unit);
    if (lane == 0) s_top[team][me >> 6] = make_float2(top, y_unit);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        top = fmaxf(top, s_top[team][k].x);
        y_unit = fmaxf(y_unit, s_top[team][k].y);
    }
    const float up = y_unit < 0x1p-64f ? 0x1p64f : 1.0f, per_unit = y_unit > 0.0f ? 1.0f / (y_unit * up) : 0.0f;  // (for denormals)
    const int c = me % kLanes, from = me / kLanes;
    float sum = 0.0f, exact = 0.0f;
    float4v y = {0.0f, 0.0f, 0.0f, 0.0f};
    if (from < kParts) {
#pragma unroll 4
        for (int i = from; i < splits; i += kParts) {
            const float4 ml = a.part_ml[part + i * stride];
            const float4v v = *(const float4v*)(a.part_o + (part + i * stride) * D + c * 4);
            const float f = ml.y > 0.0f || ml.y != ml.y ? __builtin_amdgcn_exp2f(ml.x - top) : 0.0f;
            const float fv = f * (ml.w * up * per_unit);
            sum = __builtin_fmaf(ml.y, f, sum);
            exact = __builtin_fmaf(ml.z, f, exact);
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = __builtin_fmaf(v[u], fv, y[u]);
        }
        s_y[team][from][c] = y;
        if (c == 0) s_sum[team][from] = make_float2(sum, exact);
    }
    __syncthreads();
    if (!mine || from != 0) return;
#pragma unroll
    for (int k = 1; k < kParts; ++k) {
        const float4v v = s_y[team][k][c];
        sum += s_sum[team][k].x;
        exact += s_sum[team][k].y;
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] += v[u];
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    uint32_t h[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) h[u] = to_16_bits(y[u] * inv * y_unit, a.bf16 != 0);
    *(uint2*)((uint16_t*)a.out + place * D + c * 4) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    if (c == 0) {
        if (a.lse) a.lse[place] = exact == 0.0f ? -__builtin_inff() : (top - kKvLift + log2f(exact)) * 0.69314718056f;
        if (a.row_ml) a.row_ml[uh * stride + row] = make_float2(top, exact);
    }
}

// Weights of the blocks, summed over the rows of a sequence and head: kLanes lanes to a block, each every kLanes-th row.  Runs
// where a call's rows are spread over workgroups; else the attention's own workgroup does it at its end.
template <int kLanes>
__global__ __launch_bounds__(kKvThreads) void kv_mass_kernel(KvAttendArgs a)
{
    constexpr int kBlocks = kKvThreads / kLanes;
    const int nb = a.b.max_blocks, chunks = (nb + kBlocks - 1) / kBlocks;
    const int chunk = blockIdx.x % chunks, sh = blockIdx.x / chunks;
    const int s = sh / a.c.n_heads, lane = threadIdx.x % kLanes;
    const int b = chunk * kBlocks + threadIdx.x / kLanes;
    const KvSeq q = kv_seq(a.b, s);
    if (kLanes == 16 && q.count > 0 && kv_whole(a, kv_tile<false>(a, s, s, 0, 16).n_list)) return;  // (written already)
    const bool held = b < nb && b * kKvBlock < q.len;
    float sum = 0.0f;
    if (held) {
        // (nothing was written for rows that end before the block)
        int first = 0;
        if (a.causal) first = max(0, b * kKvBlock - (q.len - q.count)) * a.group;
        const float2* block = a.block_ml + ((int64_t)sh * a.entries + b) * a.rows_pad;
        const float2* row = a.row_ml + (int64_t)sh * a.rows_pad;
        for (int r = first + lane; r < q.count * a.group; r += kLanes) sum += kv_weight(block[r], row[r]);
    }
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane != 0 || b >= nb) return;
    const int64_t to = (int64_t)sh * nb + b;
    a.mass_out[to] = held ? (a.mass_in ? a.mass_in[to] * a.decay : 0.0f) + sum : 0.0f;
}

// The same where blocks were selected: token after token, each adds to the blocks it read.
__global__ __launch_bounds__(kKvThreads) void kv_mass_selected_kernel(KvAttendArgs a)
{
    extern __shared__ float acc[];
    const int nb = a.b.max_blocks;
    const int head = blockIdx.x % a.c.n_heads, s = blockIdx.x / a.c.n_heads;
    const KvSeq q = kv_seq(a.b, s);
    const int held = (q.len + kKvBlock - 1) / kKvBlock;
    for (int b = threadIdx.x; b < held; b += kKvThreads) acc[b] = 0.0f;
    __syncthreads();
    for (int i = 0; i < q.count; ++i) {
        const int64_t th = (int64_t)(q.first + i) * a.c.n_heads + head;
        for (int j = threadIdx.x; j < a.n_sel; j += kKvThreads) {
            const int b = a.blocks[th * a.n_sel + j];
            if (b < 0 || b >= held) continue;
            float sum = 0.0f;
            for (int h = 0; h < a.group; ++h)
                sum += kv_weight(a.block_ml[(th * a.n_sel + j) * a.rows_pad + h], a.row_ml[th * a.rows_pad + h]);
            acc[b] += sum;
        }
        __syncthreads();
    }
    const int64_t to = (int64_t)blockIdx.x * nb;
    for (int b = threadIdx.x; b < nb; b += kKvThreads)
        a.mass_out[to + b] = b < held ? (a.mass_in ? a.mass_in[to + b] * a.decay : 0.0f) + acc[b] : 0.0f;
}

}  // namespace st
