// Attention over a cache of histories held in int8 (layout and definition: silvertorch.h).
//
// A block's logits are formed transposed: the matrix instruction takes 16 keys as its rows and 16 query rows as its
// columns, so that a lane holds one query row's logits of four neighbouring tokens, the softmax state of a row is one register of
// its lane, and the weights are, as they lie, the columns of the second product (values as rows).  Nothing goes through
// the LDS on the way; the values are stored in the order of slots that this gives.
//
// Integers are exact as 16-bit floats.  A query row is scaled by a power of two so that its largest magnitude is near
// 2^14 (exact but for values 2^-38 of that), the key scale of the block and the softmax scale multiply the logits in fp32.
// Weights are exp2(x - m + 14): 11 significant bits from 2^14 down to 2^-14 (a 16-bit float's denormals
// come below 2^-28 of the row's largest weight), and the sum of the weights is of the unrounded ones, in fp32.
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
    int32_t chunk, splits, tiles;
    float* part_o;      // [unit, head, tile, split, 16, d]
    float2* part_ml;    // [unit, head, tile, split, 16]: maximum, sum of weights
    float2* block_ml;   // [n_tok, n_q_heads, block_stride]: maximum so far, sum of the block's weights; or null
    int64_t block_stride;
    float2* row_ml;     // [n_tok, n_q_heads]: final maximum and sum, written where block_ml is
};

constexpr float kKvLift = 14.0f;  // weights are 2^14 times themselves

// What a tile of 16 rows of a unit (a sequence, or a token whose blocks were selected) and a head reads.
struct KvTile {
    int seq;
    int rows;       // of the unit
    int row;        // this lane's
    bool valid;
    int64_t tok;    // its token
    int q_head;
    int lim;        // it sees positions below this one
    int lim_all;    // all valid rows of the tile see those below this one
    int n_blocks;   // blocks that any row of the tile sees
    int n_list;     // entries to go through: blocks, or what was selected
};

template <bool kSelected>
__device__ inline KvTile kv_tile(const KvAttendArgs& a, int unit, int head, int tile, int n)
{
    KvTile t;
    t.seq = kSelected ? kv_seq_of(a.b, unit) : unit;
    const KvSeq q = kv_seq(a.b, t.seq);
    const bool mine = !kSelected || (unit >= q.first && unit < q.first + q.count);
    t.rows = kSelected ? a.group : q.count * a.group;
    t.row = tile * 16 + n;
    t.valid = t.row < t.rows;
    const int last = min(tile * 16 + 15, t.rows - 1);
    const int i = kSelected ? unit - q.first : min(t.row, max(t.rows - 1, 0)) / a.group;
    const int i_first = kSelected ? i : tile * 16 / a.group, i_last = kSelected ? i : last / a.group;
    t.tok = kSelected ? unit : (int64_t)q.first + i;
    t.q_head = head * a.group + (kSelected ? t.row : t.row - i * a.group);
    const int past = q.count - 1;
    t.lim = t.valid && mine ? max(0, a.causal ? q.len - (past - i) : q.len) : 0;
    t.lim_all = max(0, a.causal ? q.len - (past - i_first) : q.len);
    const int lim_max = tile * 16 < t.rows && mine ? max(0, a.causal ? q.len - (past - i_last) : q.len) : 0;
    t.n_blocks = (lim_max + kKvBlock - 1) / kKvBlock;
    t.n_list = kSelected ? a.n_sel : t.n_blocks;
    return t;
}

template <int D, bool kSelected>
__global__ __launch_bounds__(kKvThreads, 2) void kv_attend_kernel(KvAttendArgs a)
{
    constexpr int kSteps = D / 32, kWide = D / 64, kCh = D / 16;
    constexpr bool kHalf = D % 64 != 0;
    __shared__ float s_o[4][16][D + 4];
    __shared__ float2 s_ml[4][16];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    int64_t at = blockIdx.x;
    const int split = (int)(at % a.splits);
    at /= a.splits;
    const int tile = (int)(at % a.tiles);
    at /= a.tiles;
    const int head = (int)(at % a.c.n_heads), unit = (int)(at / a.c.n_heads);
    const KvTile t = kv_tile<kSelected>(a, unit, head, tile, n);
    if (tile * 16 >= t.rows) return;
    const int jb = split * a.chunk, je = min(jb + a.chunk, t.n_list);
    if (split > 0 && jb >= je) return;
    const bool bf16 = a.bf16 != 0;

    // queries: eight channels of each 32 to a lane, in the order in which it holds those of a key
    half8 q[kSteps];
    float factor;
    {
        float f[kSteps][8];
        float top = 0.0f;
        const uint16_t* src = (const uint16_t*)a.q + t.tok * a.q_stride + (int64_t)t.q_head * D;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int ch = k < 2 * kWide ? k / 2 * 64 + g * 16 + k % 2 * 8 : kWide * 64 + g * 8;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (t.valid) v = *(const uint4*)(src + ch);
            eight_floats(v, bf16, f[k]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[k][j]));
        }
        top = max_over_16_32(top);
        int e = top > 0.0f ? ilogbf(top) : 0;
        e = min(max(e, -100), 120);
        const float up = ldexpf(1.0f, 13 - e);
        factor = a.scale_log2 * ldexpf(1.0f, e - 13);
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) q[k][j] = (_Float16)(f[k][j] * up);
    }

    float m = -__builtin_inff(), l = 0.0f;
    float4v o[kCh];
#pragma unroll
    for (int c = 0; c < kCh; ++c) o[c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    for (int j0 = jb; j0 < je; j0 += 256) {
        // up to 64 blocks of this wavefront: page and scales, one to a lane
        const int j = j0 + 4 * lane + w;
        int block = -1, page = -1;
        if (j < je) {
            block = kSelected ? a.blocks[((int64_t)unit * a.c.n_heads + head) * a.n_sel + j] : j;
            if (block >= 0 && block < t.n_blocks) page = kv_page(a.c, a.b, t.seq, block);
        }
        const int64_t ph_l = (int64_t)max(page, 0) * a.c.n_heads + head;
        const float ks_l = page >= 0 ? a.c.k_scale[ph_l] : 0.0f, vs_l = page >= 0 ? a.c.v_scale[ph_l] : 0.0f;
        const int n_it = min(64, max(0, (je - j0 - w + 3) / 4));
        for (int it = 0; it < n_it; ++it) {
            const int pg = (int)lane_value((uint32_t)page, it);
            const int b = (int)lane_value((uint32_t)block, it);
            float2* bml = a.block_ml ? a.block_ml + (t.tok * a.c.n_heads * a.group + t.q_head) * a.block_stride + (j0 + 4 * it + w) : nullptr;
            uint64_t see = ~0ull;
            bool part = false;
            if (pg >= 0 && (a.mask || (b + 1) * kKvBlock > t.lim_all)) {
                part = true;
                const int left = t.lim - b * kKvBlock;
                see = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0ull;
                if (a.mask && see) see &= a.mask[t.tok * a.mask_words + b];
            }
            if (pg < 0 || (part && ballot(see != 0) == 0)) {
                if (bml && g == 0 && t.valid) *bml = make_float2(0.0f, 0.0f);
                continue;
            }
            const int64_t ph = (int64_t)pg * a.c.n_heads + head;
            const int8_t* kp = a.c.k + ph * (D * kKvBlock) + n * D;
            const int8_t* vp = a.c.v + ph * (D * kKvBlock) + n * kKvBlock + g * 16;
            const float ks = __uint_as_float(lane_value(__float_as_uint(ks_l), it)) * factor;
            const float vs = __uint_as_float(lane_value(__float_as_uint(vs_l), it));
            float4v x[4];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                x[tt] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < kWide; ++c) {
                    const uint4 r = *(const uint4*)(kp + tt * 16 * D + c * 64 + g * 16);
                    x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(r.x, r.y), q[2 * c], x[tt], 0, 0, 0);
                    x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(r.z, r.w), q[2 * c + 1], x[tt], 0, 0, 0);
                }
                if (kHalf) {
                    const uint2 r = *(const uint2*)(kp + tt * 16 * D + kWide * 64 + g * 8);
                    x[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(r.x, r.y), q[kSteps - 1], x[tt], 0, 0, 0);
                }
            }
#pragma unroll
            for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                for (int r = 0; r < 4; ++r) x[tt][r] *= ks;
            if (part) {
                const uint64_t mine = see >> (g * 4);
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!((mine >> (tt * 16 + r)) & 1)) x[tt][r] = -__builtin_inff();
            }
            float top = x[0][0];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, x[tt][r]);
            const float m_new = fmaxf(m, max_over_16_32(top));
            const float base = m_new == -__builtin_inff() ? 0.0f : m_new - kKvLift;
            const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            float sum = 0.0f;
            half8 p[2];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = __builtin_amdgcn_exp2f(x[tt][r] - base);
                    sum += e;
                    p[tt / 2][tt % 2 * 4 + r] = (_Float16)e;
                }
            l = l * alpha + sum;
            if (bml) {
                const float all = sum_over_16_32(sum);
                if (g == 0 && t.valid) *bml = make_float2(m, all);
            }
#pragma unroll
            for (int c = 0; c < kCh; ++c) {
                const uint4 r = *(const uint4*)(vp + c * 16 * kKvBlock);
                float4v y = {0.0f, 0.0f, 0.0f, 0.0f};
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(r.x, r.y), p[0], y, 0, 0, 0);
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(eight_halves(r.z, r.w), p[1], y, 0, 0, 0);
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) o[c][r4] = o[c][r4] * alpha + y[r4] * vs;
            }
        }
    }
    l = sum_over_16_32(l);

    // the four wavefronts' states into one
    if (g == 0) s_ml[w][n] = make_float2(m, l);
#pragma unroll
    for (int c = 0; c < kCh; ++c) *(float4v*)&s_o[w][n][c * 16 + g * 4] = o[c];
    __syncthreads();
    const int64_t part = ((int64_t)(unit * (int64_t)a.c.n_heads + head) * a.tiles + tile) * a.splits + split;
    const int64_t heads_all = (int64_t)a.c.n_heads * a.group;
    for (int i = threadIdx.x; i < 16 * (D / 4); i += kKvThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float top = -__builtin_inff();
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, s_ml[k][r].x);
        float sum = 0.0f;
        float4v y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 ml = s_ml[k][r];
            const float f = ml.y > 0.0f || ml.y != ml.y ? __builtin_amdgcn_exp2f(ml.x - top) : 0.0f;
            const float4v v = *(const float4v*)&s_o[k][r][c];
            sum += ml.y * f;
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] += v[u] * f;
        }
        const int row = tile * 16 + r;
        if (row >= t.rows) continue;
        if (a.splits > 1) {
            *(float4v*)(a.part_o + (part * 16 + r) * D + c) = y;
            if (c == 0) a.part_ml[part * 16 + r] = make_float2(top, sum);
            continue;
        }
        const KvTile tr = kv_tile<kSelected>(a, unit, head, tile, r);
        const int64_t place = tr.tok * heads_all + tr.q_head;
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        uint32_t h[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) h[u] = to_16_bits(y[u] * inv, bf16);
        *(uint2*)((uint16_t*)a.out + place * D + c) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
        if (c == 0) {
            if (a.lse) a.lse[place] = sum == 0.0f ? -__builtin_inff() : (top - kKvLift + log2f(sum)) * 0.69314718056f;
            if (a.row_ml) a.row_ml[place] = make_float2(top, sum);
        }
    }
}

// Joins the splits of a row.  One wavefront to a row.
template <int D, bool kSelected>
__global__ __launch_bounds__(kKvThreads) void kv_join_kernel(KvAttendArgs a)
{
    constexpr int kPer = D / 64 ? (D + 63) / 64 : 1;  // channels of a lane
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t heads_all = (int64_t)a.c.n_heads * a.group;
    const int64_t place = (int64_t)blockIdx.x * 4 + w;
    if (place >= a.b.n_tok * heads_all) return;
    const int tok = (int)(place / heads_all), qh = (int)(place % heads_all), head = qh / a.group;
    const int s = kv_seq_of(a.b, tok);
    const KvSeq q = kv_seq(a.b, s);
    if (tok < q.first || tok >= q.first + q.count) return;
    const int unit = kSelected ? tok : s;
    const int row = kSelected ? qh % a.group : (tok - q.first) * a.group + qh % a.group, tile = row / 16;
    const KvTile t = kv_tile<kSelected>(a, unit, head, tile, row % 16);
    const int splits = min(a.splits, max(1, (t.n_list + a.chunk - 1) / a.chunk));
    const int64_t part = (((int64_t)unit * a.c.n_heads + head) * a.tiles + tile) * a.splits * 16 + row % 16;
    float top = -__builtin_inff();
    for (int i = lane; i < splits; i += 64) top = fmaxf(top, a.part_ml[part + (int64_t)i * 16].x);
    for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    float sum = 0.0f, y[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) y[u] = 0.0f;
    for (int i = 0; i < splits; ++i) {
        const float2 ml = a.part_ml[part + (int64_t)i * 16];
        const float f = ml.y > 0.0f || ml.y != ml.y ? __builtin_amdgcn_exp2f(ml.x - top) : 0.0f;
        sum += ml.y * f;
        const float* src = a.part_o + (part + (int64_t)i * 16) * D;
#pragma unroll
        for (int u = 0; u < kPer; ++u)
            if (u * 64 + lane < D) y[u] += src[u * 64 + lane] * f;
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int u = 0; u < kPer; ++u)
        if (u * 64 + lane < D) ((uint16_t*)a.out)[place * D + u * 64 + lane] = (uint16_t)to_16_bits(y[u] * inv, a.bf16 != 0);
    if (lane == 0) {
        if (a.lse) a.lse[place] = sum == 0.0f ? -__builtin_inff() : (top - kKvLift + log2f(sum)) * 0.69314718056f;
        if (a.row_ml) a.row_ml[place] = make_float2(top, sum);
    }
}

struct KvMassArgs {
    KvAttendArgs t;
    const float* in;
    float decay;
    float* out;
};

__device__ inline float kv_weight(float2 block, float2 row)
{
    return row.y != 0.0f && block.y != 0.0f ? block.y * __builtin_amdgcn_exp2f(block.x - row.x) / row.y : 0.0f;
}

// Weights of the blocks, summed over the rows of a sequence and head, in the order of the rows.  A thread to a block.
__global__ __launch_bounds__(kKvThreads) void kv_mass_kernel(KvMassArgs a)
{
    const int nb = a.t.b.max_blocks, chunks = (nb + kKvThreads - 1) / kKvThreads;
    const int chunk = blockIdx.x % chunks, sh = blockIdx.x / chunks;
    const int head = sh % a.t.c.n_heads, s = sh / a.t.c.n_heads;
    const int b = chunk * kKvThreads + threadIdx.x;
    if (b >= nb) return;
    const KvSeq q = kv_seq(a.t.b, s);
    const int64_t to = (int64_t)sh * nb + b;
    if (b * kKvBlock >= q.len) {
        a.out[to] = 0.0f;
        return;
    }
    float sum = 0.0f;
    const int heads_all = a.t.c.n_heads * a.t.group;
    for (int i = 0; i < q.count; ++i) {
        const int lim = a.t.causal ? q.len - (q.count - 1 - i) : q.len;
        if (b * kKvBlock >= lim) continue;  // (nothing was written there)
        for (int h = 0; h < a.t.group; ++h) {
            const int64_t place = (int64_t)(q.first + i) * heads_all + head * a.t.group + h;
            sum += kv_weight(a.t.block_ml[place * a.t.block_stride + b], a.t.row_ml[place]);
        }
    }
    a.out[to] = (a.in ? a.in[to] * a.decay : 0.0f) + sum;
}

// The same where blocks were selected: token after token, each adds to the blocks it read.
__global__ __launch_bounds__(kKvThreads) void kv_mass_selected_kernel(KvMassArgs a)
{
    extern __shared__ float acc[];
    const int nb = a.t.b.max_blocks;
    const int head = blockIdx.x % a.t.c.n_heads, s = blockIdx.x / a.t.c.n_heads;
    const KvSeq q = kv_seq(a.t.b, s);
    const int held = (q.len + kKvBlock - 1) / kKvBlock;
    for (int b = threadIdx.x; b < held; b += kKvThreads) acc[b] = 0.0f;
    __syncthreads();
    const int heads_all = a.t.c.n_heads * a.t.group;
    for (int i = 0; i < q.count; ++i) {
        const int64_t tok = q.first + i;
        for (int j = threadIdx.x; j < a.t.n_sel; j += kKvThreads) {
            const int b = a.t.blocks[(tok * a.t.c.n_heads + head) * a.t.n_sel + j];
            if (b < 0 || b >= held) continue;
            float sum = 0.0f;
            for (int h = 0; h < a.t.group; ++h) {
                const int64_t place = tok * heads_all + head * a.t.group + h;
                sum += kv_weight(a.t.block_ml[place * a.t.block_stride + j], a.t.row_ml[place]);
            }
            acc[b] += sum;
        }
        __syncthreads();
    }
    const int64_t to = (int64_t)blockIdx.x * nb;
    for (int b = threadIdx.x; b < nb; b += kKvThreads)
        a.out[to + b] = b < held ? (a.in ? a.in[to + b] * a.decay : 0.0f) + acc[b] : 0.0f;
}

}  // namespace st
