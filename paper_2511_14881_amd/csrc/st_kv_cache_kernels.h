// Writing, reading, searching and shrinking the cache of histories (layout: silvertorch.h).
#pragma once
#include "st_kv_device.h"

namespace st {

// ---------------------------------------------------------------- append
// One workgroup to a page and head.  New rows are quantised with the page's scale as it becomes, older integers
// move to it when it grows (round(q * o / s): a block has one scale, so they have to).
__device__ inline int kv_quant(float x, float s)
{
    if (!(s > 0.0f)) return 0;
    return (int)fminf(fmaxf(rintf(__fdiv_rn(x, s)), -127.0f), 127.0f);
}
__device__ inline int kv_moved(int q, float ratio) { return (int)rintf(__fmul_rn((float)q, ratio)); }
__device__ inline uint32_t kv_moved4(uint32_t w, float ratio)
{
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= (uint32_t)(kv_moved((int)(int8_t)(w >> (8 * i)), ratio) & 255) << (8 * i);
    return r;
}

struct KvAppendArgs {
    KvCacheView c;
    KvBatchView b;
    const void* k_new;
    const void* v_new;
    int64_t k_stride, v_stride;
    int32_t bf16, touched;  // touched: pages of a sequence that the call may write
};

template <int D>
__global__ __launch_bounds__(kKvThreads) void kv_append_kernel(KvAppendArgs a)
{
    constexpr int kPieces = D / 8;  // 8 channels: 16 bytes of a new row
    __shared__ int8_t tile[D * kKvBlock];
    __shared__ float s_max[kKvThreads / 64];
    const int tid = threadIdx.x;
    const int head = blockIdx.x % a.c.n_heads, rest = blockIdx.x / a.c.n_heads;
    const int s = rest / a.touched;
    const KvSeq q = kv_seq(a.b, s);
    const int begin = q.len - q.count;  // position of the first new token
    const int block = max(begin, 0) / kKvBlock + rest % a.touched;
    const int p0 = max(begin - block * kKvBlock, 0), p1 = min(q.len - block * kKvBlock, kKvBlock);
    if (p1 <= p0 || block >= a.b.max_blocks) return;
    const int page = kv_page(a.c, a.b, s, block);
    if (page < 0) return;
    const int64_t ph = (int64_t)page * a.c.n_heads + head;
    const int64_t row0 = (int64_t)q.first + ((int64_t)block * kKvBlock - begin);  // row of the block's position 0
    const bool bf16 = a.bf16 != 0;
    const int n_new = (p1 - p0) * kPieces;
    for (int part = 0; part < 2; ++part) {  // keys, then values
        const uint16_t* src = (const uint16_t*)(part ? a.v_new : a.k_new) + head * D;
        const int64_t stride = part ? a.v_stride : a.k_stride;
        int8_t* dst = (part ? a.c.v : a.c.k) + ph * (D * kKvBlock);
        float* scale = (part ? a.c.v_scale : a.c.k_scale) + ph;
        float top = 0.0f;
        for (int i = tid; i < n_new; i += kKvThreads) {
            float f[8];
            eight_floats(*(const uint4*)(src + (row0 + p0 + i / kPieces) * stride + i % kPieces * 8), bf16, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
        }
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        if ((tid & 63) == 0) s_max[tid >> 6] = top;
        const float old = p0 > 0 ? *scale : 0.0f;
        __syncthreads();
        top = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
        const float sc = fmaxf(old, __fdiv_rn(top, 127.0f));
        const float ratio = sc > 0.0f ? __fdiv_rn(old, sc) : 0.0f;
        // older integers into the tile, at the new scale (all slots: those that hold no token do not matter)
        if (p0 > 0)
            for (int i = tid; i < D * kKvBlock / 16; i += kKvThreads) {
                uint4 w = ((const uint4*)dst)[i];
                if (ratio != 1.0f) {
                    w.x = kv_moved4(w.x, ratio);
                    w.y = kv_moved4(w.y, ratio);
                    w.z = kv_moved4(w.z, ratio);
                    w.w = kv_moved4(w.w, ratio);
                }
                ((uint4*)tile)[i] = w;
            }
        __syncthreads();
        for (int i = tid; i < n_new; i += kKvThreads) {
            const int t = p0 + i / kPieces, c = i % kPieces * 8;
            float f[8];
            eight_floats(*(const uint4*)(src + (row0 + t) * stride + c), bf16, f);
            if (part == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) tile[t * D + c + j] = (int8_t)kv_quant(f[j], sc);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) tile[(c + j) * kKvBlock + kv_slot(t)] = (int8_t)kv_quant(f[j], sc);
            }
        }
        __syncthreads();
        for (int i = tid; i < D * kKvBlock / 16; i += kKvThreads) ((uint4*)dst)[i] = ((const uint4*)tile)[i];
        if (tid == 0) *scale = sc;
        if (part == 0 && tid < D) {
            int hi = -128, lo = 127;
            for (int t = 0; t < p1; ++t) {
                const int v = tile[t * D + tid];
                hi = max(hi, v);
                lo = min(lo, v);
            }
            a.c.bounds[ph * (2 * D) + tid] = (int8_t)hi;
            a.c.bounds[ph * (2 * D) + D + tid] = (int8_t)lo;
        }
        __syncthreads();  // the tile and s_max are used again
    }
}

// ---------------------------------------------------------------- read back
struct KvReadArgs {
    KvCacheView c;
    KvBatchView b;
    int32_t n_blocks;
    float* k;
    float* v;
    float* bounds;
};

template <int D>
__global__ __launch_bounds__(kKvThreads) void kv_read_kernel(KvReadArgs a)
{
    const int tid = threadIdx.x;
    const int64_t out = blockIdx.x;  // (s, j, head)
    const int head = (int)(out % a.c.n_heads);
    const int64_t rest = out / a.c.n_heads;
    const int j = (int)(rest % a.n_blocks), s = (int)(rest / a.n_blocks);
    const KvSeq q = kv_seq(a.b, s);
    const int held = (q.len + kKvBlock - 1) / kKvBlock;
    const int block = max(0, held - a.n_blocks) + j;
    const int page = block < held ? kv_page(a.c, a.b, s, block) : -1;
    const int n = page < 0 ? 0 : min(kKvBlock, q.len - block * kKvBlock);
    const int64_t ph = (int64_t)max(page, 0) * a.c.n_heads + head;
    if (a.k) {
        const float sc = n ? a.c.k_scale[ph] : 0.0f;
        const uint32_t* src = (const uint32_t*)(a.c.k + ph * (D * kKvBlock));
        float4* dst = (float4*)(a.k + out * (D * kKvBlock));
        for (int i = tid; i < D * kKvBlock / 4; i += kKvThreads) {
            float4 r = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (i / (D / 4) < n) {
                const uint32_t w = src[i];
                r = make_float4((float)(int8_t)w * sc, (float)(int8_t)(w >> 8) * sc, (float)(int8_t)(w >> 16) * sc,
                                (float)(int8_t)(w >> 24) * sc);
            }
            dst[i] = r;
        }
    }
    if (a.v) {
        __shared__ uint32_t tile[D * kKvBlock / 4 + D];  // a row of 16 words and one of padding
        const float sc = n ? a.c.v_scale[ph] : 0.0f;
        const uint32_t* src = (const uint32_t*)(a.c.v + ph * (D * kKvBlock));
        if (n)
            for (int i = tid; i < D * kKvBlock / 4; i += kKvThreads) tile[i / 16 * 17 + i % 16] = src[i];
        __syncthreads();
        float* dst = a.v + out * (D * kKvBlock);
        for (int i = tid; i < D * kKvBlock; i += kKvThreads) {
            const int t = i / D, c = i % D, slot = kv_slot(t);
            dst[i] = t < n ? (float)(int8_t)(tile[c * 17 + slot / 4] >> (8 * (slot & 3))) * sc : 0.0f;
        }
    }
    if (a.bounds && tid < 2 * D)
        for (int i = tid; i < 2 * D; i += kKvThreads)
            a.bounds[out * (2 * D) + i] = n ? (float)a.c.bounds[ph * (2 * D) + i] * a.c.k_scale[ph] : 0.0f;
}

// ---------------------------------------------------------------- the best n of an array of keys
// Marks the `want` largest keys (0: not to be had; equal keys: the lower index first) of keys[0 .. n) by a walk over
// their four bytes from the top, and hands each marked index to emit(index, rank), rank counting the marked ones in index order.
// Returns how many there are.  All threads of the workgroup; hist and part are its scratch.
struct KvPick {
    uint32_t hist[256];
    uint32_t part[kKvThreads / 64 * 2];
    uint32_t prefix, want;
};

__device__ inline uint32_t wg_scan_add(uint32_t v, uint32_t* part, uint32_t* total)  // exclusive, over 256 threads
{
    const int tid = threadIdx.x, w = tid >> 6;
    const uint32_t inc = wave_scan_add(v);
    if ((tid & 63) == 63) part[w] = inc;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kKvThreads / 64; ++i) {
        const uint32_t p = part[i];
        before += i < w ? p : 0u;
        all += p;
    }
    __syncthreads();
    *total = all;
    return before + inc - v;
}

template <class Emit>
__device__ inline int kv_pick(const uint32_t* keys, int n, int want, KvPick* s, Emit emit)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0, need = (uint32_t)want;
    // each byte: how many keys with the bytes so far have which value, and where the want-th lies
    for (int shift = 24; shift >= 0; shift -= 8) {
        s->hist[tid] = 0;
        if (tid == 0) s->want = 0xFFFFFFFFu;
        __syncthreads();
        const uint32_t above = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
        for (int i = tid; i < n; i += kKvThreads) {
            const uint32_t k = keys[i];
            if (k != 0 && (k & above) == prefix) atomicAdd(&s->hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        const uint32_t mine = s->hist[255 - tid];
        uint32_t total;
        const uint32_t before = wg_scan_add(mine, s->part, &total);
        if (before < need && before + mine >= need) {
            s->prefix = prefix | ((uint32_t)(255 - tid) << shift);
            s->want = need - before;
        }
        __syncthreads();
        if (s->want == 0xFFFFFFFFu) {  // fewer keys than wanted: all of them (only the first byte can say so)
            prefix = 0;
            need = 0;
            break;
        }
        prefix = s->prefix;
        need = s->want;
        __syncthreads();
    }
    // keys above prefix are in, and the first `need` of those equal to it
    const int per = (n + kKvThreads - 1) / kKvThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    uint32_t over = 0, same = 0;
    for (int i = i0; i < i1; ++i) {
        over += keys[i] > prefix;
        same += prefix != 0 && keys[i] == prefix;
    }
    uint32_t total;
    const uint32_t same_before = wg_scan_add(same, s->part, &total);
    uint32_t left = same_before < need ? min(need - same_before, same) : 0u;
    uint32_t rank = wg_scan_add(over + left, s->part, &total);
    for (int i = i0; i < i1; ++i) {
        bool in = keys[i] > prefix;
        if (!in && left > 0 && keys[i] == prefix) {
            in = true;
            --left;
        }
        if (in) emit(i, (int)rank++);
    }
    return (int)total;
}

// ---------------------------------------------------------------- selection of blocks
struct KvSelectArgs {
    KvCacheView c;
    KvBatchView b;
    const void* q;
    int64_t q_stride;
    int32_t bf16, group, causal;
    const uint64_t* mask;
    int32_t mask_words, n_sel, sink, recent;
    int32_t tiles, chunks;  // of 16 tokens, of kKvScoreBlocks blocks
    int64_t key_stride;
    uint32_t* keys;         // [n_tok, n_heads, key_stride]
    int32_t* out;
};

constexpr int kKvScoreBlocks = 256;  // blocks of a workgroup

// The group's queries of one token as int8 [2 d]: this lane's 16 bytes of each 64 (lane = token n, quarter g).
template <int D>
__device__ inline void kv_query_bytes(const KvSelectArgs& a, int64_t tok, int head, bool valid, int g, int4v* out)
{
    constexpr int kSteps = 2 * D / 64;
    float u[kSteps][16];
    float top = 0.0f;
    const uint16_t* q = (const uint16_t*)a.q + tok * a.q_stride + (int64_t)head * a.group * D;
    const bool bf16 = a.bf16 != 0;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
        const int at = c * 64 + g * 16, ch = at % D;
        const bool neg = at >= D;
#pragma unroll
        for (int j = 0; j < 16; ++j) u[c][j] = 0.0f;
        if (valid)
            for (int h = 0; h < a.group; ++h) {
                float f[16];
                eight_floats(*(const uint4*)(q + h * D + ch), bf16, f);
                eight_floats(*(const uint4*)(q + h * D + ch + 8), bf16, f + 8);
#pragma unroll
                for (int j = 0; j < 16; ++j) u[c][j] = __fadd_rn(u[c][j], neg ? fminf(f[j], 0.0f) : fmaxf(f[j], 0.0f));
            }
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, fabsf(u[c][j]));
    }
    top = max_over_16_32(top);
    const float unit = __fdiv_rn(top, 127.0f);
#pragma unroll
    for (int c = 0; c < kSteps; ++c)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t r = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) r |= (uint32_t)(kv_quant(u[c][4 * w + j], unit) & 255) << (8 * j);
            out[c][w] = (int)r;
        }
}

// Keys of (token, head, block): one int8 product of 16 blocks' bounds with 16 tokens' queries to an instruction.
// Bound by the bounds, read once for every 16 tokens of a sequence.
template <int D>
__global__ __launch_bounds__(kKvThreads) void kv_score_kernel(KvSelectArgs a)
{
    constexpr int kSteps = 2 * D / 64;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    int64_t at = blockIdx.x;
    const int chunk = (int)(at % a.chunks);
    at /= a.chunks;
    const int tile = (int)(at % a.tiles);
    at /= a.tiles;
    const int head = (int)(at % a.c.n_heads), s = (int)(at / a.c.n_heads);
    const KvSeq q = kv_seq(a.b, s);
    const int i = tile * 16 + n;
    if (tile * 16 >= q.count) return;
    const bool valid = i < q.count;
    const int64_t tok = (int64_t)q.first + min(i, q.count - 1);
    const int lim = valid ? max(0, a.causal ? q.len - (q.count - 1 - i) : q.len) : 0;
    const int seen = (lim + kKvBlock - 1) / kKvBlock;  // blocks of this token
    // (every block of the stride gets a key, so that the choice finds zeros behind the last)
    const int b0 = chunk * kKvScoreBlocks, b1 = min(b0 + kKvScoreBlocks, (q.len + kKvBlock - 1) / kKvBlock);
    if (b0 >= b1) return;
    int4v u[kSteps];
    kv_query_bytes<D>(a, tok, head, valid, g, u);
    for (int bt = b0 + w * 16; bt < b1; bt += 64) {
        const int b = bt + n;
        const int page = b < b1 ? kv_page(a.c, a.b, s, b) : -1;
        const int64_t ph = (int64_t)max(page, 0) * a.c.n_heads + head;
        const float ks = page >= 0 ? a.c.k_scale[ph] : 0.0f;
        int4v acc = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            int4v row = {0, 0, 0, 0};
            if (page >= 0) row = *(const int4v*)(a.c.bounds + ph * (2 * D) + c * 64 + g * 16);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(row, u[c], acc, 0, 0, 0);
        }
        uint32_t key[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int from = g * 4 + r, bb = bt + from;
            const float scale = __shfl(ks, from);
            const int there = __shfl(page, from);
            bool can = valid && bb < seen && there >= 0;
            if (a.mask && can) {
                uint64_t word = a.mask[tok * a.mask_words + bb];
                const int left = lim - bb * kKvBlock;
                if (left < 64) word &= (1ull << left) - 1;
                can = word != 0;
            }
            const uint32_t k = min(max(score_bits(__fmul_rn((float)acc[r], scale)), 1u), 0xFFFFFFFEu);
            key[r] = !can ? 0u : bb < a.sink || bb >= seen - a.recent ? 0xFFFFFFFFu : k;
        }
        if (valid) *(uint4*)(a.keys + (tok * a.c.n_heads + head) * a.key_stride + bt + g * 4) = make_uint4(key[0], key[1], key[2], key[3]);
    }
}

__global__ __launch_bounds__(kKvThreads) void kv_choose_kernel(KvSelectArgs a)
{
    extern __shared__ uint32_t keys[];
    __shared__ KvPick pick;
    const int64_t th = blockIdx.x;  // (token, head)
    const int tok = (int)(th / a.c.n_heads);
    const int s = kv_seq_of(a.b, tok);
    const KvSeq q = kv_seq(a.b, s);
    int32_t* out = a.out + th * a.n_sel;
    int n = (q.len + kKvBlock - 1) / kKvBlock;
    if (tok < q.first || tok >= q.first + q.count) n = 0;  // a token of no sequence
    for (int i = threadIdx.x; i < n; i += kKvThreads) keys[i] = a.keys[th * a.key_stride + i];
    __syncthreads();
    const int got = kv_pick(keys, n, a.n_sel, &pick, [&](int i, int rank) { out[rank] = i; });
    for (int i = got + threadIdx.x; i < a.n_sel; i += kKvThreads) out[i] = -1;
}

// ---------------------------------------------------------------- eviction
struct KvEvictArgs {
    KvBatchView b;
    const float* mass;
    int32_t n_heads, budget, sink, recent;
    int32_t* tables;
    int32_t* lengths;
    float* out_mass;
    int32_t* freed;
    int32_t* n_freed;
};

// One workgroup to a sequence.  dynamic LDS: a key and an index to each block.  Everything that is read of a row is
// read before the row is written, so that out may be in.
__global__ __launch_bounds__(kKvThreads) void kv_evict_kernel(KvEvictArgs a)
{
    extern __shared__ uint32_t keys[];
    __shared__ KvPick pick;
    const int tid = threadIdx.x, s = blockIdx.x, nb = a.b.max_blocks;
    uint32_t* from = keys + nb;  // block that moves to each place; those that go behind them
    const int len = max(0, min(a.b.lengths[s], a.b.max_len));
    const int n = (len + kKvBlock - 1) / kKvBlock;
    const float* mass = a.mass + (int64_t)s * a.n_heads * nb;
    for (int i = tid; i < n; i += kKvThreads) {
        float m = mass[i];
        for (int h = 1; h < a.n_heads; ++h) m = fmaxf(m, mass[(int64_t)h * nb + i]);
        keys[i] = i < a.sink || i >= n - a.recent ? 0xFFFFFFFFu : min(max(score_bits(m), 1u), 0xFFFFFFFEu);
    }
    __syncthreads();
    const int kept = kv_pick(keys, n, a.budget, &pick, [&](int i, int rank) { from[rank] = (uint32_t)i; });
    __syncthreads();
    // the others, in order: place i of them is block i + (kept blocks before it)
    for (int i = tid; i < n; i += kKvThreads) keys[i] = 0;
    __syncthreads();
    for (int r = tid; r < kept; r += kKvThreads) keys[from[r]] = 1;
    __syncthreads();
    const int per = (n + kKvThreads - 1) / kKvThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    uint32_t gone = 0;
    for (int i = i0; i < i1; ++i) gone += keys[i] == 0;
    uint32_t total;
    uint32_t rank = wg_scan_add(gone, pick.part, &total);
    for (int i = i0; i < i1; ++i)
        if (keys[i] == 0) from[kept + rank++] = (uint32_t)i;
    __syncthreads();
    const int32_t* old = a.b.tables + (int64_t)s * nb;
    for (int r = tid; r < n - kept; r += kKvThreads) a.freed[(int64_t)s * nb + r] = old[from[kept + r]];
    for (int r = n - kept + tid; r < nb; r += kKvThreads) a.freed[(int64_t)s * nb + r] = -1;
    // rows close up: a round of places reads what lies at or behind it, so a barrier between reading and writing will do
    for (int h = -1; h < a.n_heads; ++h) {
        const uint32_t* src = h < 0 ? (const uint32_t*)old : (const uint32_t*)(mass + (int64_t)h * nb);
        uint32_t* dst = h < 0 ? (uint32_t*)(a.tables + (int64_t)s * nb)
                              : (uint32_t*)(a.out_mass + ((int64_t)s * a.n_heads + h) * nb);
        const uint32_t none = h < 0 ? 0xFFFFFFFFu : 0u;
        for (int r0 = 0; r0 < nb; r0 += kKvThreads) {
            const int r = r0 + tid;
            const uint32_t v = r < kept ? src[from[r]] : none;
            __syncthreads();
            if (r < nb) dst[r] = v;
        }
        __syncthreads();
    }
    if (tid == 0) {
        a.lengths[s] = len - (n - kept) * kKvBlock;
        a.n_freed[s] = n - kept;
    }
}

}  // namespace st
