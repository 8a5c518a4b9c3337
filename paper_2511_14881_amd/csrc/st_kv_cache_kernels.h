// Writing, reading, searching and shrinking the cache of histories (layout: silvertorch.h).
#pragma once
#include "st_kv_device.h"

namespace st {

// ---------------------------------------------------------------- append
// New rows are quantised with the page's scale as it becomes, older integers move to it when it grows (round(q * o / s): a
// block has one scale, so they have to).  One workgroup to a page, head and kind (keys or values), a thread to four
// neighbouring tokens and eight channels: each row is read once and stays in registers until its scale is known.  Bound by
// latency for single tokens (a chain of loads, a reduction over the workgroup, the stores), by HBM for prompts.  64 sequences,
// a token each, 8 heads of 128: 7.6 us; 3 x 4097 tokens: 28 us, 75 MB in and out.
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
__device__ inline uint4 kv_moved16(uint4 w, float ratio)
{
    return make_uint4(kv_moved4(w.x, ratio), kv_moved4(w.y, ratio), kv_moved4(w.z, ratio), kv_moved4(w.w, ratio));
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
    constexpr int kGroups = D / 8;                                              // of eight channels
    constexpr int kItems = (16 * kGroups + kKvThreads - 1) / kKvThreads;        // (four tokens, eight channels) of a thread
    constexpr int kPieces = (D * kKvBlock / 16 + kKvThreads - 1) / kKvThreads;  // 16 bytes of a page's integers
    constexpr int kRow = kKvBlock / 4 + 1;                                      // words of a channel's row in the LDS
    __shared__ uint32_t tile[D * kRow];
    __shared__ float s_max[kKvThreads / 64];
    const int tid = threadIdx.x;
    const bool values = blockIdx.x & 1;
    const int at = blockIdx.x >> 1;
    const int head = at % a.c.n_heads, rest = at / a.c.n_heads;
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
    const uint16_t* src = (const uint16_t*)(values ? a.v_new : a.k_new) + head * D;
    const int64_t stride = values ? a.v_stride : a.k_stride;
    uint4* page16 = (uint4*)((values ? a.c.v : a.c.k) + ph * (D * kKvBlock));
    float* scale = (values ? a.c.v_scale : a.c.k_scale) + ph;

    uint4 x[kItems][4];
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = i * kKvThreads + tid, t0 = item / kGroups * 4, c = item % kGroups * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[i][j] = make_uint4(0, 0, 0, 0);
            if (t0 + j >= p0 && t0 + j < p1) x[i][j] = *(const uint4*)(src + (row0 + t0 + j) * stride + c);
        }
    }
    uint4 old16[kPieces];
    if (values && p0 > 0)
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            if (i * kKvThreads + tid < D * kKvBlock / 16) old16[i] = page16[i * kKvThreads + tid];
    uint2 old8[kItems][4];  // older keys of the same tokens and channels: the bounds are theirs too
    if (!values && p0 > 0)
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int item = i * kKvThreads + tid, t0 = item / kGroups * 4, c = item % kGroups * 8;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t0 + j < p0) old8[i][j] = *(const uint2*)((const int8_t*)page16 + (t0 + j) * D + c);
        }
    const float old = p0 > 0 ? *scale : 0.0f;
#pragma unroll
    for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float f[8];
            eight_floats(x[i][j], bf16, f);
#pragma unroll
            for (int u = 0; u < 8; ++u) top = fmaxf(top, fabsf(f[u]));
        }
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if ((tid & 63) == 0) s_max[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    const float sc = fmaxf(old, __fdiv_rn(top, 127.0f));
    const float ratio = sc > 0.0f ? __fdiv_rn(old, sc) : 0.0f;
    if (tid == 0) *scale = sc;

    if (values) {
        if (p0 > 0) {  // (all slots: those that hold no token do not matter)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int p = i * kKvThreads + tid;
                if (p >= D * kKvBlock / 16) continue;
                const uint4 w = ratio != 1.0f ? kv_moved16(old16[i], ratio) : old16[i];
                uint32_t* to = tile + p / 4 * kRow + p % 4 * 4;
                to[0] = w.x;
                to[1] = w.y;
                to[2] = w.z;
                to[3] = w.w;
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int item = i * kKvThreads + tid, t0 = item / kGroups * 4, c = item % kGroups * 8;
            if (t0 + 4 <= p0 || t0 >= p1) continue;
            float f[4][8];
#pragma unroll
            for (int j = 0; j < 4; ++j) eight_floats(x[i][j], bf16, f[j]);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                uint32_t* word = tile + (c + u) * kRow + kv_slot(t0) / 4;
                uint32_t w = t0 < p0 ? *word : 0u;  // a word may hold older tokens
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t0 + j >= p0) w = (w & ~(255u << (8 * j))) | (uint32_t)(kv_quant(f[j][u], sc) & 255) << (8 * j);
                *word = w;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = i * kKvThreads + tid;
            if (p >= D * kKvBlock / 16) continue;
            const uint32_t* from = tile + p / 4 * kRow + p % 4 * 4;
            page16[p] = make_uint4(from[0], from[1], from[2], from[3]);
        }
        return;
    }

    // keys: rows of older tokens where the scale grew, rows of new ones, and the bounds of both
    int8_t* limits = (int8_t*)tile;  // [16][2][D]: of each four tokens
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = i * kKvThreads + tid, t0 = item / kGroups * 4, c = item % kGroups * 8;
        if (t0 >= p1) continue;
        int hi[8], lo[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            hi[u] = -128;
            lo[u] = 127;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (t0 + j >= p1) continue;
            const bool older = t0 + j < p0;
            uint32_t w[2] = {0, 0};
            if (older) {
                w[0] = ratio != 1.0f ? kv_moved4(old8[i][j].x, ratio) : old8[i][j].x;
                w[1] = ratio != 1.0f ? kv_moved4(old8[i][j].y, ratio) : old8[i][j].y;
            } else {
                float f[8];
                eight_floats(x[i][j], bf16, f);
#pragma unroll
                for (int u = 0; u < 8; ++u) w[u / 4] |= (uint32_t)(kv_quant(f[u], sc) & 255) << (8 * (u & 3));
            }
            if (!older || ratio != 1.0f) *(uint2*)((int8_t*)page16 + (t0 + j) * D + c) = make_uint2(w[0], w[1]);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int v = (int8_t)(w[u / 4] >> (8 * (u & 3)));
                hi[u] = max(hi[u], v);
                lo[u] = min(lo[u], v);
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            limits[t0 / 4 * (2 * D) + c + u] = (int8_t)hi[u];
            limits[t0 / 4 * (2 * D) + D + c + u] = (int8_t)lo[u];
        }
    }
    __syncthreads();
    for (int c = tid; c < 2 * D; c += kKvThreads) {
        int v = limits[c];
        for (int t = 1; t * 4 < p1; ++t) {
            const int other = limits[t * (2 * D) + c];
            v = c < D ? max(v, other) : min(v, other);
        }
        a.c.bounds[ph * (2 * D) + c] = (int8_t)v;
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

__device__ inline float4v kv_floats(uint32_t w, float sc)
{
    return float4v{(float)(int8_t)w * sc, (float)(int8_t)(w >> 8) * sc, (float)(int8_t)(w >> 16) * sc, (float)(int8_t)(w >> 24) * sc};
}

// One workgroup to a page, head and kind.  Bound by the floats it writes, which go past the caches (as fast as if they did not).
// 3 x 4097 tokens, 8 heads of 128: 20 us, 130 MB in and out, 6.5 TB/s.
template <int D>
__global__ __launch_bounds__(kKvThreads) void kv_read_kernel(KvReadArgs a)
{
    const int tid = threadIdx.x;
    const bool values = blockIdx.x & 1;
    const int64_t out = blockIdx.x >> 1;  // (s, j, head)
    const int head = (int)(out % a.c.n_heads);
    const int64_t rest = out / a.c.n_heads;
    const int j = (int)(rest % a.n_blocks), s = (int)(rest / a.n_blocks);
    const KvSeq q = kv_seq(a.b, s);
    const int held = (q.len + kKvBlock - 1) / kKvBlock;
    const int block = max(0, held - a.n_blocks) + j;
    const int page = block < held ? kv_page(a.c, a.b, s, block) : -1;
    const int n = page < 0 ? 0 : min(kKvBlock, q.len - block * kKvBlock);
    const int64_t ph = (int64_t)max(page, 0) * a.c.n_heads + head;
    const float4v zero = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!values) {
        const float sc = n ? a.c.k_scale[ph] : 0.0f;
        if (a.k) {
            constexpr int kLoads = D * kKvBlock / 4 / kKvThreads;
            const uint32_t* src = (const uint32_t*)(a.c.k + ph * (D * kKvBlock));
            float4v* dst = (float4v*)(a.k + out * (D * kKvBlock));
            uint32_t w[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) w[i] = src[i * kKvThreads + tid];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) __builtin_nontemporal_store((i * kKvThreads + tid) / (D / 4) < n ? kv_floats(w[i], sc) : zero, dst + i * kKvThreads + tid);
        }
        if (a.bounds)
            for (int i = tid; i < 2 * D; i += kKvThreads) a.bounds[out * (2 * D) + i] = n ? (float)a.c.bounds[ph * (2 * D) + i] * sc : 0.0f;
        return;
    }
    if (!a.v) return;
    // four channels' words of four tokens each to a thread: four tokens' rows of four channels
    const float sc = n ? a.c.v_scale[ph] : 0.0f;
    const uint32_t* src = (const uint32_t*)(a.c.v + ph * (D * kKvBlock));
    __shared__ uint32_t tile[D * (kKvBlock / 4 + 1)];
    if (n) {
#pragma unroll
        for (int i = 0; i < D * kKvBlock / 4 / kKvThreads; ++i) {
            const int at = i * kKvThreads + tid;
            tile[at / 16 * 17 + at % 16] = src[at];
        }
    }
    __syncthreads();
    float* dst = a.v + out * (D * kKvBlock);
    for (int i = tid; i < 16 * (D / 4); i += kKvThreads) {
        const int t0 = i / (D / 4) * 4, c = i % (D / 4) * 4, word = kv_slot(t0) / 4;
        float4v f[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) f[u] = n ? kv_floats(tile[(c + u) * 17 + word], sc) : zero;
#pragma unroll
        for (int t = 0; t < 4; ++t)
            __builtin_nontemporal_store((t0 + t < n ? float4v{f[0][t], f[1][t], f[2][t], f[3][t]} : zero), (float4v*)(dst + (t0 + t) * D + c));
    }
}

// ---------------------------------------------------------------- the best n of an array of keys
// Marks the `want` largest keys (0: not to be had; equal keys: the lower index first) of keys[0 .. n) by a walk over
// their four bytes from the top, and hands each marked index to emit(index, rank), rank counting the marked ones in index order.
// Returns how many there are.  All threads of the workgroup.
template <int kThreads>
struct KvPick {
    uint32_t hist[2][256];
    uint32_t part[2][kThreads / 64];
    uint32_t found[2];  // where the want-th key lies: its bytes so far, and how many of those are wanted
    uint32_t state;     // 1: all keys of these bytes are
};

template <int kThreads>
__device__ inline uint32_t wg_scan_add(uint32_t v, uint32_t* part, uint32_t* total)  // exclusive
{
    const int tid = threadIdx.x, w = tid >> 6;
    const uint32_t inc = wave_scan_add(v);
    if ((tid & 63) == 63) part[w] = inc;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) {
        const uint32_t p = part[i];
        before += i < w ? p : 0u;
        all += p;
    }
    *total = all;
    return before + inc - v;
}

template <int kThreads, class Emit>
__device__ inline int kv_pick(const uint32_t* keys, int n, int want, KvPick<kThreads>* s, Emit emit)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0, need = (uint32_t)want, total;
    bool ends = false;  // the want-th key is the last of those from prefix up
    for (int i = tid; i < 512; i += kThreads) s->hist[i >> 8][i & 255] = 0;
    if (tid == 0) s->state = 2;
    __syncthreads();
    // each byte: how many keys with the bytes so far have which value, and where the want-th lies
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        uint32_t* hist = s->hist[pass & 1];
        const uint32_t above = pass == 0 ? 0u : 0xFFFFFFFFu << (shift + 8);
        for (int i = tid; i < n; i += kThreads) {
            const uint32_t k = keys[i];
            if (k != 0 && (k & above) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        const uint32_t mine = tid < 256 ? hist[255 - tid] : 0u;
        const uint32_t before = wg_scan_add<kThreads>(mine, s->part[pass & 1], &total);
        if (pass == 0 && total < need) {  // fewer keys than wanted: all of them
            prefix = 1;
            ends = true;
            break;
        }
        if (before < need && before + mine >= need) {
            s->found[0] = prefix | ((uint32_t)(255 - tid) << shift);
            s->found[1] = need - before;
            s->state = before + mine == need ? 1 : 0;
        }
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        prefix = s->found[0];
        need = s->found[1];
        ends = s->state == 1;
        if (ends) break;
    }
    // keys above prefix are in, and the first `need` of those equal to it (all of them from prefix up where it ends there)
    if (ends) {
        prefix = max(prefix, 1u) - 1;
        need = 0;
    }
    const int per = (n + kThreads - 1) / kThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    uint32_t over = 0, same = 0;
    for (int i = i0; i < i1; ++i) {
        over += keys[i] > prefix;
        same += keys[i] == prefix;
    }
    uint32_t left = 0;
    __syncthreads();
    if (need > 0) {
        const uint32_t same_before = wg_scan_add<kThreads>(same, s->part[0], &total);
        left = same_before < need ? min(need - same_before, same) : 0u;
    }
    uint32_t rank = wg_scan_add<kThreads>(over + left, s->part[1], &total);
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

// The same for up to 64 * kPer keys by one wavefront, lane l holding keys l * kPer ..: the want-th key is found bit by bit, from
// the first in which keys differ that are neither 0 nor the largest number (those are always in) down to where it is alone.
template <int kPer, class Emit>
__device__ inline int kv_pick_wave(const uint32_t (&keys)[kPer], int want, Emit emit)
{
    // (counted in the lanes and summed across them: ballots would go through the scalar unit one by one)
    auto all = [](uint32_t v) { return (int)lane_value(wave_scan_add(v), 63); };
    uint32_t ones = 0, zeros = 0, over = 0, same = 0, mine = 0, open = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const bool is_open = keys[i] != 0 && keys[i] != 0xFFFFFFFFu;
        ones |= is_open ? keys[i] : 0u;
        zeros |= is_open ? ~keys[i] : 0u;
        mine += keys[i] == 0xFFFFFFFFu;
        open += is_open;
    }
    const int sure = all(mine), some = all(open);
    ones = lane_value(wave_or_u32(ones), 63);
    zeros = lane_value(wave_or_u32(zeros), 63);
    const uint32_t differ = ones & zeros;
    const int top = 31 - __builtin_clz(differ | 1u);
    uint32_t t;
    if (sure >= want) t = 0xFFFFFFFFu;
    else if (sure + some <= want) t = 1;  // no more than wanted: all of them
    else {
        t = differ ? ones & ~((2u << top) - 1u) : ones;  // what all of them share
#pragma unroll 1
        for (int bit = differ ? top : -1; bit >= 0; --bit) {
            const uint32_t c = t | 1u << bit;
            mine = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) mine += keys[i] >= c;
            const int count = all(mine);
            if (count >= want) t = c;
            if (count == want) break;
        }
    }
    // those above t are in, and of those equal to t the first that are left to be had
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        over += keys[i] > t;
        same += keys[i] == t;
    }
    const uint32_t need = (uint32_t)max(want - all(over), 0);
    const uint32_t same_before = wave_scan_add(same) - same;
    uint32_t left = same_before < need ? min(need - same_before, same) : 0u;
    const uint32_t inc = wave_scan_add(over + left);
    uint32_t rank = inc - (over + left);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        bool in = keys[i] > t;
        if (!in && left > 0 && keys[i] == t) {
            in = true;
            --left;
        }
        if (in) emit(i, (int)rank++);
    }
    return (int)lane_value(inc, 63);
}

// One wavefront's keys from a row that is a multiple of 16 long, and the blocks it chooses.
template <int kPer>
__device__ inline void kv_choose_row(const uint32_t* row, int n, int want, int32_t* out)
{
    static_assert(kPer % 4 == 0, "whole loads");
    const int lane = threadIdx.x & 63;
    uint32_t keys[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
        const int b = lane * kPer + i;
        uint4 k = make_uint4(0, 0, 0, 0);
        if (b < n) k = *(const uint4*)(row + b);
        keys[i] = k.x;
        keys[i + 1] = b + 1 < n ? k.y : 0u;
        keys[i + 2] = b + 2 < n ? k.z : 0u;
        keys[i + 3] = b + 3 < n ? k.w : 0u;
    }
    const int got = kv_pick_wave<kPer>(keys, want, [&](int i, int rank) { out[rank] = lane * kPer + i; });
    for (int i = got + lane; i < want; i += 64) out[i] = -1;
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
    int32_t tiles, chunks, rounds;  // of 16 tokens, of `rounds` times kKvScoreBlocks blocks
    int64_t key_stride;
    uint32_t* keys;         // [n_tok, n_heads, key_stride]
    int32_t* out;
};

constexpr int kKvScoreBlocks = 256;  // blocks of a workgroup's round

// Queries of up to 16 tokens as int8 [token][2 d], each the group's positive parts and its negative ones, into the LDS.
// A thread to eight channels of a token.
template <int D, int kThreads>
__device__ inline void kv_query_bytes(const KvSelectArgs& a, int64_t tok0, int tokens, int head, int8_t* out, int out_stride, uint32_t* tops)
{
    constexpr int kGroups = D / 8, kItems = (16 * kGroups + kThreads - 1) / kThreads;
    const int tid = threadIdx.x;
    const bool bf16 = a.bf16 != 0;
    if (tid < 16) tops[tid] = 0;
    __syncthreads();
    float u[kItems][16];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = i * kThreads + tid, t = item / kGroups, c = item % kGroups * 8;
        if (t >= tokens) continue;
        const uint16_t* q = (const uint16_t*)a.q + (tok0 + t) * a.q_stride + (int64_t)head * a.group * D + c;
#pragma unroll
        for (int j = 0; j < 16; ++j) u[i][j] = 0.0f;
        for (int h = 0; h < a.group; h += 4) {
            uint4 raw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) raw[k] = h + k < a.group ? *(const uint4*)(q + (h + k) * D) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < 4; ++k) {  // (a row of zeros behind the last head changes no sum)
                float f[8];
                eight_floats(raw[k], bf16, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    u[i][j] = __fadd_rn(u[i][j], fmaxf(f[j], 0.0f));
                    u[i][8 + j] = __fadd_rn(u[i][8 + j], fminf(f[j], 0.0f));
                }
            }
        }
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, fabsf(u[i][j]));
        atomicMax(&tops[t], __float_as_uint(top));  // (floats from 0 up order as their bits)
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = i * kThreads + tid, t = item / kGroups, c = item % kGroups * 8;
        if (t >= 16) continue;
        uint32_t w[4] = {0, 0, 0, 0};
        if (t < tokens) {
            const float unit = __fdiv_rn(__uint_as_float(tops[t]), 127.0f);
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j / 4] |= (uint32_t)(kv_quant(u[i][j], unit) & 255) << (8 * (j & 3));
        }
        *(uint2*)(out + t * out_stride + c) = make_uint2(w[0], w[1]);
        *(uint2*)(out + t * out_stride + D + c) = make_uint2(w[2], w[3]);
    }
    __syncthreads();
}

// The same for one token, a thread to a channel; the other 15 rows are zeros.
template <int D, int kThreads>
__device__ inline void kv_query_bytes_of_one(const KvSelectArgs& a, int64_t tok, int head, int8_t* out, int out_stride, uint32_t* tops)
{
    static_assert(D <= kThreads, "a thread to a channel");
    const int tid = threadIdx.x;
    const bool bf16 = a.bf16 != 0;
    float pos = 0.0f, neg = 0.0f;
    if (tid < D) {
        const uint16_t* q = (const uint16_t*)a.q + tok * a.q_stride + (int64_t)head * a.group * D + tid;
        for (int h = 0; h < a.group; h += 4) {
            uint32_t raw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) raw[k] = h + k < a.group ? q[(h + k) * D] : 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = bf16 ? bf16_float(raw[k]) : f16_float(raw[k]);
                pos = __fadd_rn(pos, fmaxf(f, 0.0f));
                neg = __fadd_rn(neg, fminf(f, 0.0f));
            }
        }
    }
    for (int i = tid; i < 16 * out_stride / 4; i += kThreads) ((uint32_t*)out)[i] = 0;
    const uint32_t top = wave_max_u32(__float_as_uint(fmaxf(pos, -neg)));  // (floats from 0 up order as their bits)
    if (tid < 16) tops[tid] = 0;
    __syncthreads();
    if (lane_id() == 63 && tid < D + 63) atomicMax(&tops[0], top);
    __syncthreads();
    if (tid < D) {
        const float unit = __fdiv_rn(__uint_as_float(tops[0]), 127.0f);
        out[tid] = (int8_t)kv_quant(pos, unit);
        out[D + tid] = (int8_t)kv_quant(neg, unit);
    }
    __syncthreads();
}

// Keys of (token, head, block): one int8 product of 16 blocks' bounds with 16 tokens' queries to an instruction.
// Bound by the bounds, read once for every 16 tokens of a sequence.  kOne: sequences have one token each, and the workgroup that
// has formed the keys of all blocks chooses among them in its LDS.  800 tokens over 20001 of 8 sequences, 4 heads of 128: 13 us;
// 16 tokens over 65536 each, 8 heads, with the choice of 64 blocks of 1024: 18 us, of which the bounds' 21 MB take 3.5.
template <int D, bool kOne, int kThreads>
__global__ __launch_bounds__(kThreads) void kv_score_kernel(KvSelectArgs a)
{
    constexpr int kSteps = 2 * D / 64, kStride = 2 * D + 16, kAt = D > 128 ? 2 : 4;  // (tiles of 16 blocks at a time)
    extern __shared__ uint32_t keys[];
    __shared__ __align__(16) int8_t s_u[16 * kStride];
    __shared__ uint32_t s_top[16];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    int64_t at = blockIdx.x;
    const int chunk = (int)(at % a.chunks);
    at /= a.chunks;
    const int tile = (int)(at % a.tiles);
    at /= a.tiles;
    const int head = (int)(at % a.c.n_heads), s = (int)(at / a.c.n_heads);
    const KvSeq q = kv_seq(a.b, s);
    if (tile * 16 >= q.count) return;
    const int held = (q.len + kKvBlock - 1) / kKvBlock;
    const int round = kOne ? held : kKvScoreBlocks * a.rounds;
    const int b0 = chunk * round, b1 = min(b0 + round, held);
    if (!kOne && b0 >= b1) return;
    const int64_t tok0 = (int64_t)q.first + tile * 16;
    const int tokens = min(16, q.count - tile * 16);
    const int i = tile * 16 + n;
    const bool valid = n < tokens;
    const int64_t tok = tok0 + (valid ? n : 0);
    const int lim = valid ? max(0, a.causal ? q.len - (q.count - 1 - i) : q.len) : 0;
    const int seen = (lim + kKvBlock - 1) / kKvBlock;  // blocks of this token
    // 64 blocks of a wavefront's round, one to a lane; the page is asked for a round ahead
    const int32_t* table = a.b.tables + (int64_t)s * a.b.max_blocks;
    int entry = b0 < b1 ? table[min(b0 + w * 64 + lane, b1 - 1)] : -1;
    if (kOne) kv_query_bytes_of_one<D, kThreads>(a, tok0, head, s_u, kStride, s_top);
    else kv_query_bytes<D, kThreads>(a, tok0, tokens, head, s_u, kStride, s_top);
    int4v u[kSteps];
#pragma unroll
    for (int c = 0; c < kSteps; ++c) u[c] = *(const int4v*)(s_u + n * kStride + c * 64 + g * 16);
    for (int bw = b0 + w * 64; bw < b1; bw += kThreads) {
        const int page_l = bw + lane < b1 ? kv_page_of(a.c, entry) : -1;
        const float ks_l = a.c.k_scale[(int64_t)max(page_l, 0) * a.c.n_heads + head];  // (not used where there is no page)
#pragma unroll
        for (int t0 = 0; t0 < 4; t0 += kAt) {
            int4v row[kAt][kSteps];
            uint64_t word[kAt][4];
#pragma unroll
            for (int t = 0; t < kAt; ++t) {
                const int page = __shfl(page_l, (t0 + t) * 16 + n);
                const int8_t* src = a.c.bounds + ((int64_t)max(page, 0) * a.c.n_heads + head) * (2 * D) + g * 16;
#pragma unroll
                for (int c = 0; c < kSteps; ++c) row[t][c] = *(const int4v*)(src + c * 64);
                if (a.mask)
#pragma unroll
                    for (int r = 0; r < 4; ++r) word[t][r] = a.mask[tok * a.mask_words + min(bw + (t0 + t) * 16 + g * 4 + r, held - 1)];
            }
#pragma unroll
            for (int t = 0; t < kAt; ++t) {
                if (t0 + t == 0) entry = table[min(bw + kThreads + lane, b1 - 1)];
                const int bt = bw + (t0 + t) * 16;
                int4v acc = {0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < kSteps; ++c) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(row[t][c], u[c], acc, 0, 0, 0);
                uint32_t key[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int from = (t0 + t) * 16 + g * 4 + r, bb = bw + from;
                    const float scale = __shfl(ks_l, from);
                    bool can = __shfl(page_l, from) >= 0 && bb < seen;
                    if (a.mask && can) {
                        const int left = lim - bb * kKvBlock;
                        can = (left < 64 ? word[t][r] & ((1ull << left) - 1) : word[t][r]) != 0;
                    }
                    const uint32_t k = min(max(score_bits(__fmul_rn((float)acc[r], scale)), 1u), 0xFFFFFFFEu);
                    key[r] = !can ? 0u : bb < a.sink || bb >= seen - a.recent ? 0xFFFFFFFFu : k;
                }
                if (bt >= b1) continue;
                // (every block of a tile gets a key, so that the choice finds zeros behind the last)
                if (kOne) {
                    if (n == 0) *(uint4*)(keys + bt + g * 4) = make_uint4(key[0], key[1], key[2], key[3]);
                } else if (valid) {
                    *(uint4*)(a.keys + (tok * a.c.n_heads + head) * a.key_stride + bt + g * 4) = make_uint4(key[0], key[1], key[2], key[3]);
                }
            }
        }
    }
    if (!kOne) return;
    __shared__ KvPick<kThreads> pick;
    int32_t* out = a.out + (tok0 * a.c.n_heads + head) * a.n_sel;
    __syncthreads();
    if (held <= 1024) {  // (one wavefront without a barrier: 2 us less than all of them at 1024 blocks)
        if (w != 0) return;
        if (held <= 256) kv_choose_row<4>(keys, held, a.n_sel, out);
        else kv_choose_row<16>(keys, held, a.n_sel, out);
        return;
    }
    const int got = kv_pick<kThreads>(keys, held, a.n_sel, &pick, [&](int b, int rank) { out[rank] = b; });
    for (int b = got + threadIdx.x; b < a.n_sel; b += kThreads) out[b] = -1;
}

__global__ __launch_bounds__(kKvThreads) void kv_choose_kernel(KvSelectArgs a)
{
    extern __shared__ uint32_t keys[];
    __shared__ KvPick<kKvThreads> pick;
    const int64_t th = blockIdx.x;  // (token, head)
    const int tok = (int)(th / a.c.n_heads);
    const KvSeq q = kv_seq(a.b, kv_seq_of(a.b, tok));
    int32_t* out = a.out + th * a.n_sel;
    int n = (q.len + kKvBlock - 1) / kKvBlock;
    if (tok < q.first || tok >= q.first + q.count) n = 0;  // a token of no sequence
    for (int i = threadIdx.x; i < n; i += kKvThreads) keys[i] = a.keys[th * a.key_stride + i];
    __syncthreads();
    const int got = kv_pick<kKvThreads>(keys, n, a.n_sel, &pick, [&](int i, int rank) { out[rank] = i; });
    for (int i = got + threadIdx.x; i < a.n_sel; i += kKvThreads) out[i] = -1;
}

// Up to 64 * kPer blocks: one wavefront to a token and head, its keys in registers.  3200 of them, 8 of 313 blocks: 7 us.
template <int kPer>
__global__ __launch_bounds__(kKvThreads) void kv_choose_wave_kernel(KvSelectArgs a)
{
    const int64_t th = (int64_t)blockIdx.x * (kKvThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (th >= (int64_t)a.b.n_tok * a.c.n_heads) return;
    const int tok = (int)(th / a.c.n_heads);
    const KvSeq q = kv_seq(a.b, kv_seq_of(a.b, tok));
    int32_t* out = a.out + th * a.n_sel;
    int n = (q.len + kKvBlock - 1) / kKvBlock;
    if (tok < q.first || tok >= q.first + q.count) n = 0;  // a token of no sequence
    kv_choose_row<kPer>(a.keys + th * a.key_stride, n, a.n_sel, out);
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

constexpr int kKvEvictThreads = 1024;

// One workgroup to a sequence; dynamic LDS: a key and an index to each block.  Bound by latency: the weights once through, a
// choice in the LDS, and the rows that close up.  A round of places reads what lies at or behind it, for up to
// eight rows at a time, before it writes, so that out may be in.  64 sequences of 1024 blocks, 8 heads, cut to half: 12.7 us.
__global__ __launch_bounds__(kKvEvictThreads) void kv_evict_kernel(KvEvictArgs a)
{
    extern __shared__ uint32_t keys[];
    __shared__ KvPick<kKvEvictThreads> pick;
    const int tid = threadIdx.x, s = blockIdx.x, nb = a.b.max_blocks;
    uint32_t* from = keys + nb;  // block that moves to each place; those that go behind them
    const int len = max(0, min(a.b.lengths[s], a.b.max_len));
    const int n = (len + kKvBlock - 1) / kKvBlock;
    const float* mass = a.mass + (int64_t)s * a.n_heads * nb;
    for (int i = tid; i < n; i += kKvEvictThreads) {
        float m = mass[i];
#pragma unroll 8
        for (int h = 1; h < a.n_heads; ++h) m = fmaxf(m, mass[(int64_t)h * nb + i]);
        keys[i] = i < a.sink || i >= n - a.recent ? 0xFFFFFFFFu : min(max(score_bits(m), 1u), 0xFFFFFFFEu);
    }
    __syncthreads();
    const int kept = kv_pick<kKvEvictThreads>(keys, n, a.budget, &pick, [&](int i, int rank) { from[rank] = (uint32_t)i; });
    __syncthreads();
    // the others, in order
    for (int i = tid; i < n; i += kKvEvictThreads) keys[i] = 0;
    __syncthreads();
    for (int r = tid; r < kept; r += kKvEvictThreads) keys[from[r]] = 1;
    __syncthreads();
    const int per = (n + kKvEvictThreads - 1) / kKvEvictThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    uint32_t gone = 0;
    for (int i = i0; i < i1; ++i) gone += keys[i] == 0;
    uint32_t total;
    uint32_t rank = wg_scan_add<kKvEvictThreads>(gone, pick.part[0], &total);
    for (int i = i0; i < i1; ++i)
        if (keys[i] == 0) from[kept + rank++] = (uint32_t)i;
    __syncthreads();
    const int32_t* old = a.b.tables + (int64_t)s * nb;
    for (int r = tid; r < nb; r += kKvEvictThreads) a.freed[(int64_t)s * nb + r] = r < n - kept ? old[from[kept + r]] : -1;
    for (int h0 = -1; h0 < a.n_heads; h0 += 8) {  // row -1: the table
        for (int r0 = 0; r0 < nb; r0 += kKvEvictThreads) {
            const int r = r0 + tid;
            const uint32_t f = r < kept ? from[r] : 0u;
            uint32_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int h = h0 + u;
                v[u] = h < 0 ? 0xFFFFFFFFu : 0u;
                if (h < a.n_heads && r < kept) v[u] = h < 0 ? (uint32_t)old[f] : __float_as_uint(mass[(int64_t)h * nb + f]);
            }
            __syncthreads();
            if (r < nb)
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int h = h0 + u;
                    if (h >= a.n_heads) continue;
                    if (h < 0) a.tables[(int64_t)s * nb + r] = (int32_t)v[u];
                    else a.out_mass[((int64_t)s * a.n_heads + h) * nb + r] = __uint_as_float(v[u]);
                }
        }
    }
    if (tid == 0) {
        a.lengths[s] = len - (n - kept) * kKvBlock;
        a.n_freed[s] = n - kept;
    }
}

}  // namespace st
