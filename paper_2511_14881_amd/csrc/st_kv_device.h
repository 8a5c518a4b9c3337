// What the kernels on cached histories share: the views of cache and batch that travel in kernel arguments,
// conversions between 8, 16 and 32 bits, and steps across a wavefront.
#pragma once
#include "st_device.h"

namespace st {

constexpr int kKvBlock = 64;        // tokens of a page
constexpr int kKvThreads = 256;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef int int4v __attribute__((ext_vector_type(4)));

struct KvCacheView {
    int8_t* k;
    int8_t* v;
    float* k_scale;
    float* v_scale;
    int8_t* bounds;
    int64_t n_pages;
    int32_t n_heads;
};

struct KvBatchView {
    const int32_t* tables;
    const int32_t* lengths;
    const int32_t* offsets;
    int32_t n_seq, max_blocks, n_tok, max_tok, max_len;
};

struct KvSeq {
    int first;  // the sequence's first token of this call
    int count;  // and how many there are
    int len;    // tokens it holds, those included
};

// What a device array says is cut to what the call allows.
__device__ inline void kv_tokens(const KvBatchView& b, int s, int* first, int* count)
{
    if (b.offsets) {
        *first = max(0, min(b.offsets[s], b.n_tok));
        *count = max(0, min(min(b.offsets[s + 1], b.n_tok) - *first, b.max_tok));
    } else {
        *first = s * b.max_tok;
        *count = b.max_tok;
    }
}
__device__ inline KvSeq kv_seq(const KvBatchView& b, int s)
{
    KvSeq r;
    r.len = max(0, min(b.lengths[s], b.max_len));
    kv_tokens(b, s, &r.first, &r.count);
    return r;
}

// The sequence that token `tok` belongs to: the last one whose tokens begin at or before it.
__device__ inline int kv_seq_of(const KvBatchView& b, int tok)
{
    if (!b.offsets) return tok / b.max_tok;
    int lo = 0, hi = b.n_seq - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (b.offsets[mid] <= tok) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Page of block b, -1 where the table names none.
__device__ inline int kv_page_of(const KvCacheView& c, int entry) { return entry >= 0 && (int64_t)entry < c.n_pages ? entry : -1; }
__device__ inline int kv_page(const KvCacheView& c, const KvBatchView& b, int s, int block)
{
    return kv_page_of(c, b.tables[(int64_t)s * b.max_blocks + block]);
}

// Slot of token t of a block in a row of values: bits 5 4 3 2 1 0 of t in the order 3 2 5 4 1 0.
__host__ __device__ inline int kv_slot(int t) { return ((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3); }

__device__ inline float bf16_float(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ inline float f16_float(uint32_t bits)
{
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
// Two 16-bit numbers of a word as floats.
__device__ inline void two_floats(uint32_t w, bool bf16, float* a, float* b)
{
    if (bf16) {
        *a = bf16_float(w & 0xFFFFu);
        *b = __uint_as_float(w & 0xFFFF0000u);
    } else {
        *a = f16_float(w & 0xFFFFu);
        *b = f16_float(w >> 16);
    }
}
__device__ inline void eight_floats(const uint4& w, bool bf16, float* f)
{
    two_floats(w.x, bf16, f, f + 1);
    two_floats(w.y, bf16, f + 2, f + 3);
    two_floats(w.z, bf16, f + 4, f + 5);
    two_floats(w.w, bf16, f + 6, f + 7);
}
// To the nearest 16-bit number, ties to even (NaN stays one).
__device__ inline uint32_t to_16_bits(float f, bool bf16)
{
    if (!bf16) return __builtin_bit_cast(uint16_t, (_Float16)f);
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (u >> 16) | 0x40u;
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// Four int8 as four 16-bit floats, exactly: byte b + 128 put behind the byte 0x64 is the number 1152 + b.
__device__ inline uint2 halves_of_bytes(uint32_t w)
{
    const uint32_t x = w ^ 0x80808080u;
    const half2v c = {(_Float16)1152.0f, (_Float16)1152.0f};
    const half2v a = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) - c;
    const half2v b = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) - c;
    return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
__device__ inline half8 eight_halves(uint32_t lo, uint32_t hi)
{
    const uint2 a = halves_of_bytes(lo), b = halves_of_bytes(hi);
    return __builtin_bit_cast(half8, make_uint4(a.x, a.y, b.x, b.y));
}

// Steps over the lanes that share lane % 16 (or lane % 32), with moves between registers in place of the LDS: a swap of
// rows of 16 (halves of 32) lanes of a value with itself leaves one partner's value in the one result, the other's in the other.
__device__ inline float2 both_of_16(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float2 both_of_32(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_over_32(float v)
{
    const float2 r = both_of_32(v);
    return fmaxf(r.x, r.y);
}
__device__ inline float sum_over_32(float v)
{
    const float2 r = both_of_32(v);
    return r.x + r.y;
}
__device__ inline float max_over_16_32(float v)
{
    const float2 r = both_of_16(v);
    return max_over_32(fmaxf(r.x, r.y));
}
__device__ inline float sum_over_16_32(float v)
{
    const float2 r = both_of_16(v);
    return sum_over_32(r.x + r.y);
}

// sum + the eight 16-bit floats, in fp32.
__device__ inline float add_halves(const half8& p, float sum)
{
    const half2v one = {(_Float16)1.0f, (_Float16)1.0f};
    sum = __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 0, 1), one, sum, false);
    sum = __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 2, 3), one, sum, false);
    sum = __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 4, 5), one, sum, false);
    return __builtin_amdgcn_fdot2(__builtin_shufflevector(p, p, 6, 7), one, sum, false);
}

// Exclusive prefix sum over a workgroup; part: a word for each wavefront.
template <int kThreads>
__device__ inline uint32_t wg_scan_add(uint32_t v, uint32_t* part, uint32_t* total)
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

// x where the bit is 1, -inf where it is 0.
__device__ inline float kv_seen(float x, uint32_t bits, int bit)
{
    const uint32_t yes = (uint32_t)((int)(bits << (31 - bit)) >> 31);
    return __uint_as_float((__float_as_uint(x) & yes) | (0xFF800000u & ~yes));
}

}  // namespace st
