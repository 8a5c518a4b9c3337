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
__device__ inline KvSeq kv_seq(const KvBatchView& b, int s)
{
    KvSeq r;
    r.len = max(0, min(b.lengths[s], b.max_len));
    if (b.offsets) {
        r.first = max(0, min(b.offsets[s], b.n_tok));
        r.count = max(0, min(min(b.offsets[s + 1], b.n_tok) - r.first, b.max_tok));
    } else {
        r.first = s * b.max_tok;
        r.count = b.max_tok;
    }
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
__device__ inline int kv_page(const KvCacheView& c, const KvBatchView& b, int s, int block)
{
    const int p = b.tables[(int64_t)s * b.max_blocks + block];
    return p >= 0 && (int64_t)p < c.n_pages ? p : -1;
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

__device__ inline float max_over_16_32(float v)  // over the lanes that share lane % 16
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ inline float sum_over_16_32(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

}  // namespace st
