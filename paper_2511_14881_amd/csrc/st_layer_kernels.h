// Rows on their way into and out of the calls on cached histories (definitions: silvertorch.h): the norm that turns
// them into int8, and rotary positions.
#pragma once
#include "st_kv_device.h"

namespace st {

constexpr int kLayerThreads = 256;

// Sums and maxima over 16, 64 or 256 threads, in every one of them: rotations inside rows of 16 lanes, then swaps of rows and halves,
// then four words of the LDS.  Partners add the same two numbers, so all lanes hold the same bits.
template <int N>
__device__ inline float row_ror(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + N, 0xF, 0xF, false));
}
template <int N>
__device__ inline uint32_t row_ror(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xF, 0xF, false);
}
template <int kLanes>
__device__ inline float sum_of_lanes(float v, float* part)
{
    v += row_ror<8>(v);
    v += row_ror<4>(v);
    v += row_ror<2>(v);
    v += row_ror<1>(v);
    if (kLanes >= 64) v = sum_over_16_32(v);
    if (kLanes == 256) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (part[0] + part[1]) + (part[2] + part[3]);
    }
    return v;
}
template <int kLanes>
__device__ inline uint32_t max_of_lanes(uint32_t v, uint32_t* part)
{
    v = max(v, row_ror<8>(v));
    v = max(v, row_ror<4>(v));
    v = max(v, row_ror<2>(v));
    v = max(v, row_ror<1>(v));
    if (kLanes >= 64) {
        auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max((uint32_t)r[0], (uint32_t)r[1]);
        r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max((uint32_t)r[0], (uint32_t)r[1]);
    }
    if (kLanes == 256) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    return v;
}

// To the nearest 16-bit numbers, ties to even (the hardware's conversions; NaN stays one).
template <bool kBf16>
__device__ inline uint16_t one_16(float f)
{
    return kBf16 ? __builtin_bit_cast(uint16_t, (__bf16)f) : __builtin_bit_cast(uint16_t, (_Float16)f);
}
template <bool kBf16>
__device__ inline uint32_t two_16(float a, float b)
{
    return (uint32_t)one_16<kBf16>(a) | (uint32_t)one_16<kBf16>(b) << 16;
}

// Eight neighbouring values of a type as they lie in memory, and as floats.
template <int kType>
struct Eight {
    static constexpr bool kBf16 = kType == ST_BF16;
    uint4 w;
    __device__ void load(const void* p, int64_t at) { w = *(const uint4*)((const uint16_t*)p + at); }
    __device__ void floats(float* f) const { eight_floats(w, kBf16, f); }
    __device__ void wait() { asm volatile("" : "+v"(w.x)); }  // its load has ended behind this
    __device__ static void store(void* p, int64_t at, const float* f)
    {
        *(uint4*)((uint16_t*)p + at) = make_uint4(two_16<kBf16>(f[0], f[1]), two_16<kBf16>(f[2], f[3]), two_16<kBf16>(f[4], f[5]), two_16<kBf16>(f[6], f[7]));
    }
    __device__ static float rounded(float f)
    {
        const uint32_t b = one_16<kBf16>(f);
        return kBf16 ? bf16_float(b) : f16_float(b);
    }
};
template <>
struct Eight<ST_F32> {
    float4 a, b;
    __device__ void load(const void* p, int64_t at)
    {
        a = *(const float4*)((const float*)p + at);
        b = *(const float4*)((const float*)p + at + 4);
    }
    __device__ void floats(float* f) const
    {
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    }
    __device__ void wait() { asm volatile("" : "+v"(a.x), "+v"(b.x)); }
    __device__ static void store(void* p, int64_t at, const float* f)
    {
        *(float4*)((float*)p + at) = make_float4(f[0], f[1], f[2], f[3]);
        *(float4*)((float*)p + at + 4) = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ static float rounded(float f) { return f; }
};

// ---------------------------------------------------------------- norm
struct NormArgs {
    const void* x;
    const void* residual;
    const void* weight;
    void* sum;
    int8_t* q;
    float* scale;
    void* y;
    int64_t x_stride, residual_stride, sum_stride, n_rows;
    int32_t d, normalise;
    float eps;
};

// h = x + residual, t = h w, q = rint(127 t / max |t|), scale = max |t| / 127 / sqrt(mean h^2 + eps): the integers need the row's largest
// magnitude alone, so that the two reductions do not wait for each other's result.  Sums, maximum and products are fp32; h is rounded to the
// type (what the next layer adds to), the quotient to an integer and y to the type.  Bound by memory: a row's threads hold it in registers,
// eight neighbouring values to a vector and kVectors vectors to a thread, so that everything is read and written once.  With residual
// and sum, bf16: 65536 x 2048 175 us (5.4 TB/s), 32768 x 4096 158 (5.9), 16384 x 8192 163, 1048576 x 128 161 (5.8); fp32 65536 x 1024 150; a
// copy reaches 5.04.  The same with other threads to a row: 2048 with 128 or 256 183 and 191, 4096 with 64 or 128 172 and 163, 1024 with 16
// 228, 128 with 16 and more of a row each 267.  Stores past the caches gain 1 to 3 % with 16-bit rows, 5 to 14 % with
// calls that a cache would hold (8000 x 1008, fp16, with the norm's output 12.2 to 10.6), lose 3 % with fp32 rows, and whoever reads the rows next misses
// them (64 x 4096 and the projection behind it 14.1 to 15.4): not used.
template <int kType, int kLanes, int kVectors>
__global__ __launch_bounds__(kLayerThreads) void norm_rows_kernel(NormArgs a)
{
    __shared__ float s_sum[kLayerThreads / 64];
    __shared__ uint32_t s_max[2 * (kLayerThreads / 64)];
    const int lane = threadIdx.x % kLanes;
    const int64_t row = (int64_t)blockIdx.x * (kLayerThreads / kLanes) + threadIdx.x / kLanes;
    const bool live = row < a.n_rows;
    const int64_t at = live ? row : a.n_rows - 1;  // (a wavefront's lanes all take part in its steps)
    const int n8 = a.d >> 3;
    // All loads come first and without conditions (behind a row's end its last vector is read again): one under a condition is waited for
    // before the next, and one behind a store waits for that too.
    Eight<kType> x[kVectors], r[kVectors], w[kVectors];
    int64_t v8[kVectors];
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        v8[i] = min(i * kLanes + lane, n8 - 1) * 8;
        x[i].load(a.x, at * a.x_stride + v8[i]);
    }
    if (a.residual)
#pragma unroll
        for (int i = 0; i < kVectors; ++i) r[i].load(a.residual, at * a.residual_stride + v8[i]);
    if (a.weight)
#pragma unroll
        for (int i = 0; i < kVectors; ++i) w[i].load(a.weight, v8[i]);
#pragma unroll
    for (int i = 0; i < kVectors; ++i) w[i].wait();
    float h[kVectors][8];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        x[i].floats(h[i]);
        if (a.residual) {
            float f[8];
            r[i].floats(f);
#pragma unroll
            for (int u = 0; u < 8; ++u) h[i][u] = Eight<kType>::rounded(h[i][u] + f[u]);
        }
        if (i * kLanes + lane < n8) {
            if (a.sum && live) Eight<kType>::store(a.sum, row * a.sum_stride + v8[i], h[i]);
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) h[i][u] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += h[i][u] * h[i][u];
    }
    float rms = 1.0f;
    if (a.normalise) {
        sum = sum_of_lanes<kLanes>(sum, s_sum);
        float eps = a.eps;
        if (!(sum < 0x1p120f)) {  // (not for NaN either, which stays one); ST_MAX_ROW squares of up to 2^96 are below 2^128
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kVectors; ++i)
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    h[i][u] *= 0x1p-80f;
                    sum += h[i][u] * h[i][u];
                }
            if (kLanes == 256) __syncthreads();  // the words of the sum before are read
            sum = sum_of_lanes<kLanes>(sum, s_sum);
            eps = 0.0f;  // (eps / 2^160 beside at least 2^-54)
        }
        rms = 1.0f / __fsqrt_rn(sum / (float)a.d + eps);
    }
    uint32_t top = 0;  // largest magnitude as its bits, of which NaN's are the largest
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        if (a.weight) {
            float f[8];
            w[i].floats(f);
#pragma unroll
            for (int u = 0; u < 8; ++u) h[i][u] = i * kLanes + lane < n8 ? h[i][u] * f[u] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) top = max(top, __float_as_uint(h[i][u]) & 0x7FFFFFFFu);
    }
    top = max_of_lanes<kLanes>(top, s_max);
    const bool bad = top >= 0x7F800000u || !(rms < __builtin_inff());
    const float unit = __fdiv_rn(__uint_as_float(top), 127.0f);
    const float nan = __uint_as_float(0x7FC00000u);
    if (!live) return;
    if (a.scale && lane == 0) a.scale[row] = bad ? nan : unit * rms;
    const bool zero = bad || !(unit > 0.0f);
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        const int v = i * kLanes + lane;
        if (v >= n8) continue;
        if (a.q) {
            uint32_t w[2] = {0, 0};
            if (!zero)
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    w[u / 4] |= (uint32_t)((int)fminf(fmaxf(rintf(__fdiv_rn(h[i][u], unit)), -127.0f), 127.0f) & 255) << (8 * (u & 3));
            *(uint2*)(a.q + row * a.d + v * 8) = make_uint2(w[0], w[1]);
        }
        if (a.y) {
            float f[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) f[u] = bad ? nan : h[i][u] * rms;
            Eight<kType>::store(a.y, row * a.d + v * 8, f);
        }
    }
}

// ---------------------------------------------------------------- rotary positions
constexpr int kAxes = 8;

struct RotateArgs {
    const uint16_t* in[2];  // queries, keys
    uint16_t* out[2];
    int64_t in_stride[2], out_stride[2];
    int32_t heads[2];
    int32_t d, pairs, n_tok, n_axes;
    int32_t ends[kAxes];  // pairs of the axes so far
    const int32_t* positions;
    const double* freqs;
    int32_t inverse, parts[2], columns;  // parts: threads to a token and column for the heads of queries and keys; columns: threads to a token and part
};

// (a, b) -> (a cos - b sin, a sin + b cos).  Bound by the rows read and written once.  A thread takes eight pairs of a token (or 16
// values that are not rotated) through up to kRotateHeads heads: all loads first, then cos and sin, formed once, then the products.  Its
// heads lie parts[] apart, so that at each step neighbouring threads take a token's neighbouring heads, and a wavefront's accesses are
// one stretch of the row: 32768 tokens, 32 heads of 128, in place, 123.5 us (5.4 TB/s); with a thread's heads side by side 160 us.
// One, two and eight heads to a thread: 215, 142 and 125 us (8000 tokens of 8 heads 13.3, 11.6 and 12.1, four 11.4; calls of few tokens
// take the same with any).  Turns are counted in fp64, of which the fraction goes to the hardware's cos and sin of turns.  Three roundings,
// of 1 / 2 pi (0.56 of a half step) and of two products, are 1.3 * 2^-52 of an angle at most.
constexpr int kRotateHeads = 4;
template <bool kBf16, bool kInterleaved>
__global__ __launch_bounds__(kLayerThreads) void rotate_kernel(RotateArgs a)
{
    const int64_t at = (int64_t)blockIdx.x * kLayerThreads + threadIdx.x;
    const int column = (int)(at % a.columns), all = a.parts[0] + a.parts[1];
    const int64_t rest = at / a.columns, tok = rest / all;
    if (tok >= a.n_tok) return;
    const int part = (int)(rest % all), k = part >= a.parts[0], first = k ? part - a.parts[0] : part;
    const int n = (a.heads[k] - first + a.parts[k] - 1) / a.parts[k], step = a.parts[k] * a.d;
    const uint16_t* in = a.in[k] + tok * a.in_stride[k] + (int64_t)first * a.d;
    uint16_t* out = a.out[k] + tok * a.out_stride[k] + (int64_t)first * a.d;
    const bool turns = column < a.pairs / 8;
    const int plain = 2 * a.pairs + (column - a.pairs / 8) * 16;  // (the second eight values may lie behind the row)
    const int c0 = !turns ? plain : kInterleaved ? column * 16 : column * 8;
    const int c1 = !turns ? min(plain + 8, a.d - 8) : kInterleaved ? c0 + 8 : c0 + a.pairs;
    if (!turns && in == out) return;
    uint4 v[kRotateHeads][2];
#pragma unroll
    for (int h = 0; h < kRotateHeads; ++h)
        if (h < n) {
            v[h][0] = *(const uint4*)(in + (int64_t)h * step + c0);
            v[h][1] = *(const uint4*)(in + (int64_t)h * step + c1);
        }
    if (!turns) {
#pragma unroll
        for (int h = 0; h < kRotateHeads; ++h)
            if (h < n) {
                *(uint4*)(out + (int64_t)h * step + c0) = v[h][0];
                *(uint4*)(out + (int64_t)h * step + c1) = v[h][1];
            }
        return;
    }
    float cs[8], sn[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int pair = column * 8 + u;
        int axis = 0;
        for (int e = 0; e < a.n_axes - 1; ++e) axis += pair >= a.ends[e];
        const double t = (double)a.positions[(int64_t)axis * a.n_tok + tok] * (a.freqs[pair] * 0.15915494309189533577);
        const float turn = (float)(t - rint(t));
        cs[u] = __builtin_amdgcn_cosf(turn);
        sn[u] = __builtin_amdgcn_sinf(a.inverse ? -turn : turn);
    }
#pragma unroll
    for (int h = 0; h < kRotateHeads; ++h)
        if (h < n) {
            float f[16], g[16];
            eight_floats(v[h][0], kBf16, f);
            eight_floats(v[h][1], kBf16, f + 8);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int x = kInterleaved ? 2 * u : u, y = kInterleaved ? 2 * u + 1 : 8 + u;
                g[x] = f[x] * cs[u] - f[y] * sn[u];
                g[y] = f[x] * sn[u] + f[y] * cs[u];
            }
            Eight<kBf16 ? ST_BF16 : ST_F16>::store(out, (int64_t)h * step + c0, g);
            Eight<kBf16 ? ST_BF16 : ST_F16>::store(out, (int64_t)h * step + c1, g + 8);
        }
}

}  // namespace st
