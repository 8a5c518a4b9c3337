// Projection of int8 rows by shared int8 weights, with a low-rank adapter for each row (definition: silvertorch.h).
#pragma once
#include "st_kv_device.h"

namespace st {

typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));

struct ProjectArgs {
    const int8_t* x;
    const float* x_scale;
    const int8_t* w;
    const float* w_scale;
    const uint16_t* a;  // adapters; NULL: none
    const uint16_t* b;
    const float* alpha;
    const int32_t* adapter_of;
    uint16_t* inner;    // [n_rows, rank]: alpha x_scale a x / 2^e, rounded
    float* power;       // [n_rows]: 2^e
    void* out;
    int64_t out_stride;
    int32_t n_rows, k, n, n_adapters, rank, bf16;
};

// The adapter of a row, -1: none.
__device__ inline int project_adapter(const ProjectArgs& a, int64_t row)
{
    if (row >= a.n_rows) return -1;
    const int i = a.adapter_of[row];
    return i >= 0 && i < a.n_adapters ? i : -1;
}

// The smallest number above `last` that a lane of the wavefront holds, INT32_MAX if there is none.
template <int N>
__device__ inline int next_of(const int (&v)[N], int last)
{
    int m = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < N; ++i) m = v[i] > last && v[i] < m ? v[i] : m;
    for (int o = 32; o > 0; o >>= 1) m = min(m, __shfl_xor(m, o));
    return m;
}

// D += A B of 16-bit floats, 16 x 16 x 32: lane l holds row l % 16 of A and column l % 16 of B, elements (l / 16) * 8 ..; of D
// column l % 16, rows (l / 16) * 4 ..
__device__ inline float4v mfma_16(const uint4& a, const uint4& b, const float4v& d, bool bf16)
{
    if (bf16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), d, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), d, 0, 0, 0);
}

// Eight int8 as 16-bit floats, exactly.
__device__ inline uint4 eight_16(uint32_t lo, uint32_t hi, bool bf16)
{
    if (!bf16) return __builtin_bit_cast(uint4, eight_halves(lo, hi));
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = (i < 2 ? lo : hi) >> (16 * (i & 1));
        const uint32_t a = __float_as_uint((float)(int8_t)w), b = __float_as_uint((float)(int8_t)(w >> 8));
        r[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// ---------------------------------------------------------------- inner values of the adapters
constexpr int kInnerWaves = 8;

// One workgroup to 16 rows; its wavefronts share k between them and join their sums in the LDS.  Each adapter among the rows in turn:
// the other rows' results of it are not used.
template <int kTiles>  // of 16 ranks
__global__ __launch_bounds__(kInnerWaves * 64) void project_inner_kernel(ProjectArgs p)
{
    constexpr int kRanks = 16 * kTiles;
    __shared__ float s_sum[kInnerWaves][16][kRanks + 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = (int64_t)blockIdx.x * 16, row = row0 + (lane & 15);
    const int8_t* x = p.x + min(row, (int64_t)p.n_rows - 1) * p.k;
    const bool bf16 = p.bf16 != 0;
    int mine[1] = {project_adapter(p, row)};
    for (int a = next_of(mine, -1); a != 0x7FFFFFFF; a = next_of(mine, a)) {
        const uint16_t* wa = p.a + (int64_t)a * p.rank * p.k;
        float4v acc[kTiles] = {};
        for (int k0 = wave * 64; k0 < p.k; k0 += kInnerWaves * 64) {
            const int k = k0 + (lane >> 4) * 16;
            const bool in = k < p.k;
            uint4 xi = make_uint4(0, 0, 0, 0);
            if (in) xi = *(const uint4*)(x + k);
            const uint4 x0 = eight_16(xi.x, xi.y, bf16), x1 = eight_16(xi.z, xi.w, bf16);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const int r = t * 16 + (lane & 15);
                uint4 a0 = make_uint4(0, 0, 0, 0), a1 = a0;
                if (in && r < p.rank) {
                    a0 = *(const uint4*)(wa + (int64_t)r * p.k + k);
                    a1 = *(const uint4*)(wa + (int64_t)r * p.k + k + 8);
                }
                acc[t] = mfma_16(a0, x0, acc[t], bf16);
                acc[t] = mfma_16(a1, x1, acc[t], bf16);
            }
        }
        __syncthreads();  // the sums of the adapter before are read
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
            *(float4v*)&s_sum[wave][lane & 15][t * 16 + (lane >> 4) * 4] = acc[t];
        __syncthreads();
        // 32 threads to a row
        const int m = tid >> 5, l = tid & 31;
        if (project_adapter(p, row0 + m) == a) {
            const float factor = p.alpha[a] * p.x_scale[row0 + m];
            float v[(kRanks + 31) / 32];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < (kRanks + 31) / 32; ++i) {
                const int r = i * 32 + l;
                v[i] = 0.0f;
                if (r < p.rank) {
                    for (int u = 0; u < kInnerWaves; ++u) v[i] += s_sum[u][m][r];
                    v[i] *= factor;
                }
                top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
            }
            for (int o = 16; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
            // 2^e of the largest, kept within what can be inverted; 1 where there is none or it is no number
            uint32_t e = top >> 23;
            e = e < 27 ? 127u : e == 255 ? 127u : min(e, 227u);
            const float down = __uint_as_float((254u - e) << 23);
#pragma unroll
            for (int i = 0; i < (kRanks + 31) / 32; ++i) {
                const int r = i * 32 + l;
                if (r < p.rank) p.inner[(row0 + m) * p.rank + r] = (uint16_t)to_16_bits(v[i] * down, bf16);
            }
            if (l == 0) p.power[row0 + m] = __uint_as_float(e << 23);
        }
    }
}

// ---------------------------------------------------------------- what follows the int8 products
// A wavefront holds kM x kN tiles of 16 rows x 16 columns: in tile (i, j) lane l has row m0 + 16 i + l % 16, columns
// n0 + 16 j + (l / 16) * 4 .. + 3.  Scales, the adapters' products on top of the scaled sums (both over 2^e), rounding, stores.
template <int kM, int kN>
__device__ inline void project_finish(const ProjectArgs& p, int4v (&dot)[kM][kN], int64_t m0, int n0)
{
    const int lane = threadIdx.x & 63;
    const bool bf16 = p.bf16 != 0;
    float xs[kM], power[kM];
    int mine[kM];
#pragma unroll
    for (int i = 0; i < kM; ++i) {
        const int64_t row = m0 + 16 * i + (lane & 15);
        xs[i] = row < p.n_rows ? p.x_scale[row] : 0.0f;
        mine[i] = -1;
        power[i] = 1.0f;
        if (p.a) {
            mine[i] = project_adapter(p, row);
            if (mine[i] >= 0) {
                power[i] = p.power[row];
                xs[i] *= __uint_as_float(0x7F000000u - __float_as_uint(power[i]));  // 1 / 2^e
            }
        }
    }
    float4v sum[kM][kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) {
        const int n = n0 + 16 * j + (lane >> 4) * 4;
        float4v ws = {0.0f, 0.0f, 0.0f, 0.0f};
        if (n < p.n) ws = *(const float4v*)(p.w_scale + n);
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int u = 0; u < 4; ++u) sum[i][j][u] = (float)dot[i][j][u] * xs[i] * ws[u];
    }
    if (p.a)
        for (int a = next_of(mine, -1); a != 0x7FFFFFFF; a = next_of(mine, a)) {
            const uint16_t* wb = p.b + (int64_t)a * p.n * p.rank;
            for (int r0 = 0; r0 < p.rank; r0 += 32) {
                const int r = r0 + (lane >> 4) * 8;
                uint4 b[kN];
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    const int n = n0 + 16 * j + (lane & 15);
                    b[j] = make_uint4(0, 0, 0, 0);
                    if (n < p.n && r < p.rank) b[j] = *(const uint4*)(wb + (int64_t)n * p.rank + r);
                }
#pragma unroll
                for (int i = 0; i < kM; ++i) {
                    if (ballot(mine[i] == a) == 0) continue;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (mine[i] == a && r < p.rank) v = *(const uint4*)(p.inner + (m0 + 16 * i + (lane & 15)) * p.rank + r);
#pragma unroll
                    for (int j = 0; j < kN; ++j) sum[i][j] = mfma_16(b[j], v, sum[i][j], bf16);
                }
            }
        }
#pragma unroll
    for (int i = 0; i < kM; ++i) {
        const int64_t row = m0 + 16 * i + (lane & 15);
        if (row >= p.n_rows) continue;
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            const int n = n0 + 16 * j + (lane >> 4) * 4;
            if (n >= p.n) continue;
            uint32_t h[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) h[u] = to_16_bits(sum[i][j][u] * power[i], bf16);
            *(uint2*)((uint16_t*)p.out + row * p.out_stride + n) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
        }
    }
}

// ---------------------------------------------------------------- tiles of 128 x 128
// Rows and weights pass through the LDS, 64 values of k at a time; four wavefronts have 64 x 64 each.
__global__ __launch_bounds__(256) void project_tile_kernel(ProjectArgs p)
{
    constexpr int kRow = 80;  // bytes of a row in the LDS
    __shared__ __align__(16) int8_t s_x[128 * kRow], s_w[128 * kRow];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tiles_n = (p.n + 127) / 128;
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * 128;
    const int n0 = (int)(blockIdx.x % tiles_n) * 128;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    int4v dot[4][4] = {};
    for (int k0 = 0; k0 < p.k; k0 += 64) {
        uint4 xv[2], wv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = (i * 256 + tid) >> 2, k = k0 + (tid & 3) * 16;
            xv[i] = wv[i] = make_uint4(0, 0, 0, 0);
            if (k < p.k) {
                xv[i] = *(const uint4*)(p.x + min(m0 + row, (int64_t)p.n_rows - 1) * p.k + k);
                wv[i] = *(const uint4*)(p.w + (int64_t)min(n0 + row, p.n - 1) * p.k + k);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = ((i * 256 + tid) >> 2) * kRow + (tid & 3) * 16;
            *(uint4*)(s_x + at) = xv[i];
            *(uint4*)(s_w + at) = wv[i];
        }
        __syncthreads();
        int4v xf[4], wf[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xf[i] = *(const int4v*)(s_x + (wm + i * 16 + (lane & 15)) * kRow + (lane >> 4) * 16);
            wf[i] = *(const int4v*)(s_w + (wn + i * 16 + (lane & 15)) * kRow + (lane >> 4) * 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) dot[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[j], xf[i], dot[i][j], 0, 0, 0);
    }
    project_finish<4, 4>(p, dot, m0 + wm, n0 + wn);
}

}  // namespace st
