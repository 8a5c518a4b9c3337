// Projection of int8 rows by shared int8 weights, with a low-rank adapter for each row (definition: silvertorch.h).
#pragma once
#include "st_layer_kernels.h"

namespace st {

typedef int int16v __attribute__((ext_vector_type(16)));
typedef float float16v __attribute__((ext_vector_type(16)));
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
    uint16_t* inner;    // [n_rows, 2, rank]: alpha x_scale a x / 2^e, rounded, and what the rounding left, rounded
    float* power;       // [n_rows]: 2^e
    float* parts;       // few rows, in place of inner and power: [kInnerParts, n_rows, rank], a x over a part of k each
    int32_t* order;     // [n_rows]: rows of one adapter side by side; NULL: as they come
    void* out;
    int64_t out_stride;
    int32_t n_rows, k, n, n_adapters, rank;
};

// The adapter of a row, -1: none.
__device__ inline int project_adapter(const ProjectArgs& a, int64_t row)
{
    if (row >= a.n_rows) return -1;
    const int i = a.adapter_of[row];
    return i >= 0 && i < a.n_adapters ? i : -1;
}

// The rows at some places of the order, the last row's for a place behind it.  All loads begin together: a wait for each would be a trip
// to memory for each.
template <int N>
__device__ inline void project_places(const ProjectArgs& p, const int64_t (&m)[N], int64_t (&row)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) row[i] = min(m[i], (int64_t)p.n_rows - 1);
    if (p.order) {
        int32_t at[N];
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = p.order[row[i]];
#pragma unroll
        for (int i = 0; i < N; ++i) row[i] = at[i];
    }
}
// The adapters of those rows, -1 for a place behind the last row too.
template <int N>
__device__ inline void project_adapters(const ProjectArgs& p, const int64_t (&m)[N], const int64_t (&row)[N], int (&of)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) of[i] = p.adapter_of[row[i]];
#pragma unroll
    for (int i = 0; i < N; ++i) of[i] = m[i] < p.n_rows && of[i] >= 0 && of[i] < p.n_adapters ? of[i] : -1;
}

// The smallest number above `last` that a lane holds, INT32_MAX if there is none.  Lanes that lie kLanes apart hold the same.
template <int kLanes, int N>
__device__ inline int next_of(const int (&v)[N], int last)
{
    uint32_t m = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < N; ++i) m = v[i] > last ? min(m, (uint32_t)v[i]) : m;
    m = min(m, row_ror<8>(m));
    m = min(m, row_ror<4>(m));
    m = min(m, row_ror<2>(m));
    m = min(m, row_ror<1>(m));
    if (kLanes == 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        m = min((uint32_t)r[0], (uint32_t)r[1]);
    }
    return __builtin_amdgcn_readfirstlane((int)m);
}

// D += A B of 16-bit floats, 16 x 16 x 32: lane l holds row l % 16 of A and column l % 16 of B, elements (l / 16) * 8 ..; of D
// column l % 16, rows (l / 16) * 4 ..
template <bool kBf16>
__device__ inline float4v mfma_16(const uint4& a, const uint4& b, const float4v& d)
{
    if (kBf16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), d, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), d, 0, 0, 0);
}

// The same, 32 x 32 x 16: lane l holds row l % 32 of A and column l % 32 of B, elements (l / 32) * 8 ..; of D column l % 32, rows
// 8 * (i / 4) + 4 * (l / 32) + i % 4.
template <bool kBf16>
__device__ inline float16v mfma_32(const uint4& a, const uint4& b, const float16v& d)
{
    if (kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), d, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), d, 0, 0, 0);
}

// Eight int8 as 16-bit floats, exactly.
template <bool kBf16>
__device__ inline uint4 eight_16(uint32_t lo, uint32_t hi)
{
    if (!kBf16) return __builtin_bit_cast(uint4, eight_halves(lo, hi));
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = (i < 2 ? lo : hi) >> (16 * (i & 1));
        const uint32_t a = __float_as_uint((float)(int8_t)w), b = __float_as_uint((float)(int8_t)(w >> 8));
        r[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// 16 bytes for each lane, from where it points to `to` + 16 * lane (`to` the same in all lanes).
__device__ inline void load_to_lds(const int8_t* from, int8_t* to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// The same, 4 bytes.
__device__ inline void word_to_lds(const void* from, int8_t* to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 4, 0, 0);
}

// ---------------------------------------------------------------- rows in the order of their adapters
// Rows of a segment are dealt into buckets by adapter (those without one behind the others), so that a tile of the kernels below
// meets few adapters: each costs it a load of operands and products with all its rows.  A segment to a workgroup, counts and places in the
// LDS; which of a bucket's rows comes first may vary from call to call, and no row's result goes by it.
constexpr int kOrderThreads = 512, kOrderRows = 2048, kBuckets = 2048;

__global__ __launch_bounds__(kOrderThreads) void project_order_kernel(ProjectArgs p)
{
    __shared__ uint32_t count[kBuckets];
    __shared__ uint32_t part[kOrderThreads / 64];
    constexpr int kEach = kOrderRows / kOrderThreads, kOwn = kBuckets / kOrderThreads;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t first = (int64_t)blockIdx.x * kOrderRows;
    int bucket[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t row = first + i * kOrderThreads + tid;
        const int a = project_adapter(p, row);
        bucket[i] = row >= p.n_rows ? -1 : a < 0 ? kBuckets - 1 : a % (kBuckets - 1);
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) count[i * kOrderThreads + tid] = 0;
    __syncthreads();
    // Places among the counts of `count`; a wavefront whose rows share a bucket asks once.
    auto take = [&](int b) -> uint32_t {
        const int b0 = __builtin_amdgcn_readfirstlane(b);
        if (ballot(b != b0) == 0) {
            uint32_t at = 0;
            if (lane == 0 && b0 >= 0) at = atomicAdd(&count[b0], 64u);
            return (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + lane;
        }
        return b >= 0 ? atomicAdd(&count[b], 1u) : 0u;
    };
#pragma unroll
    for (int i = 0; i < kEach; ++i) (void)take(bucket[i]);
    __syncthreads();
    uint32_t own[kOwn], sum = 0, total;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        own[i] = sum;
        sum += count[tid * kOwn + i];
    }
    const uint32_t before = wg_scan_add<kOrderThreads>(sum, part, &total);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) count[tid * kOwn + i] = before + own[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t at = take(bucket[i]);
        if (bucket[i] >= 0) p.order[first + at] = (int32_t)(first + i * kOrderThreads + tid);
    }
}

// ---------------------------------------------------------------- inner values of the adapters
constexpr int kInnerParts = 8;

// What one wavefront does for 16 kM rows, an adapter, kTiles x 16 of its ranks and a part of k: the 64 values from 64 (part + 8 i) on,
// i = 0, 1, ..  `wa`: the lane's row and place in a, `ranks`: how many of the ranks there are.  Loads of kChunks of those run ahead.
template <bool kBf16, int kTiles, int kM, int kRegisters = 96>
struct InnerPart {
    static constexpr int kFit = kRegisters / (kTiles * 8 + kM * 4), kChunks = kFit < 1 ? 1 : kFit > 8 ? 8 : kFit;
    uint4 xv[kChunks][kM], av[kChunks][kTiles][2];
    float4v acc[kM][kTiles];

    __device__ void load_x(const int8_t* const (&x)[kM], int c, int k, int k_end)
    {
        const bool in = k + (int)((threadIdx.x & 63) >> 4) * 16 < k_end;
#pragma unroll
        for (int i = 0; i < kM; ++i) {
            xv[c][i] = make_uint4(0, 0, 0, 0);
            if (in) xv[c][i] = *(const uint4*)(x[i] + k);
        }
    }
    __device__ void load_a(const uint16_t* wa, int ranks, int c, int k, int k_end)
    {
        const int lane = threadIdx.x & 63;
        const bool in = k + (lane >> 4) * 16 < k_end;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            av[c][t][0] = av[c][t][1] = make_uint4(0, 0, 0, 0);
            if (in && t * 16 + (lane & 15) < ranks) {
                av[c][t][0] = *(const uint4*)(wa + (int64_t)t * 16 * k_end + k);
                av[c][t][1] = *(const uint4*)(wa + (int64_t)t * 16 * k_end + k + 8);
            }
        }
    }
    __device__ void first_x(const int8_t* const (&x)[kM], int part, int k_end)
    {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) load_x(x, c, (part + c * kInnerParts) * 64, k_end);
    }
    // The first chunks of x are there.  A chunk's registers take on a later one as soon as its products are under way.
    __device__ void run(const int8_t* const (&x)[kM], const uint16_t* wa, int ranks, int part, int k_end)
    {
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) acc[i][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < kChunks; ++c) load_a(wa, ranks, c, (part + c * kInnerParts) * 64, k_end);
        for (int k0 = part * 64; k0 < k_end; k0 += kChunks * kInnerParts * 64)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                if (k0 + c * kInnerParts * 64 >= k_end) break;  // (its registers were not loaded again)
#pragma unroll
                for (int i = 0; i < kM; ++i) {
                    const uint4 x0 = eight_16<kBf16>(xv[c][i].x, xv[c][i].y), x1 = eight_16<kBf16>(xv[c][i].z, xv[c][i].w);
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        acc[i][t] = mfma_16<kBf16>(av[c][t][0], x0, acc[i][t]);
                        acc[i][t] = mfma_16<kBf16>(av[c][t][1], x1, acc[i][t]);
                    }
                }
                const int k = k0 + (kChunks + c) * kInnerParts * 64;
                if (k < k_end) {
                    load_x(x, c, k, k_end);
                    load_a(wa, ranks, c, k, k_end);
                }
            }
    }
};

// The exponent (with its bias) of the power of two 2^e that a row's inner values are divided by, and with them what they are added to, from the bits
// of the largest.  Neither term may leave fp32 for the other's sake.  bf16 has fp32's range: 1, but 2 where rounding up could leave it.  fp16: the
// largest's own, from 2^-100 (sums of products that leave fp32 by it, from 2^28 on, are beyond fp16 in any case) to 2^120 (they are off by
// 2^-30 then, 2^-25 being half of fp16's least); 1 where the largest is below or no number.
template <bool kBf16>
__device__ inline uint32_t project_exponent(uint32_t top)
{
    const uint32_t e = top >> 23;
    if (kBf16) return e == 254 ? 128u : 127u;
    return e < 27 || e == 255 ? 127u : min(e, 247u);
}

// A number as the sum of two 16-bit ones: rounded, and what the rounding left, rounded (nothing beside an infinity).  Inner values are held so, and an
// adapter's products made twice, since one half alone shows in the outputs (bf16, adapters' part as large as the rest: 2^-9.2 of them, and
// 2^-14 with both, beside plain sums in fp32).  It costs 2 % of a call with rank 32 (16384 x 4096 x 5120, 16 adapters 362 -> 370 us), 8 % with 128
// (16384 x 4096 x 4096 374 -> 404), nothing with few rows.
template <bool kBf16>
__device__ inline void two_halves(float v, uint16_t* high, uint16_t* low)
{
    *high = one_16<kBf16>(v);
    const float h = kBf16 ? bf16_float(*high) : f16_float(*high);
    *low = one_16<kBf16>(fabsf(h) < __builtin_inff() ? v - h : 0.0f);
}

// The same for many rows: operands come through the LDS, in space of the wavefront's own, kSlots - 1 steps ahead.  A load straight into a
// lane's operand touches 64 places with 64 lanes, which an address unit takes one by one; rows in the LDS come in by lines.  A step is
// 64 values of k and two tiles of ranks; the rows come with a chunk's first.
template <bool kBf16, int kTiles, int kM>
struct InnerStream {
    static constexpr int kGroup = kTiles < 2 ? 1 : 2, kGroups = kTiles / kGroup;  // tiles of ranks to a step, steps to 64 values
    static constexpr int kSlot = kM * 1024 + kGroup * 2048, kSlots = kGroup < 2 ? 4 : 3, kBytes = kSlots * kSlot;
    static constexpr int kRowLoads = kM, kRankLoads = 2 * kGroup;
    float4v acc[kM][kTiles];
    const int8_t* x[kM];  // of each 16 rows row lane / 4, its first piece
    const uint16_t* a;    // of the adapter's first rank
    int k, rank, part, slot, to;

    // The place of a row's piece of 16 bytes: 16 neighbouring rows have a piece at 16 places of the banks.
    __device__ static int row_place(int row, int piece) { return piece ^ ((row >> 2) & 3); }
    __device__ static int rank_place(int row, int piece) { return piece ^ ((row >> 1) & 7); }

    template <int kG>
    __device__ void load(int8_t* own, int chunk)
    {
        const int lane = threadIdx.x & 63, k0 = chunk * 64;
        int8_t* at = own + to * kSlot;
        if (kG == 0) {
            const int piece = row_place(lane >> 2, lane & 3) * 16;
#pragma unroll
            for (int i = 0; i < kM; ++i) load_to_lds(x[i] + k0 + (k0 + piece < k ? piece : 0), at + i * 1024);
        }
#pragma unroll
        for (int t = 0; t < kRankLoads; ++t) {
            const int row = t * 8 + (lane >> 3), piece = rank_place(row, lane & 7) * 8;
            load_to_lds((const int8_t*)(a + (int64_t)min(kG * kGroup * 16 + row, rank - 1) * k + k0 + (k0 + piece < k ? piece : 0)), at + kM * 1024 + t * 1024);
        }
        to = to + 1 == kSlots ? 0 : to + 1;
    }
    // One step, of group kG of its chunk: `ahead_chunk` is that of the step kSlots - 1 further on.
    template <int kG>
    __device__ void one(int8_t* own, int chunk, int ahead_chunk, uint4 (&x0)[kM], uint4 (&x1)[kM])
    {
        constexpr int kNext = (kG + 1) % kGroups == 0 ? kRowLoads + kRankLoads : kRankLoads;
        // this step lies in the LDS, and the one before it is read
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kSlots == 3 ? kNext : 2 * kNext) : "memory");
        load<(kG + kSlots - 1) % kGroups>(own, ahead_chunk);
        const int lane = threadIdx.x & 63, piece = lane >> 4;
        const int8_t* at = own + slot * kSlot;
        slot = slot + 1 == kSlots ? 0 : slot + 1;
        if (kG == 0) {
            const uint32_t in = chunk * 64 + piece * 16 < k ? 0xFFFFFFFFu : 0u;  // (behind a row's end lies something else)
#pragma unroll
            for (int i = 0; i < kM; ++i) {
                const int4v v = *(const int4v*)(at + i * 1024 + (lane & 15) * 64 + row_place(lane & 15, piece) * 16);
                x0[i] = eight_16<kBf16>(v[0] & in, v[1] & in);
                x1[i] = eight_16<kBf16>(v[2] & in, v[3] & in);
            }
        }
#pragma unroll
        for (int t = 0; t < kGroup; ++t) {
            const int8_t* row = at + kM * 1024 + (t * 16 + (lane & 15)) * 128;
            int4v v0 = *(const int4v*)(row + rank_place(lane & 15, 2 * piece) * 16), v1 = *(const int4v*)(row + rank_place(lane & 15, 2 * piece + 1) * 16);
            if (chunk * 64 + 64 > k) {  // (there too: 0 times an infinity is no number)
                const int in = chunk * 64 + piece * 16 < k ? -1 : 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) v0[u] &= in, v1[u] &= in;
            }
            const uint4 a0 = make_uint4(v0[0], v0[1], v0[2], v0[3]), a1 = make_uint4(v1[0], v1[1], v1[2], v1[3]);
#pragma unroll
            for (int i = 0; i < kM; ++i) {
                float4v& d = acc[i][kG * kGroup + t];
                d = mfma_16<kBf16>(a0, x0[i], d);
                d = mfma_16<kBf16>(a1, x1[i], d);
            }
        }
    }
    template <int kG>
    __device__ void first(int8_t* own, int last)
    {
        if constexpr (kG < kSlots - 1) {
            load<kG % kGroups>(own, min(part + kG / kGroups * kInnerParts, last));
            first<kG + 1>(own, last);
        }
    }
    template <int kG>
    __device__ void all(int8_t* own, int chunk, int last, uint4 (&x0)[kM], uint4 (&x1)[kM])
    {
        if constexpr (kG < kGroups) {
            one<kG>(own, chunk, min(chunk + (kG + kSlots - 1) / kGroups * kInnerParts, last), x0, x1);
            all<kG + 1>(own, chunk, last, x0, x1);
        }
    }
    __device__ void run(int8_t* own)
    {
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) acc[i][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        const int chunks = (k + 63) >> 6;
        if (part >= chunks) return;
        const int last = part + (chunks - 1 - part) / kInnerParts * kInnerParts;  // (loaded again where a step further on is not)
        slot = to = 0;
        first<0>(own, last);
        uint4 x0[kM], x1[kM];
        for (int chunk = part; chunk <= last; chunk += kInnerParts) all<0>(own, chunk, last, x0, x1);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }
};

// 16 kM rows and every gridDim.y-th adapter among them; the other rows' results of an adapter are not kept.  A wavefront to each part of
// k; the parts are summed in their order, so that a row's sums have one order whatever kM, the grid and the kernel.  kM 1: operands
// straight from memory (shorter where there are few workgroups); 2: through the LDS.
template <bool kBf16, int kTiles, int kM>
__global__ __launch_bounds__(kInnerParts * 64) void project_inner_kernel(ProjectArgs p)
{
    constexpr int kRanks = 16 * kTiles, kRow = kRanks + 4;
    constexpr int kSums = kInnerParts * 16 * kRow * 4, kSteps = kM == 1 ? 0 : kInnerParts * InnerStream<kBf16, kTiles, kM>::kBytes;
    __shared__ __align__(1024) int8_t lds[kSums > kSteps ? kSums : kSteps];  // steps, and then sums [part][16][kRow]
    float* s_sum = (float*)lds;
    const int tid = threadIdx.x, lane = tid & 63, part = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t m0 = (int64_t)blockIdx.x * (16 * kM);
    // rows of each 16: that whose adapter counts as a lane's, that which the lane loads, and that which it sums with 31 others
    const int m = tid >> 5, l = tid & 31;
    int64_t at[3 * kM], rows[3 * kM];
    int of[3 * kM], mine[kM];
    float scale[kM];
    const int8_t* x[kM];
#pragma unroll
    for (int i = 0; i < kM; ++i) {
        at[i] = m0 + 16 * i + (lane & 15);
        at[kM + i] = m0 + 16 * i + (kM == 1 ? lane & 15 : lane >> 2);
        at[2 * kM + i] = m0 + 16 * i + m;
    }
    project_places<3 * kM>(p, at, rows);
#pragma unroll
    for (int i = 0; i < kM; ++i) scale[i] = p.x_scale[rows[2 * kM + i]];
    project_adapters<3 * kM>(p, at, rows, of);
#pragma unroll
    for (int i = 0; i < kM; ++i) {
        mine[i] = of[i];
        x[i] = p.x + rows[kM + i] * p.k + (kM == 1 ? (lane >> 4) * 16 : 0);
    }
    int index = 0;
    for (int a = next_of<16>(mine, -1); a != 0x7FFFFFFF; a = next_of<16>(mine, a), ++index) {
        if (index % gridDim.y != blockIdx.y) continue;
        const float alpha = p.alpha[a];
        const uint16_t* wa = p.a + (int64_t)a * p.rank * p.k;
        float4v acc[kM][kTiles];
        if constexpr (kM == 1) {
            InnerPart<kBf16, kTiles, kM> inner;
            inner.first_x(x, part, p.k);
            inner.run(x, wa + (int64_t)(lane & 15) * p.k + (lane >> 4) * 16, p.rank, part, p.k);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) acc[0][t] = inner.acc[0][t];
        } else {
            InnerStream<kBf16, kTiles, kM> inner;
#pragma unroll
            for (int i = 0; i < kM; ++i) inner.x[i] = x[i];
            inner.a = wa;
            inner.k = p.k;
            inner.rank = p.rank;
            inner.part = part;
            __syncthreads();  // the sums before are read
            inner.run(lds + part * InnerStream<kBf16, kTiles, kM>::kBytes);
#pragma unroll
            for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int t = 0; t < kTiles; ++t) acc[i][t] = inner.acc[i][t];
        }
        constexpr int kEach = (kRanks + 31) / 32;
#pragma unroll
        for (int i = 0; i < kM; ++i) {
            __syncthreads();  // the sums before, or the steps, are read
#pragma unroll
            for (int t = 0; t < kTiles; ++t) *(float4v*)&s_sum[(part * 16 + (lane & 15)) * kRow + t * 16 + (lane >> 4) * 4] = acc[i][t];
            __syncthreads();
            if (of[2 * kM + i] != a) continue;
            const int64_t row = rows[2 * kM + i];
            const float factor = alpha * scale[i];
            float v[kEach];
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < kEach; ++c) {
                const int r = c * 32 + l;
                v[c] = 0.0f;
                if (r < p.rank) {
                    v[c] = s_sum[m * kRow + r];
#pragma unroll
                    for (int u = 1; u < kInnerParts; ++u) v[c] += s_sum[(u * 16 + m) * kRow + r];
                    v[c] *= factor;
                }
                top = max(top, __float_as_uint(v[c]) & 0x7FFFFFFFu);
            }
            top = max(top, row_ror<8>(top));
            top = max(top, row_ror<4>(top));
            top = max(top, row_ror<2>(top));
            top = max(top, row_ror<1>(top));
            const auto both = __builtin_amdgcn_permlane16_swap(top, top, false, false);
            const uint32_t e = project_exponent<kBf16>(max((uint32_t)both[0], (uint32_t)both[1]));
            const float down = __uint_as_float((254u - e) << 23);
#pragma unroll
            for (int c = 0; c < kEach; ++c) {
                const int r = c * 32 + l;
                if (r < p.rank) {
                    uint16_t* at = p.inner + row * 2 * p.rank + r;
                    two_halves<kBf16>(v[c] * down, at, at + p.rank);
                }
            }
            if (l == 0) p.power[row] = __uint_as_float(e << 23);
        }
    }
}

// For few rows: a workgroup of one wavefront to each 16 rows, adapter among them, 16 ranks and part of k, so that the adapters' rows
// come in over the whole chip (16 rows, 8 adapters, rank 64, k = 4096: 4.7 us against 20 us by eight workgroups of the kernel
// above).  The sums of a part stay as they are.
template <bool kBf16>
__global__ __launch_bounds__(64) void project_parts_kernel(ProjectArgs p)
{
    const int lane = threadIdx.x, part = blockIdx.z % kInnerParts, rank0 = blockIdx.z / kInnerParts * 16;
    const int row = blockIdx.x * 16 + (lane & 15);
    const int8_t* x[1] = {p.x + (int64_t)min(row, p.n_rows - 1) * p.k + (lane >> 4) * 16};
    const int mine[1] = {project_adapter(p, row)};
    InnerPart<kBf16, 1, 1> inner;
    inner.first_x(x, part, p.k);
    int a = next_of<16>(mine, -1);
    for (int i = 0; i < (int)blockIdx.y && a != 0x7FFFFFFF; ++i) a = next_of<16>(mine, a);
    if (a == 0x7FFFFFFF) return;
    inner.run(x, p.a + ((int64_t)a * p.rank + rank0 + (lane & 15)) * p.k + (lane >> 4) * 16, p.rank - rank0, part, p.k);
    const int r = rank0 + (lane >> 4) * 4;
    if (mine[0] == a && r < p.rank) *(float4v*)(p.parts + ((int64_t)part * p.n_rows + row) * p.rank + r) = inner.acc[0][0];
}

// ---------------------------------------------------------------- what follows the int8 products
// Tiles are 32 rows x 32 columns, as the columns and rows of a matrix product w x^T: lane l has row m0 + l % 32, and columns
// n0 + 8 * (u / 4) + 4 * (l / 32) + u % 4 for u < 16.  The sums of products take on scales and the adapters' part in the same registers.
struct ProjectRow {
    int row, adapter;
    float scale;  // x_scale, bf16: divided by 2^e
    float power;  // 2^e
};
// 1 / 2^e.  fp16: the sums of products with both scales are divided by it, since x_scale / 2^e by itself could be beyond fp32.
__device__ inline float project_inverse(float power) { return __uint_as_float(0x7F000000u - __float_as_uint(power)); }

// The halves of eight of a row's inner values, from rank r on; zeros for a row of another adapter and behind the last rank.
struct InnerValues {
    uint4 high, low;
};
__device__ inline InnerValues project_inner_values(const ProjectArgs& p, int row, int r, bool mine)
{
    InnerValues v = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (mine && r < p.rank) {
        const uint16_t* at = p.inner + (int64_t)row * 2 * p.rank + r;
        v.high = *(const uint4*)at;
        v.low = *(const uint4*)(at + p.rank);
    }
    return v;
}

// An adapter's products with inner values: with the first halves, and then with the second.
template <bool kBf16>
__device__ inline float16v project_inner_products(const uint4& b, const InnerValues& v, const float16v& sum)
{
    return mfma_32<kBf16>(b, v.low, mfma_32<kBf16>(b, v.high, sum));
}

// The weights' scales of a lane's columns.
template <int kN>
__device__ inline void project_scales(const ProjectArgs& p, float4v (&ws)[kN][4], int n0)
{
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int n = n0 + 32 * j + 8 * g + (threadIdx.x >> 5 & 1) * 4;
            ws[j][g] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
            if (n < p.n) ws[j][g] = *(const float4v*)(p.w_scale + n);
        }
}

// Rounding; eight neighbouring columns to a lane: lanes l and l + 32 hold four of each eight and swap half of them.
// out[j][g]: columns 32 j + 16 g + 8 * (l / 32) ..
template <bool kBf16, int kN>
__device__ inline void project_round(const float16v (&sum)[kN], float power, uint4 (&out)[kN][2])
{
#pragma unroll
    for (int j = 0; j < kN; ++j) {
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = two_16<kBf16>(sum[j][2 * i] * power, sum[j][2 * i + 1] * power);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            // words 4 g, 4 g + 1: columns 16 g + 4 half ..; words 4 g + 2, 4 g + 3: columns 16 g + 8 + 4 half ..
            const auto a = __builtin_amdgcn_permlane32_swap(h[4 * g], h[4 * g + 2], false, false);
            const auto b = __builtin_amdgcn_permlane32_swap(h[4 * g + 1], h[4 * g + 3], false, false);
            out[j][g] = make_uint4(a[0], b[0], a[1], b[1]);
        }
    }
}

// Sums of the rows of one adapter with its part, of other rows as they were: what they would take on is 0 times an adapter's values, which
// is no number for an infinite one.
__device__ inline float16v project_with(const float16v& sum, const float16v& with, bool mine)
{
    float16v r;
#pragma unroll
    for (int u = 0; u < 16; ++u) r[u] = mine ? with[u] : sum[u];
    return r;
}

// The adapters' products on top of the scaled sums of kTM x kTN tiles, 16 ranks of an adapter at a time, all rows' operands with one trip to
// memory.
template <bool kBf16, int kTM, int kTN>
__device__ inline void project_add_adapters(const ProjectArgs& p, float16v (&sum)[kTM][kTN], const ProjectRow (&rows)[kTM], int n0)
{
    const int lane = threadIdx.x & 63;
    int of[kTM];
#pragma unroll
    for (int i = 0; i < kTM; ++i) of[i] = rows[i].adapter;
    for (int a = next_of<32>(of, -1); a != 0x7FFFFFFF; a = next_of<32>(of, a)) {
        const uint16_t* wb = p.b + (int64_t)a * p.n * p.rank;
        bool alone = true;
#pragma unroll
        for (int i = 0; i < kTM; ++i) alone = alone && ballot(of[i] != a) == 0;
        for (int r0 = 0; r0 < p.rank; r0 += 16) {
            const int r = r0 + (lane >> 5) * 8;
            InnerValues v[kTM];
            uint4 b[kTN];
#pragma unroll
            for (int i = 0; i < kTM; ++i) v[i] = project_inner_values(p, rows[i].row, r, of[i] == a);
#pragma unroll
            for (int j = 0; j < kTN; ++j) {
                const int n = n0 + 32 * j + (lane & 31);
                b[j] = make_uint4(0, 0, 0, 0);
                if (n < p.n && r < p.rank) b[j] = *(const uint4*)(wb + (int64_t)n * p.rank + r);
            }
            if (alone) {
#pragma unroll
                for (int i = 0; i < kTM; ++i)
#pragma unroll
                    for (int j = 0; j < kTN; ++j) sum[i][j] = project_inner_products<kBf16>(b[j], v[i], sum[i][j]);
            } else {
#pragma unroll
                for (int i = 0; i < kTM; ++i)
#pragma unroll
                    for (int j = 0; j < kTN; ++j) {
                        sum[i][j] = project_with(sum[i][j], project_inner_products<kBf16>(b[j], v[i], sum[i][j]), of[i] == a);
                        __builtin_amdgcn_sched_barrier(0);  // (one tile's sums twice, not all)
                    }
            }
        }
    }
}

template <int kN>
__device__ inline void project_store(const ProjectArgs& p, const uint4 (&out)[kN][2], int64_t row, int n0)
{
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int n = n0 + 32 * j + 16 * g + (threadIdx.x >> 5 & 1) * 8;
            if (row < p.n_rows && n < p.n) *(uint4*)((uint16_t*)p.out + row * p.out_stride + n) = out[j][g];
        }
}

// The same by whole lines, through 4096 bytes of the LDS that are the wavefront's own: neighbouring lanes store a row's neighbouring
// columns, 128 bytes of it (as they lie in the registers, 32; 1024 values of k, 16384 x 4096: 121 us against 107; half lines
// with tiles of 64 gain nothing).  row: -1 behind the last one.
__device__ inline void project_store_lines(const ProjectArgs& p, const uint4 (&out)[2][2], int row, int n0, int8_t* own)
{
    const int lane = threadIdx.x & 63, m = lane & 31;
    auto place = [](int m, int piece) { return m * 128 + (piece ^ (m & 7)) * 16; };
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int g = 0; g < 2; ++g) *(int4v*)(own + place(m, j * 4 + g * 2 + (lane >> 5))) = __builtin_bit_cast(int4v, out[j][g]);
    const int n = n0 + (lane & 7) * 8;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int at = q * 8 + (lane >> 3), to = __shfl(row, at);
        const int4v v = *(const int4v*)(own + place(at, lane & 7));
        if (to >= 0 && n < p.n) *(int4v*)((uint16_t*)p.out + to * p.out_stride + n) = v;
    }
}

// ---------------------------------------------------------------- tiles that share rows and weights
// Rows and weights go from memory to the LDS past the registers, 128 values of k (a step, a memory line of each row) at a time,
// kStages - 1 steps ahead of the products at most.  Operands of half a step are in registers before its products begin: while one
// half multiplies, those of the next are read from the LDS.  A row's eight pieces of 16 bytes lie in an order that the row's
// number gives, so that 16 lanes that read one piece of 16 rows meet all banks (no conflicts counted).  The last k % 128 values
// come first, through registers, with zeros behind them.
//
// Bound by the matrix units and, with the whole chip at work, by its power: 8192 x 8192 x 8192 takes 512 us (2150 TOP/s), the products
// alone 334, without loads 423, without reads of the LDS 457 (the clock is at 1.8 GHz then, 2.4 with a tenth of the chip, where a
// step of 256 x 256 takes 1.02 us and its products 0.85).  16384 x 4096 x 5120: 315 us, 2180 TOP/s, with 16 adapters of rank 32 in runs of rows 370
// in all.  What follows the products takes some 8 us of a tile of 256 x 256, half of it the stores, which all workgroups begin at once.
// Its rows' and columns' words therefore come with the first steps, and the adapters' operands with one trip for two rows of tiles (16384 x
// 4096 x 4096 266 us -> 255; with the adapters above 3 %).  Tried: four wavefronts with 128 x 128 each
// (345 us for 323; fewer reads, but a SIMD waits with its only wavefront), steps of 64 values with four and five stages (356), tiles of
// 256 x 128 (498), loads and reads in the first half of the products between which they stand (327); all rows of tiles at once behind
// the products (registers spill); stores past the caches (417 for 348).
// kWM x kWN wavefronts of kTM x kTN tiles of 32 x 32, kStages steps in the LDS
template <bool kBf16, int kWM, int kWN, int kTM, int kTN, int kStages>
__global__ __launch_bounds__(kWM* kWN * 64) void project_tile_kernel(ProjectArgs p)
{
    constexpr int kWaves = kWM * kWN, kBM = kWM * kTM * 32, kBN = kWN * kTN * 32, kStage = (kBM + kBN) * 128;
    constexpr int kLoads = (kBM + kBN) / 8 / kWaves;  // of 1024 bytes, a wavefront's of a step
    static_assert((kBM + kBN) / 8 % kWaves == 0, "a step's loads are shared evenly");
    static_assert((kStages - 1) * kLoads <= 63, "loads in flight are counted in six bits");
    static_assert(kWaves * 64 >= kBM && kWaves * 64 >= kBN, "a thread to each row and column");
    // behind the steps: of the rows their number, adapter, scale and power of two, of the columns the scale
    constexpr int kRowOf = kStages * kStage, kAdapter = kRowOf + kBM * 4, kScale = kAdapter + kBM * 4, kPower = kScale + kBM * 4, kColumn = kPower + kBM * 4;
    __shared__ __align__(1024) int8_t lds[kColumn + kBN * 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tiles_n = (p.n + kBN - 1) / kBN, tiles_m = (int)(((int64_t)p.n_rows + kBM - 1) / kBM);
    // A die's workgroups take neighbouring tiles, eight rows of tiles at a time.
    int id = blockIdx.x;
    {
        const int all = tiles_m * tiles_n, die = id & 7, q = all >> 3, r = all & 7;
        id = die * q + min(die, r) + (id >> 3);
    }
    const int group = id / (8 * tiles_n), in = id % (8 * tiles_n), high = min(8, tiles_m - group * 8);
    const int64_t m0 = (int64_t)(group * 8 + in % high) * kBM;
    const int n0 = in / high * kBN;

    // The place of a row's piece in the row's 128 bytes: 16 neighbouring rows have a piece at 16 places of the banks.
    auto place = [](int row, int piece) { return piece ^ ((row >> 1) & 7); };
    // what this lane loads: of each eight rows row lane / 8, the piece that lies at place lane % 8
    const int8_t* from[kLoads];
    const int steps = (p.k + 127) >> 7, tail = p.k & 127;
    auto piece_of = [&](int i) { return place((wave * kLoads + i) * 8 + (lane >> 3), lane & 7) * 16; };
    {
        // (64 rows' or columns' words are a wavefront's where wave * 64 lies among them)
        int64_t at[kLoads + 1], rows[kLoads + 1];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) at[i] = m0 + (wave * kLoads + i) * 8 + (lane >> 3);
        at[kLoads] = m0 + wave * 64 + lane;
        project_places<kLoads + 1>(p, at, rows);
        if (wave * 64 < kBM) {
            const int64_t row = rows[kLoads];
            word_to_lds(p.x_scale + row, lds + kScale + wave * 256);
            if (p.a) {
                word_to_lds(p.adapter_of + row, lds + kAdapter + wave * 256);
                word_to_lds(p.power + row, lds + kPower + wave * 256);
            }
            if (p.order) word_to_lds(p.order + min(at[kLoads], (int64_t)p.n_rows - 1), lds + kRowOf + wave * 256);
        }
        if (wave * 64 < kBN) word_to_lds(p.w_scale + min(n0 + wave * 64 + lane, p.n - 1), lds + kColumn + wave * 256);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int first = (wave * kLoads + i) * 8;
            const int64_t row = first < kBM ? rows[i] : min(n0 + first - kBM + (lane >> 3), p.n - 1);
            from[i] = (first < kBM ? p.x : p.w) + row * p.k + piece_of(i);
        }
    }
    if (tail) {
        uint4 v[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            v[i] = make_uint4(0, 0, 0, 0);
            if (piece_of(i) < tail) v[i] = *(const uint4*)(from[i] + (p.k - tail));
            if (piece_of(i) >= p.k) from[i] -= piece_of(i);  // (loads of steps that there are not stay inside the row)
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) *(uint4*)(lds + (wave * kLoads + i) * 1024 + lane * 16) = v[i];
    }
    int ahead = tail ? 1 : 0;  // the step that is loaded next; behind the last one it is loaded again, to where it is not read
    int to = ahead, on = 0;    // its stage
    auto load_one = [&](int i) {
        load_to_lds(from[i], lds + to * kStage + (wave * kLoads + i) * 1024);
        from[i] += on;
    };
    auto loaded = [&]() {
        ++ahead;
        to = to + 1 == kStages ? 0 : to + 1;
        on = ahead + 1 < steps ? 128 : 0;
    };
    on = ahead + 1 < steps ? 128 : 0;
    for (int s = ahead; s < kStages; ++s) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_one(i);
        loaded();
    }

    const int wm = wave / kWN * kTM * 32, wn = wave % kWN * kTN * 32;
    // of row lane % 32 piece lane / 32, of which pieces + 2, + 4, + 6 are those with another bit
    const int at = (lane & 31) * 128 + place(lane & 31, lane >> 5) * 16;
    struct Operands {
        int4v x[2][kTM], w[2][kTN];
    };
    constexpr int kReads = 2 * (kTM + kTN), kProducts = 2 * kTM * kTN;
    auto fetch_one = [&](Operands& o, int stage, int half, int r) {
        const int h = r / (kTM + kTN), i = r % (kTM + kTN);
        const int8_t* s = lds + stage * kStage + (at ^ (half * 64 + h * 32));
        if (i < kTM) o.x[h][i] = *(const int4v*)(s + (wm + i * 32) * 128);
        else o.w[h][i - kTM] = *(const int4v*)(s + (kBM + wn + (i - kTM) * 32) * 128);
    };
    int16v dot[kTM][kTN] = {};
    // The products of 64 values of k, and between them the reads of the next 64's operands and loads of a later step: a wavefront has its
    // SIMD with one other at most and issues in order, so that loads in a row would leave the matrix unit without work
    // while they queue.
    auto half_step = [&](const Operands& now, Operands& next, int stage, int half, bool loads) {
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
            const int h = m / (kTM * kTN), i = m / kTN % kTM, j = m % kTN;
            dot[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(now.w[h][j], now.x[h][i], dot[i][j], 0, 0, 0);
#pragma unroll
            for (int r = m * kReads / kProducts; r < (m + 1) * kReads / kProducts; ++r) fetch_one(next, stage, half, r);
            if (loads)
#pragma unroll
                for (int l = m * kLoads / kProducts; l < (m + 1) * kLoads / kProducts; ++l) load_one(l);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    Operands a, b;
    // the first step lies in the LDS
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 1) * kLoads) : "memory");
#pragma unroll
    for (int r = 0; r < kReads; ++r) fetch_one(a, 0, 0, r);
    int stage = 0;
    for (int s = 0; s < steps; ++s) {
        half_step(a, b, stage, 1, false);
        // the next step lies in the LDS for all wavefronts, and none reads this one any more
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
        stage = stage + 1 == kStages ? 0 : stage + 1;
        half_step(b, a, stage, 0, true);
        loaded();
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");  // the steps are read, and nothing is on its way to them
    // All loads come before the first store: a wait for a load would be one for the stores before it too.
    const int half = lane >> 5;
    auto word = [&](int at, int i) { return *(const int*)(lds + at + i * 4); };
    // Two rows of tiles at a time: all at once do not fit the registers, and one by one they take as many trips to memory.
    constexpr int kAtOnce = kTM < 4 ? 1 : 2;
    uint4 out[kTM][kTN][2];
#pragma unroll
    for (int i0 = 0; i0 < kTM; i0 += kAtOnce) {
        float16v sum[kAtOnce][kTN];
        ProjectRow mine[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int m = wm + 32 * (i0 + i) + (lane & 31);
            mine[i] = {p.order ? word(kRowOf, m) : (int)min(m0 + m, (int64_t)p.n_rows - 1), -1, __int_as_float(word(kScale, m)), 1.0f};
            if (p.a) {
                const int of = word(kAdapter, m);
                if (m0 + m < p.n_rows && of >= 0 && of < p.n_adapters) {
                    mine[i].adapter = of;
                    mine[i].power = __int_as_float(word(kPower, m));
                }
                if (kBf16) mine[i].scale *= project_inverse(mine[i].power);
            }
#pragma unroll
            for (int j = 0; j < kTN; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int4v ws = *(const int4v*)(lds + kColumn + (wn + 32 * j + 8 * g + 4 * half) * 4);
#pragma unroll
                    for (int u = 0; u < 4; ++u) sum[i][j][4 * g + u] = (float)dot[i0 + i][j][4 * g + u] * mine[i].scale * __int_as_float(ws[u]);
                }
            if (!kBf16 && p.a)
#pragma unroll
                for (int j = 0; j < kTN; ++j)
#pragma unroll
                    for (int u = 0; u < 16; ++u) sum[i][j][u] *= project_inverse(mine[i].power);
        }
        if (p.a) project_add_adapters<kBf16, kAtOnce, kTN>(p, sum, mine, n0 + wn);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) project_round<kBf16, kTN>(sum[i], mine[i].power, out[i0 + i]);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < kTM; ++i) {
        const int m = wm + 32 * i + (lane & 31), row = p.order ? word(kRowOf, m) : (int)min(m0 + m, (int64_t)p.n_rows - 1);
        if constexpr (kTN == 2) project_store_lines(p, out[i], m0 + m < p.n_rows ? row : -1, n0 + wn, lds + wave * 4096);
        else project_store<kTN>(p, out[i], m0 + m < p.n_rows ? (int64_t)row : (int64_t)p.n_rows, n0 + wn);
    }
}

// ---------------------------------------------------------------- few rows
// Up to 32 kTM rows to a workgroup: bound by the weights' way from memory, read once for as many (4096 x 5120: one row 7.2 us a call, 64 9.3, of which a launch is 5;
// 64 of 32 adapters of rank 16 18).  A workgroup has 32 columns; rows and weights come to the LDS kStages - 1 steps of 256 values of k ahead, of
// which each wavefront multiplies 32; they join their sums in the LDS.  Then each wavefront has a tile and every kShare-th adapter among the
// rows: it multiplies those, and stores the rows (its lanes) that have one of them.  Tried: further adapters' operands four at a time too
// (the same); the parts of the inner values summed before this kernel, by workgroups of all parts (18.9 for 18.2 with rank 16, 19.7 for
// 22.6 with three adapters of rank 128).
constexpr int kFewWaves = 8;

// kWithInner: the adapters' inner values are summed here too, by each workgroup for itself, a part of k by each wavefront: one launch
// where the rows' adapters have up to kFusedRanks ranks in all and few values (rank 16, one row, from 512 values: a call 7.0 us against 9.9 with a
// kernel of their own, from 4096 14.6 against 12.7; rank 32, from 4096: 18.5 and 13.5).
constexpr int kFusedRanks = 32, kFusedValues = 32768;  // ranks times k

template <bool kBf16, int kTM, bool kWithInner>
__global__ __launch_bounds__(kFewWaves * 64) void project_few_kernel(ProjectArgs p)
{
    static_assert(kFewWaves == kInnerParts, "a wavefront to each part of k");
    static_assert(!kWithInner || kTM == 1, "few rows");
    constexpr int kRows = 32 * kTM + 32, kLoads = kRows / 4 / kFewWaves;  // of a step, and loads of 1024 bytes of a wavefront
    constexpr int kStages = kTM == 1 ? 4 : 5;
    constexpr int kShare = kFewWaves / kTM;   // wavefronts to a tile
    constexpr int kHeld = 4;                  // operands of adapters (16 ranks x 32 columns) that are loaded ahead
    // the sums and the inner values (first halves and second halves of a row) take the place of the steps
    constexpr int kSteps = kStages * kRows * 256, kInner = kFewWaves * kTM * 4096, kLow = ST_MAX_RANK, kInnerRow = 2 * ST_MAX_RANK + 8;
    static_assert(kInner + 32 * kTM * kInnerRow * 2 <= kSteps, "they fit");
    constexpr int kPower = kSteps, kParts = kPower + 32 * kTM * 4;
    // (one array for all, read as int4v: beside another, or read as a struct, the compiler has the reads of a step wait for the loads of later ones)
    __shared__ __align__(1024) int8_t lds[kParts + (kWithInner ? kInnerParts * kFusedRanks * 4 : 0)];
    int32_t(*s_dot)[kTM][1024] = (int32_t(*)[kTM][1024])lds;
    uint16_t(*s_inner)[kInnerRow] = (uint16_t(*)[kInnerRow])(lds + kInner);
    float* s_power = (float*)(lds + kPower);
    float* s_parts = (float*)(lds + kParts);  // [part][row][rank]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * 32, n = n0 + (lane & 31);
    const int row0 = blockIdx.y * (32 * kTM), n_rows = min(p.n_rows - row0, 32 * kTM);  // rows are counted from row0 on
    // (what others' addresses come from is asked for before the steps: loads end in the order in which they begin)
    const int tile = wave / kShare, share = wave % kShare;
    const int row = 32 * tile + (lane & 31);
    const float scale = row < n_rows ? p.x_scale[row0 + row] : 0.0f;
    const int asked = p.a && row < n_rows ? p.adapter_of[row0 + row] : -1;
    float4v ws[1][4];
    project_scales<1>(p, ws, n0);
    // the parts of the inner values: kWide threads to a row, two ranks at a time
    constexpr int kWide = kFewWaves * 2 / kTM, kTurns = ST_MAX_RANK / 2 / kWide;
    const int m = tid / kWide, l = tid % kWide;
    const int part_asked = p.a && m < n_rows ? p.adapter_of[row0 + m] : -1;
    const float part_scale = p.a && m < n_rows ? p.x_scale[row0 + m] : 0.0f;
    // what this lane loads: of each four rows row lane / 16, the piece that lies at place lane % 16
    const int8_t* from[kLoads];
    const int steps = (p.k + 255) >> 8, tail = p.k & 255;
    auto piece_of = [&](int i) { return ((lane & 15) ^ (((wave * kLoads + i) * 4 + (lane >> 4)) & 15)) * 16; };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int at = (wave * kLoads + i) * 4 + (lane >> 4);
        const bool rows = at < 32 * kTM;
        from[i] = (rows ? p.x : p.w) + (int64_t)(rows ? row0 + min(at, n_rows - 1) : min(n0 + at - 32 * kTM, p.n - 1)) * p.k + piece_of(i);
    }
    int ahead = 0, to = 0;  // the step that is loaded next and its stage; behind the last one it is loaded again, to where it is not read
    if (tail) {
        uint4 v[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            v[i] = make_uint4(0, 0, 0, 0);
            if (piece_of(i) < tail) v[i] = *(const uint4*)(from[i] + (p.k - tail));
            if (piece_of(i) >= p.k) from[i] -= piece_of(i);  // (loads of steps that there are not stay inside the row)
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) *(uint4*)(lds + (wave * kLoads + i) * 1024 + lane * 16) = v[i];
        ahead = to = 1;
    }
    auto load = [&]() {
        const int on = ahead + 1 < steps ? 256 : 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            load_to_lds(from[i], lds + to * (kRows * 256) + (wave * kLoads + i) * 1024);
            from[i] += on;
        }
        ++ahead;
        to = to + 1 == kStages ? 0 : to + 1;
    };
    while (ahead < kStages - 1) load();
    const int adapter = asked >= 0 && asked < p.n_adapters ? asked : -1, part_of = part_asked >= 0 && part_asked < p.n_adapters ? part_asked : -1;
    // the adapters of the tile's rows: lanes that are the first with theirs, and of those the wavefront's
    uint32_t left = 0;
    bool stores = true;
    const int ranks16 = (p.rank + 15) >> 4;
    int next = 0, c = 0;  // the adapter and chunk of ranks whose operand comes next; c == ranks16: go on to another
    uint4 held[kHeld];
    int held_of[kHeld];
    auto operand = [&](int a, int at) -> uint4 {
        const int r = at * 16 + (lane >> 5) * 8;
        if (n < p.n && r < p.rank) return *(const uint4*)(p.b + ((int64_t)a * p.n + n) * p.rank + r);
        return make_uint4(0, 0, 0, 0);
    };
    auto advance = [&]() -> bool {
        if (++c < ranks16) return true;
        if (!left) return false;
        next = __builtin_amdgcn_readlane(adapter, __builtin_ctz(left));
        left &= left - 1;
        c = 0;
        return true;
    };
    if (p.a) {
        bool again = adapter < 0;
        int first = lane & 31;  // the first row with this one's adapter
        for (int i = min(n_rows - 32 * tile, 32) - 1; i >= 0; --i)
            if (__builtin_amdgcn_readlane(adapter, i) == adapter) first = i;
        again = again || first != (lane & 31);
        const uint32_t firsts = (uint32_t)ballot(!again);
        const int index = __builtin_popcount(firsts & ((1u << first) - 1));  // of this row's adapter among them
        stores = adapter < 0 ? share == 0 : index % kShare == share;
        left = (uint32_t)ballot(!again && index % kShare == share);
        c = ranks16 - 1;
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        held_of[i] = -1;
        if (p.a && advance()) {
            held_of[i] = next * 8 + c;
            held[i] = operand(next, c);
        }
    }
    if (kWithInner) {
        InnerPart<kBf16, 1, 1, 36> inner;
        const int8_t* xs[1] = {p.x + (int64_t)min(lane & 15, p.n_rows - 1) * p.k + (lane >> 4) * 16};
        const int of[1] = {project_adapter(p, lane & 15)};
        for (int a = next_of<16>(of, -1); a != 0x7FFFFFFF; a = next_of<16>(of, a))
            for (int rank0 = 0; rank0 < p.rank; rank0 += 16) {
                inner.first_x(xs, wave, p.k);
                inner.run(xs, p.a + ((int64_t)a * p.rank + rank0 + (lane & 15)) * p.k + (lane >> 4) * 16, p.rank - rank0, wave, p.k);
                const int r = rank0 + (lane >> 4) * 4;
                if (of[0] == a && r < p.rank) *(float4v*)&s_parts[(wave * p.n_rows + (lane & 15)) * p.rank + r] = inner.acc[0][0];
            }
        __syncthreads();
    }
    float alpha = 0.0f;
    const bool has = part_of >= 0;
    float2 parts[kTurns][kInnerParts];
    if (has) {
        alpha = p.alpha[part_of];
#pragma unroll
        for (int t = 0; t < kTurns; ++t)
            if (2 * (t * kWide + l) < p.rank)
#pragma unroll
                for (int q = 0; q < kInnerParts; ++q)
                    parts[t][q] = *(const float2*)((kWithInner ? s_parts : p.parts) + ((int64_t)q * p.n_rows + row0 + m) * p.rank + 2 * (t * kWide + l));
    }
    int16v dot[kTM] = {};
    // a wavefront has 32 of a step's 256 values of k: pieces 2 wave and 2 wave + 1
    const int at = (lane & 31) * 256 + (((2 * wave + (lane >> 5)) ^ (lane & 15)) * 16);
    for (int s = 0, stage = 0; s < steps; ++s) {
        // this step lies in the LDS for all wavefronts, and none reads the one before any more
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
        load();
        const int8_t* held = lds + stage * (kRows * 256) + at;
        const int4v wv = *(const int4v*)(held + 32 * kTM * 256);
#pragma unroll
        for (int i = 0; i < kTM; ++i) dot[i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv, *(const int4v*)(held + i * 32 * 256), dot[i], 0, 0, 0);
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");  // the steps are read, and nothing is on its way to them
    if (p.a) {
        // the inner values: their parts summed in order, the power of two of the largest, rounding
        const float factor = alpha * part_scale;
        uint32_t top = 0;
        float2 v[kTurns];
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            v[t] = make_float2(0.0f, 0.0f);
            if (!has || 2 * (t * kWide + l) >= p.rank) continue;
            v[t] = parts[t][0];
#pragma unroll
            for (int q = 1; q < kInnerParts; ++q) {
                v[t].x += parts[t][q].x;
                v[t].y += parts[t][q].y;
            }
            v[t].x *= factor;
            v[t].y *= factor;
            top = max(top, max(__float_as_uint(v[t].x) & 0x7FFFFFFFu, __float_as_uint(v[t].y) & 0x7FFFFFFFu));
        }
        for (int o = kWide / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        const uint32_t e = project_exponent<kBf16>(top);
        const float down = __uint_as_float((254u - e) << 23);
#pragma unroll
        for (int t = 0; t < kTurns; ++t)
            if (2 * t * kWide < 16 * ranks16) {
                uint16_t h[4];
                two_halves<kBf16>(v[t].x * down, h, h + 2);
                two_halves<kBf16>(v[t].y * down, h + 1, h + 3);
                uint16_t* at = &s_inner[m][2 * (t * kWide + l)];
                *(uint32_t*)at = h[0] | (uint32_t)h[1] << 16;
                *(uint32_t*)(at + kLow) = h[2] | (uint32_t)h[3] << 16;
            }
        if (l == 0) s_power[m] = has ? __uint_as_float(e << 23) : 1.0f;
    }
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) *(int4*)&s_dot[wave][i][g * 256 + lane * 4] = make_int4(dot[i][4 * g], dot[i][4 * g + 1], dot[i][4 * g + 2], dot[i][4 * g + 3]);
    __syncthreads();
    if (tid < 256 * kTM) {  // four sums to a thread
        int4* at = (int4*)&s_dot[0][0][0] + tid;
        int4 d = *at;
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v) {
            const int4 o = at[v * 256 * kTM];
            d = make_int4(d.x + o.x, d.y + o.y, d.z + o.z, d.w + o.w);
        }
        *at = d;
    }
    __syncthreads();
    const float power = p.a ? s_power[row] : 1.0f, inverse = project_inverse(power), x_scale = kBf16 ? scale * inverse : scale;
    float16v sum[1];
#pragma unroll
    for (int u = 0; u < 16; ++u) sum[0][u] = (float)s_dot[0][tile][u / 4 * 256 + lane * 4 + u % 4] * x_scale * ws[0][u / 4][u % 4] * (kBf16 ? 1.0f : inverse);
    auto add = [&](int a, int at, const uint4& b) {
        InnerValues v = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (adapter == a) {
            const uint16_t* mine = &s_inner[row][at * 16 + (lane >> 5) * 8];
            v = {*(const uint4*)mine, *(const uint4*)(mine + kLow)};
        }
        sum[0] = project_with(sum[0], project_inner_products<kBf16>(b, v, sum[0]), adapter == a);
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (held_of[i] >= 0) add(held_of[i] >> 3, held_of[i] & 7, held[i]);
    if (p.a)
        while (advance()) add(next, c, operand(next, c));
    uint4 out[1][2];
    project_round<kBf16, 1>(sum, power, out);
    project_store<1>(p, out, stores && row < n_rows ? (int64_t)row0 + row : (int64_t)p.n_rows, n0);
}

}  // namespace st
