// Entry points of a layer around the cached histories (silvertorch.h): argument checks, launch shapes and launches.
#include "st_host.h"
#include "st_layer_kernels.h"
#include "st_plan.h"
#include "st_project_kernels.h"

#include <algorithm>
#include <cmath>

namespace {

using st::fail;
using st::guarded;
using st::TimedLaunch;

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Rows that a call reads or writes; NULL passes.
int check_rows(const char* name, const void* p, int64_t stride, int64_t least)
{
    if (!p) return ST_OK;
    if (stride < least || stride % 8 != 0 || misaligned(p))
        return fail(ST_EINVAL, "%s: rows of %lld elements, %lld apart, have to begin at multiples of 16 bytes", name, (long long)least, (long long)stride);
    return ST_OK;
}

int check_grid(int64_t groups)  // (a launch has fewer than 2^32 threads)
{
    return groups <= 0x7FFFFFll ? (int)ST_OK : fail(ST_EINVAL, "too many rows for one call: %lld workgroups of at most 8388607", (long long)groups);
}

template <int kType, int kLanes, int kVectors>
int launch_norm(const st::NormArgs& a, hipStream_t stream)
{
    const int64_t groups = (a.n_rows + st::kLayerThreads / kLanes - 1) / (st::kLayerThreads / kLanes);
    int rc;
    if ((rc = check_grid(groups))) return rc;
    TimedLaunch t(0, stream);
    hipLaunchKernelGGL((st::norm_rows_kernel<kType, kLanes, kVectors>), dim3((unsigned)groups), dim3(st::kLayerThreads), 0, stream, a);
    return ST_OK;
}

// Threads to a row: enough that each holds few vectors, few enough that rows of a few hundred bytes share a wavefront.
template <int kType>
int norm_of_type(const st::NormArgs& a, hipStream_t stream)
{
    if (a.d <= 128) return launch_norm<kType, 16, 1>(a, stream);
    if (a.d <= 512) return launch_norm<kType, 64, 1>(a, stream);
    if (a.d <= 1024) return launch_norm<kType, 64, 2>(a, stream);
    if (a.d <= 2048) return launch_norm<kType, 64, 4>(a, stream);
    if (a.d <= 4096) return launch_norm<kType, 256, 2>(a, stream);
    if (a.d <= 8192) return launch_norm<kType, 256, 4>(a, stream);
    return launch_norm<kType, 256, 8>(a, stream);
}

int check_project(int32_t n_rows, int32_t k, int32_t n, const st_adapters* adapters)
{
    if (n_rows < 0) return fail(ST_EINVAL, "negative size");
    if (k < 16 || k > ST_MAX_ROW || k % 16 != 0) return fail(ST_EINVAL, "k=%d must be a multiple of 16 up to %d", k, ST_MAX_ROW);
    if (n < 16 || n > ST_MAX_OUT || n % 16 != 0) return fail(ST_EINVAL, "n=%d must be a multiple of 16 up to %d", n, ST_MAX_OUT);
    if (!adapters) return ST_OK;
    if (adapters->n_adapters < 1 || adapters->n_adapters > ST_MAX_ADAPTERS) return fail(ST_EINVAL, "n_adapters=%d out of range", adapters->n_adapters);
    if (adapters->rank < 8 || adapters->rank > ST_MAX_RANK || adapters->rank % 8 != 0)
        return fail(ST_EINVAL, "rank=%d must be a multiple of 8 up to %d", adapters->rank, ST_MAX_RANK);
    return ST_OK;
}

// Rows that a workgroup takes where there are few, and rows up to which there may be several such workgroups to 32 columns: as long as the
// compute units take all of them at once, they need no more time than one, and the adapters' inner values come in over the whole chip, unless
// those are many.  Calls in us, tiles / this, mixed rows: k = 4096, n = 896, 96 rows without adapters 9.8 / 8.2, 36 adapters of rank 16
// 30.4 / 17.3, 8 of 128 61 / 31, 192 rows 58 / 38, 384 rows 10.3 / 8.5, 26.0 / 23.2, 54.4 / 53.6; 96 rows, k = n = 512 6.6 / 6.5, 19.9 / 11.8, 28.5 / 19.6;
// 229 rows, 752, 1568, 20 of 128 32.9 / 35.4; 128 rows, 512, 4096 6.6 / 6.4, 18.6 / 12.3.  In more than one round: 96 rows, k = 4096, n = 5120 10.7 / 14.8;
// of more rows: 1024, 4096, 256, 36 adapters of rank 16 25.1 / 36.8.
constexpr int kFewRows = 64, kFewMost = 384, kFewRanks = 24576;  // of all rows
int32_t project_most_few(int32_t n, const st_adapters* a)
{
    const int32_t most = std::min(kFewMost, st::kComputeUnits / ((n + 31) / 32) * kFewRows);
    return std::max(kFewRows, a ? std::min(most, kFewRanks / a->rank) : most);
}
bool project_few(int32_t n_rows, int32_t n, const st_adapters* a) { return n_rows <= project_most_few(n, a); }

// Rows up to which a workgroup that sums inner values takes 16, beyond 32.  Kernel in us, 16 / 32 / 64: 2048 rows, k = 4096, rank 16 9.9 / 11.7 /
// 17.4; 4096, 1024, 64 14.5 / 13.9 / 18.7; 16384, 4096, 32 57 / 36 / 39.
constexpr int kOneTileRows = 2048;
// Whether rows are brought into the order of their adapters first: each adapter more in a tile costs loads and products by its rank.
// Calls in us, as they come / ordered, mixed rows: k = 4096, n = 5120: 256 rows, 32 adapters of rank 16 37.1 / 30.6, 2048, 2 of 16 59.6 / 63.4, 8 of 16
// 93 / 64, 16384, 3 of 32 428 / 375, 16 of 32 823 / 389; 1040, 1296: 1001, 5 of 8 16.0 / 15.6, 2 of 32 13.4 / 16.9, 300, 3 of 64 14.7 / 14.6; 2048, 2560:
// 4096, 2 of 16 39.7 / 43.4, 2 of 64 51.3 / 53.9, 3 of 32 51.6 / 46.0, 16384, 3 of 32 167 / 140; 1024, 1024: 4096, 16 of 64 119 / 34.5.  Rows that come in
// runs pay for it: 1000, 2048, 2560, 16 of 16 22.1 / 26.5, 16384, 4096, 5120, 16 of 32 366 / 372.
bool project_ordered(int32_t n_rows, const st_adapters* a)
{
    return a->n_adapters >= 5 || (n_rows > kOneTileRows && (a->n_adapters - 1) * a->rank >= 64);
}

struct ProjectPlan {
    int64_t inner, power, order;  // bytes
    int64_t bytes() const { return inner + power + order; }
};

ProjectPlan project_plan(int32_t n_rows, int32_t n, const st_adapters* adapters)
{
    if (!adapters) return {0, 0, 0};
    const int64_t values = (int64_t)n_rows * adapters->rank, words = st::round_up((int64_t)n_rows * 4, 256);
    if (project_few(n_rows, n, adapters)) return {st::round_up(values * 4 * st::kInnerParts, 256), 0, 0};
    return {st::round_up(values * 4, 256), words, project_ordered(n_rows, adapters) ? words : 0};
}

// Bytes that are enough for every call of up to n_rows rows: the few rows' parts take more to a row than what many rows need, so that the most
// rows that go that way may need more than n_rows do.
int64_t project_bytes(int32_t n_rows, int32_t n, const st_adapters* adapters)
{
    const int32_t few = std::min(n_rows, project_most_few(n, adapters));
    return std::max(project_plan(n_rows, n, adapters).bytes(), project_plan(few, n, adapters).bytes());
}

// Edge of the tiles of many rows by an estimate of the call's microseconds.  64 (three workgroups to a compute unit): the longer of one
// workgroup's way alone and its share of all; 128 (two): rounds, and a quarter for the last; 256 (one): whole rounds and the last by how
// full it is.  Measured with 64 / 128 / 256 (k x n, rows): 4096 x 5120, 256 15.3 / 23.9 / 46, 512 22.6 / 24.4 / 47, 1024 40 / 35 / 48, 2048
// 71 / 60 / 52, 4096 135 / 101 / 107, 8192 287 / 205 / 182, 16384 561 / 403 / 329; 2048 x 2560, 1024 14.3 / 15.9 / 29, 4096 40 / 36 / 32,
// 8192 77 / 58 / 64; 1024 x 1024, 2048 7.4 / 10.4 / 19, 8192 22.5 / 18.1 / 22.2; 512 x 8192, 512 9.9 / 8.9 / 15, 2048 29 / 23 / 22, 8192
// 113 / 91 / 109.
int project_edge(int32_t n_rows, int32_t k, int32_t n)
{
    const double steps = (k + 127) / 128;
    auto tiles = [&](int64_t edge) { return (double)((n_rows + edge - 1) / edge * ((n + edge - 1) / edge)); };
    const double c64 = std::max(3.5 + 0.24 * steps, 4 + tiles(64) * (0.0035 + 0.00078 * steps));
    const double c128 = std::max(6 + 0.55 * steps, (tiles(128) / (2 * st::kComputeUnits) + 0.25) * (6 + 1.05 * steps));
    const double all = tiles(256) / st::kComputeUnits, full = std::floor(all), last = all - full;
    const double c256 = full * std::max(23.0, 12 + 1.55 * steps) + (last > 0 ? std::max(18.0, 8 + (1.25 + 0.3 * last) * steps) : 0);
    return c64 <= c128 && c64 <= c256 ? 64 : c128 <= c256 ? 128 : 256;
}

template <bool kBf16, int kM>
void launch_inner(const st::ProjectArgs& p, hipStream_t stream)
{
    const int64_t tiles = (p.n_rows + 16ll * kM - 1) / (16 * kM);
    const int64_t split = std::max<int64_t>(1, std::min<int64_t>({1024 / tiles, p.n_adapters, 16 * kM}));
    const dim3 groups((unsigned)tiles, (unsigned)split), threads(st::kInnerParts * 64);
    if (p.rank <= 16) hipLaunchKernelGGL((st::project_inner_kernel<kBf16, 1, kM>), groups, threads, 0, stream, p);
    else if (p.rank <= 32) hipLaunchKernelGGL((st::project_inner_kernel<kBf16, 2, kM>), groups, threads, 0, stream, p);
    else if (p.rank <= 64) hipLaunchKernelGGL((st::project_inner_kernel<kBf16, 4, kM>), groups, threads, 0, stream, p);
    else hipLaunchKernelGGL((st::project_inner_kernel<kBf16, 8, kM>), groups, threads, 0, stream, p);
}

// What a call runs: a function of its sizes alone.
struct ProjectRoute {
    bool few, fused;  // few: a workgroup takes 64 rows; fused: it sums the inner values too
    int edge;         // of the tiles where there are many
    bool order;
    int64_t tiles;
};

ProjectRoute project_route(int32_t n_rows, int32_t k, int32_t n, const st_adapters* adapters)
{
    ProjectRoute r;
    r.few = project_few(n_rows, n, adapters);
    const int64_t ranks = adapters ? (int64_t)n_rows * ((adapters->rank + 15) / 16 * 16) : 0;
    r.fused = adapters && ranks <= st::kFusedRanks && ranks * k <= st::kFusedValues;
    r.edge = project_edge(n_rows, k, n);
    r.order = adapters && !r.few && project_ordered(n_rows, adapters);
    r.tiles = r.few ? (n + 31) / 32 : ((int64_t)n_rows + r.edge - 1) / r.edge * ((n + r.edge - 1) / r.edge);
    return r;
}

template <bool kBf16>
void launch_project(const st::ProjectArgs& p, const ProjectRoute& r, hipStream_t stream)
{
    if (p.a && !r.fused) {
        TimedLaunch t(1, stream);
        if (p.order)
            hipLaunchKernelGGL(st::project_order_kernel, dim3((unsigned)((p.n_rows + (int64_t)st::kOrderRows - 1) / st::kOrderRows)), dim3(st::kOrderThreads), 0, stream, p);
        if (r.few)
            hipLaunchKernelGGL((st::project_parts_kernel<kBf16>), dim3((unsigned)((p.n_rows + 15) / 16), (unsigned)std::min({p.n_adapters, p.n_rows, 16}),
                                                                       (unsigned)((p.rank + 15) / 16 * st::kInnerParts)), dim3(64), 0, stream, p);
        else if (p.n_rows <= kOneTileRows) launch_inner<kBf16, 1>(p, stream);
        else launch_inner<kBf16, 2>(p, stream);
    }
    TimedLaunch t(0, stream);
    const dim3 groups((unsigned)r.tiles, r.few ? (unsigned)((p.n_rows + kFewRows - 1) / kFewRows) : 1u), few(st::kFewWaves * 64);
    if (r.fused) hipLaunchKernelGGL((st::project_few_kernel<kBf16, 1, true>), groups, few, 0, stream, p);
    else if (r.few && p.n_rows <= 32) hipLaunchKernelGGL((st::project_few_kernel<kBf16, 1, false>), groups, few, 0, stream, p);
    else if (r.few) hipLaunchKernelGGL((st::project_few_kernel<kBf16, 2, false>), groups, few, 0, stream, p);
    else if (r.edge == 64) hipLaunchKernelGGL((st::project_tile_kernel<kBf16, 2, 2, 1, 1, 3>), groups, dim3(256), 0, stream, p);
    else if (r.edge == 128) hipLaunchKernelGGL((st::project_tile_kernel<kBf16, 2, 2, 2, 2, 2>), groups, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((st::project_tile_kernel<kBf16, 2, 4, 4, 2, 2>), groups, dim3(512), 0, stream, p);
}

}  // namespace

extern "C" {

int st_norm_rows(const void* dev_x, int64_t x_stride, const void* dev_residual, int64_t residual_stride,
                 const void* dev_weight, int32_t dtype, int64_t n_rows, int32_t d, int32_t normalise, float eps,
                 void* dev_out_sum, int64_t sum_stride, int8_t* dev_out_q, float* dev_out_scale, void* dev_out_y,
                 void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if (dtype != ST_BF16 && dtype != ST_F16 && dtype != ST_F32) return fail(ST_EINVAL, "unknown dtype %d", dtype);
    if (n_rows < 0 || n_rows > 0x7FFFFFFFll) return fail(ST_EINVAL, "n_rows=%lld out of range", (long long)n_rows);
    if (d < 16 || d > ST_MAX_ROW || d % 16 != 0) return fail(ST_EINVAL, "d=%d must be a multiple of 16 up to %d", d, ST_MAX_ROW);
    if (normalise && !(eps >= 1e-12f && eps <= 1.0f)) return fail(ST_EINVAL, "eps=%g must be in [1e-12, 1]", (double)eps);
    if (n_rows == 0) return ST_OK;
    if (!dev_x || (!dev_out_sum && !dev_out_q && !dev_out_y) || !dev_out_q != !dev_out_scale) return fail(ST_EINVAL, "null argument");
    if ((rc = check_rows("x", dev_x, x_stride, d)) || (rc = check_rows("residual", dev_residual, residual_stride, d)) ||
        (rc = check_rows("sum", dev_out_sum, sum_stride, d)))
        return rc;
    if ((dev_out_sum == dev_x && sum_stride != x_stride) || (dev_out_sum && dev_out_sum == dev_residual && sum_stride != residual_stride))
        return fail(ST_EINVAL, "a sum in the place of x or of the residual keeps its stride");
    if (dev_out_y && (dev_out_y == dev_x || dev_out_y == dev_residual || dev_out_y == dev_out_sum))
        return fail(ST_EINVAL, "the norm's output lies apart from its inputs and from the sum");
    if (misaligned(dev_weight) || misaligned(dev_out_q) || misaligned(dev_out_y) || ((uintptr_t)dev_out_scale & 3))
        return fail(ST_EINVAL, "misaligned buffer (16 B)");
    const st::NormArgs a = {dev_x, dev_residual, dev_weight, dev_out_sum, dev_out_q, dev_out_scale, dev_out_y, x_stride, residual_stride,
                            sum_stride, n_rows, d, normalise != 0, eps};
    hipStream_t stream = (hipStream_t)hip_stream;
    rc = dtype == ST_BF16 ? norm_of_type<ST_BF16>(a, stream) : dtype == ST_F16 ? norm_of_type<ST_F16>(a, stream) : norm_of_type<ST_F32>(a, stream);
    if (rc != ST_OK) return rc;
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

int64_t st_project_workspace_bytes(int32_t n_rows, int32_t k, int32_t n, const st_adapters* adapters)
{
    int rc;
    if ((rc = check_project(n_rows, k, n, adapters))) return rc;
    return std::max<int64_t>(256, project_bytes(n_rows, n, adapters));
}

int st_project(const int8_t* dev_x, const float* dev_x_scale, int32_t n_rows, int32_t k, const int8_t* dev_w,
               const float* dev_w_scale, int32_t n, const st_adapters* adapters, const int32_t* dev_adapter_of,
               int32_t dtype, void* dev_out, int64_t out_stride, void* dev_workspace, int64_t workspace_bytes,
               void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if (dtype != ST_BF16 && dtype != ST_F16) return fail(ST_EINVAL, "unknown dtype %d", dtype);
    if ((rc = check_project(n_rows, k, n, adapters))) return rc;
    if (n_rows == 0) return ST_OK;
    if (!dev_x || !dev_x_scale || !dev_w || !dev_w_scale || !dev_out || !adapters != !dev_adapter_of ||
        (adapters && (!adapters->dev_a || !adapters->dev_b || !adapters->dev_alpha)))
        return fail(ST_EINVAL, "null argument");
    if (misaligned(dev_x) || misaligned(dev_w) || misaligned(dev_w_scale) || ((uintptr_t)dev_x_scale & 3) || ((uintptr_t)dev_adapter_of & 3) ||
        (adapters && (misaligned(adapters->dev_a) || misaligned(adapters->dev_b) || ((uintptr_t)adapters->dev_alpha & 3))))
        return fail(ST_EINVAL, "misaligned buffer (16 B)");
    if ((rc = check_rows("out", dev_out, out_stride, n))) return rc;
    if (dev_out == dev_x || dev_out == dev_w) return fail(ST_EINVAL, "the output lies apart from rows and weights");
    const ProjectPlan plan = project_plan(n_rows, n, adapters);
    if (plan.bytes() > 0 && (!dev_workspace || workspace_bytes < plan.bytes()))
        return fail(ST_EWORKSPACE, "workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)plan.bytes());
    if ((uintptr_t)dev_workspace & 255) return fail(ST_EINVAL, "misaligned workspace (256 B)");
    char* ws = (char*)dev_workspace;
    st::ProjectArgs p = {dev_x, dev_x_scale, dev_w, dev_w_scale, nullptr, nullptr, nullptr, dev_adapter_of, (uint16_t*)ws, (float*)(ws + plan.inner), (float*)ws,
                         plan.order ? (int32_t*)(ws + plan.inner + plan.power) : nullptr, dev_out, out_stride, n_rows, k, n, 0, 0};
    if (adapters) {
        p.a = (const uint16_t*)adapters->dev_a;
        p.b = (const uint16_t*)adapters->dev_b;
        p.alpha = adapters->dev_alpha;
        p.n_adapters = adapters->n_adapters;
        p.rank = adapters->rank;
    }
    const ProjectRoute route = project_route(n_rows, k, n, adapters);
    if ((rc = check_grid(route.tiles)) || (rc = check_grid(((int64_t)n_rows + 15) / 16))) return rc;
    hipStream_t stream = (hipStream_t)hip_stream;
    if (dtype == ST_BF16) launch_project<true>(p, route, stream);
    else launch_project<false>(p, route, stream);
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

int st_project_host_plan(int32_t n_rows, int32_t k, int32_t n, const st_adapters* adapters, int32_t* host_out_plan)
{
    return guarded([&]() -> int {
    int rc;
    if (!host_out_plan) return fail(ST_EINVAL, "null argument");
    if ((rc = check_project(n_rows, k, n, adapters))) return rc;
    const ProjectRoute r = project_route(n_rows, k, n, adapters);
    host_out_plan[0] = r.few ? 0 : r.edge;
    host_out_plan[1] = !adapters || r.fused ? 0 : r.few ? 1 : n_rows <= kOneTileRows ? 16 : 32;
    host_out_plan[2] = r.order;
    return ST_OK;
    });
}

int st_rotate(const void* dev_q, int64_t q_stride, int32_t n_q_heads, const void* dev_k, int64_t k_stride, int32_t n_k_heads,
              int32_t d, int32_t dtype, int32_t n_tok, const int32_t* dev_positions, const double* dev_freqs,
              const int32_t* host_sections, int32_t n_axes, int32_t interleaved, int32_t inverse, void* dev_out_q,
              int64_t out_q_stride, void* dev_out_k, int64_t out_k_stride, void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if (dtype != ST_BF16 && dtype != ST_F16) return fail(ST_EINVAL, "unknown dtype %d", dtype);
    if (n_tok < 0) return fail(ST_EINVAL, "negative size");
    if (d < 16 || d > 512 || d % 8 != 0) return fail(ST_EINVAL, "d=%d must be a multiple of 8 from 16 to 512", d);
    if (n_q_heads < 0 || n_k_heads < 0 || n_q_heads > 64 * ST_KV_MAX_HEADS || n_k_heads > ST_KV_MAX_HEADS)
        return fail(ST_EINVAL, "heads out of range");
    if (n_axes < 1 || n_axes > ST_MAX_AXES) return fail(ST_EINVAL, "n_axes=%d out of range", n_axes);
    if (!host_sections) return fail(ST_EINVAL, "null argument");
    st::RotateArgs a = {};
    for (int i = 0; i < n_axes; ++i) {
        if (host_sections[i] < 0 || host_sections[i] > d / 2) return fail(ST_EINVAL, "section of %d pairs out of range", host_sections[i]);
        a.pairs += host_sections[i];
        a.ends[i] = a.pairs;
    }
    if (a.pairs < 8 || a.pairs % 8 != 0 || a.pairs > d / 2) return fail(ST_EINVAL, "%d pairs must be a multiple of 8 up to d / 2 = %d", a.pairs, d / 2);
    if (n_tok == 0 || n_q_heads + n_k_heads == 0) return ST_OK;
    if (!dev_positions || !dev_freqs || (n_q_heads > 0 && (!dev_q || !dev_out_q)) || (n_k_heads > 0 && (!dev_k || !dev_out_k)))
        return fail(ST_EINVAL, "null argument");
    if (((uintptr_t)dev_positions & 3) || ((uintptr_t)dev_freqs & 7)) return fail(ST_EINVAL, "misaligned positions or frequencies");
    const int64_t q_width = (int64_t)n_q_heads * d, k_width = (int64_t)n_k_heads * d;
    if ((n_q_heads > 0 && ((rc = check_rows("queries", dev_q, q_stride, q_width)) || (rc = check_rows("queries out", dev_out_q, out_q_stride, q_width)))) ||
        (n_k_heads > 0 && ((rc = check_rows("keys", dev_k, k_stride, k_width)) || (rc = check_rows("keys out", dev_out_k, out_k_stride, k_width)))))
        return rc;
    if ((n_q_heads > 0 && dev_q == dev_out_q && q_stride != out_q_stride) || (n_k_heads > 0 && dev_k == dev_out_k && k_stride != out_k_stride))
        return fail(ST_EINVAL, "rows rotated in place keep their stride");
    if (n_q_heads > 0 && n_k_heads > 0 && (dev_out_q == dev_k || dev_out_k == dev_q || dev_out_q == dev_out_k))
        return fail(ST_EINVAL, "queries and keys are not rotated into each other's place");
    a.in[0] = (const uint16_t*)dev_q;
    a.in[1] = (const uint16_t*)dev_k;
    a.out[0] = (uint16_t*)dev_out_q;
    a.out[1] = (uint16_t*)dev_out_k;
    a.in_stride[0] = q_stride;
    a.in_stride[1] = k_stride;
    a.out_stride[0] = out_q_stride;
    a.out_stride[1] = out_k_stride;
    a.heads[0] = n_q_heads;
    a.heads[1] = n_k_heads;
    a.d = d;
    a.n_tok = n_tok;
    a.n_axes = n_axes;
    a.positions = dev_positions;
    a.freqs = dev_freqs;
    a.inverse = inverse != 0;
    a.columns = a.pairs / 8 + (d - 2 * a.pairs + 15) / 16;
    a.parts[0] = (n_q_heads + st::kRotateHeads - 1) / st::kRotateHeads;
    a.parts[1] = (n_k_heads + st::kRotateHeads - 1) / st::kRotateHeads;
    const int64_t groups = ((int64_t)n_tok * a.columns * (a.parts[0] + a.parts[1]) + st::kLayerThreads - 1) / st::kLayerThreads;
    if ((rc = check_grid(groups))) return rc;
    hipStream_t stream = (hipStream_t)hip_stream;
    const auto launch = [&](auto bf16, auto pairs) {
        TimedLaunch t(0, stream);
        hipLaunchKernelGGL((st::rotate_kernel<decltype(bf16)::value, decltype(pairs)::value>), dim3((unsigned)groups), dim3(st::kLayerThreads), 0, stream, a);
    };
    const auto yes = std::true_type();
    const auto no = std::false_type();
    if (dtype == ST_BF16) interleaved ? launch(yes, yes) : launch(yes, no);
    else interleaved ? launch(no, yes) : launch(no, no);
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

}  // extern "C"
