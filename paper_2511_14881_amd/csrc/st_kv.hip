// Entry points on cached histories (silvertorch.h): argument checks, launch shapes and launches.
#include "st_host.h"
#include "st_kv_attend_kernels.h"
#include "st_kv_cache_kernels.h"
#include "st_kv_rows_kernels.h"
#include "st_plan.h"

#include <algorithm>
#include <cmath>

namespace {

using st::fail;
using st::guarded;
using st::TimedLaunch;

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

int check_batch(const st_kv_batch* b)
{
    if (!b) return fail(ST_EINVAL, "null argument");
    if (b->n_seq < 0 || b->n_tok < 0 || b->max_tok < 0 || b->max_len < 0)
        return fail(ST_EINVAL, "negative size");
    if (b->max_blocks < 1 || b->max_blocks > ST_KV_MAX_BLOCKS)
        return fail(ST_EINVAL, "max_blocks=%d out of range", b->max_blocks);
    if (b->max_len > b->max_blocks * ST_KV_BLOCK)
        return fail(ST_EINVAL, "max_len=%d exceeds %d blocks", b->max_len, b->max_blocks);
    if (b->max_tok > b->n_tok) return fail(ST_EINVAL, "max_tok=%d exceeds n_tok=%d", b->max_tok, b->n_tok);
    if (b->n_seq == 0 && b->n_tok != 0) return fail(ST_EINVAL, "tokens of no sequence");
    if (!b->dev_offsets && (int64_t)b->n_seq * b->max_tok != b->n_tok)
        return fail(ST_EINVAL, "without offsets n_tok has to be n_seq * max_tok");
    if (b->n_seq > 0 && (!b->dev_tables || !b->dev_lengths)) return fail(ST_EINVAL, "null argument");
    return ST_OK;
}

bool known_dim(int32_t d) { return d == 64 || d == 96 || d == 128 || d == 256; }

int check_cache(const st_kv_cache* c, bool keys, bool values)
{
    if (!c) return fail(ST_EINVAL, "null argument");
    if (!known_dim(c->d)) return fail(ST_EINVAL, "d=%d must be 64, 96, 128 or 256", c->d);
    if (c->n_heads < 1 || c->n_heads > ST_KV_MAX_HEADS) return fail(ST_EINVAL, "n_heads=%d out of range", c->n_heads);
    if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFFll) return fail(ST_EINVAL, "n_pages=%lld out of range", (long long)c->n_pages);
    if (!c->dev_k_scale || (keys && !c->dev_k) || (values && (!c->dev_v || !c->dev_v_scale)) || !c->dev_bounds)
        return fail(ST_EINVAL, "null argument");
    if (misaligned(c->dev_k) || misaligned(c->dev_v) || misaligned(c->dev_k_scale) || misaligned(c->dev_v_scale) || misaligned(c->dev_bounds))
        return fail(ST_EINVAL, "misaligned cache (16 B)");
    return ST_OK;
}

int check_rows(const char* name, const void* p, int64_t stride, int64_t least, int32_t n)
{
    if (n == 0) return ST_OK;
    if (!p) return fail(ST_EINVAL, "null argument");
    if (stride < least || stride % 8 != 0 || misaligned(p))
        return fail(ST_EINVAL, "%s: rows of %lld elements, %lld apart, have to begin at multiples of 16 bytes", name, (long long)least, (long long)stride);
    return ST_OK;
}

int check_dtype(int32_t t) { return t == ST_BF16 || t == ST_F16 ? (int)ST_OK : fail(ST_EINVAL, "unknown dtype %d", t); }

int check_heads(const st_kv_cache* c, int32_t n_q_heads)
{
    if (n_q_heads < c->n_heads || n_q_heads % c->n_heads != 0 || n_q_heads > 64 * ST_KV_MAX_HEADS)
        return fail(ST_EINVAL, "n_q_heads=%d is no multiple of n_heads=%d", n_q_heads, c->n_heads);
    return ST_OK;
}

int check_mask(const uint64_t* mask, int32_t words, const st_kv_batch* b)
{
    if (!mask) return ST_OK;
    if ((uintptr_t)mask & 7) return fail(ST_EINVAL, "misaligned mask (8 B)");
    if (words < (b->max_len + 63) / 64) return fail(ST_EINVAL, "mask rows of %d words do not cover max_len=%d", words, b->max_len);
    return ST_OK;
}

int check_grid(int64_t groups)  // (a launch has fewer than 2^32 threads)
{
    return groups <= 0xFFFFFFll ? (int)ST_OK : fail(ST_EINVAL, "too many rows for one call: %lld workgroups of at most 16777215 (they go by n_seq times max_tok)", (long long)groups);
}

st::KvCacheView view(const st_kv_cache* c)
{
    return {c->dev_k, c->dev_v, c->dev_k_scale, c->dev_v_scale, c->dev_bounds, c->n_pages, c->n_heads};
}
st::KvBatchView view(const st_kv_batch* b)
{
    return {b->dev_tables, b->dev_lengths, b->dev_offsets, b->n_seq, b->max_blocks, b->n_tok, b->max_tok, b->max_len};
}

int blocks_of(int32_t tokens) { return (tokens + ST_KV_BLOCK - 1) / ST_KV_BLOCK; }

// body(std::integral_constant<int, d>)
template <class F>
int with_dim(int32_t d, F&& body)
{
    switch (d) {
    case 64: return body(std::integral_constant<int, 64>());
    case 96: return body(std::integral_constant<int, 96>());
    case 128: return body(std::integral_constant<int, 128>());
    case 256: return body(std::integral_constant<int, 256>());
    }
    return fail(ST_EINVAL, "d=%d must be 64, 96, 128 or 256", d);
}

// Rows of a sequence and head up to which tiles of 16 read the cache themselves, as against tiles of 256 (d = 256: 128) rows that
// share it.  8 x 16384 tokens, 4 heads, us: d = 64, 96 rows 43 against 52, 192 rows 66 against 58; d = 96, 96 rows 53 against 62,
// 128 rows 68 against 63; d = 128, 64 rows 56.2 against 55.3, 96 rows 72 against 58; d = 256, 80 rows 114 against 129, 128 rows
// 204 against 136.  Where all is little, the shared tiles leave most of the chip idle: one sequence of 4000 tokens, 192 rows,
// d = 64 14 against 18, d = 128 19 against 26, d = 256 27 against 39.
constexpr int64_t kLittle = 512;  // blocks of all sequences and heads
constexpr int few_rows(int d, int64_t blocks) { return blocks <= kLittle ? 256 : d > 128 ? 96 : d > 96 ? 64 : 128; }
constexpr int row_waves(int d) { return d > 128 ? 4 : 8; }  // of the kernel for many rows (256: 512 registers to a lane)
// Tiles of 16 rows from which on a wavefront takes a tile by itself.  Calls in us, a wavefront to a tile against four: 8 selected blocks,
// 1600 tiles 41 against 43, 3200 67 against 72, 6400 102 against 109; 11 blocks, 2048 tiles 55 against 57.  Longer lists do not
// gain: 2048 tiles of up to 32 blocks 134 against 130, 4096 of them 271 against 245, 1536 of up to 70 blocks 153 against 130.
constexpr int kManyRows = 2048;
// Blocks of a split, at least: one for each wavefront that takes blocks by itself, two where the workgroup takes them together.
// 1500 tokens, 4 heads: 16 rows, d = 128, 13.2 us against 15.8 with splits of 16 blocks; d = 256, 15.2 against 23.6; 256 rows,
// d = 128, 23.0 against 45.5.  A list of up to whole_list blocks is not split, joining would take longer: 700 tokens, 16 rows,
// d = 128, 11.2 us against 13.2.
constexpr int least_chunk(bool many) { return many ? 2 : 4; }
constexpr int whole_list(int d) { return d > 128 ? 8 : 16; }
// Many rows: a block takes about this long in microseconds; joining splits this long, and the partial outputs' way out and in.  A list is
// not split where that takes longer (4 heads, 600 rows, calls in us): 8 histories of 300 tokens whole 21.5, split 32.0; 4 of 700 tokens split
// 30.8, whole 33.8; of 1500 tokens 33.5 and 54.9 (d = 64 27 and 38, d = 256, 400 rows, 46 and 105), of 3000 42 and 96.
constexpr double rows_block_us(int d) { return d > 128 ? 3.0 : 1.7; }
constexpr double kRowsJoinUs = 3.0, kRowsJoinBytes = 5e6;  // of a microsecond
// Start of a workgroup, and joining splits, in blocks: what decides where the last round of workgroups is to be filled.  Calls in us with
// these, with (0, 0) and with (12, 18): 64 selected blocks for 24 x 8 sequences and heads 61, 62, 62; 48 for 40 x 8 78, 82, 81; 32 for 175 x 4
// 100, 112, 93; 1500 tokens over one history of 4000, 8 heads 94, 103, 87; 800 over 8000, 4 heads 87, 85, 86.
constexpr double kSplitStart = 4.0, kSplitJoin = 6.0;
constexpr int kDies = 8;  // of the chip, each with an L2 of its own

struct AttendPlan {
    bool many;          // the kernel for many rows
    int32_t tile_rows, tiles, chunk, splits, rows_pad, entries, dies, waves;
    int32_t join_waves;  // to a row whose splits are joined; 0: nothing to join
    int32_t sum_lanes;   // lanes to a block where a kernel of its own sums the weights; 0: none does
    int64_t units;
    int64_t grid, sum_grid;
    int64_t o_bytes, ml_bytes, block_bytes, row_bytes;
    int64_t bytes() const { return o_bytes + ml_bytes + block_bytes + row_bytes; }
};

// Which kernel, and how the blocks of a row are split over workgroups: a function of the call's sizes alone.
AttendPlan attend_plan(const st_kv_cache* c, const st_kv_batch* b, int32_t n_q_heads, int32_t n_sel, bool mass)
{
    AttendPlan p;
    const int32_t group = n_q_heads / c->n_heads;
    const int64_t rows = (n_sel > 0 ? 1 : (int64_t)b->max_tok) * group;  // of a unit and head
    p.units = n_sel > 0 ? b->n_tok : b->n_seq;
    const int32_t list = std::max(1, n_sel > 0 ? std::min(n_sel, blocks_of(b->max_len)) : blocks_of(b->max_len));
    p.many = n_sel == 0 && rows > few_rows(c->d, (int64_t)b->n_seq * c->n_heads * list);
    p.tile_rows = p.many ? row_waves(c->d) * 32 : 16;
    p.tiles = (int32_t)((rows + p.tile_rows - 1) / p.tile_rows);
    p.rows_pad = (int32_t)st::round_up(rows, 16);
    p.entries = n_sel > 0 ? n_sel : list;
    const int64_t pairs = std::max<int64_t>(1, p.units * p.tiles * c->n_heads);
    p.waves = pairs >= kManyRows ? 1 : 4;
    // Workgroups that the chip holds at a time (registers and LDS), and splits of a row's blocks: one round of workgroups where
    // there are few rows (as long as a split has work for its wavefronts), two where sequences of different lengths
    // would leave a single round to the longest, and for a lone sequence what wastes least of its last round.  (Calls in us with 4, 3 and
    // 2 workgroups to a compute unit for d = 64, 96 and more, with 2 for all and with 4: d = 64, 40 x 8192 tokens, 8 heads 51, 55, 51; d = 96 72, 79,
    // 75; d = 128, 64 x 8192 149, 149, 159; d = 256, 24 x 6000 87, 87, 91.)
    const int64_t slots = (int64_t)st::kComputeUnits * (p.many ? 1 : c->d <= 64 ? 4 : c->d <= 96 ? 3 : 2);
    int64_t splits = 1;
    if (p.waves == 1 && !p.many) splits = 1;
    else if (pairs * 4 <= slots) splits = slots / pairs;
    else if (b->n_seq > 1 && n_sel == 0) splits = (slots + pairs - 1) / pairs;
    else {
        double best = 1e30;
        for (int64_t s = 1; s <= 16; ++s) {
            const double rounds = (double)((pairs * s + slots - 1) / slots);
            const double cost = rounds * ((double)((list + s - 1) / s) + kSplitStart) + (s > 1 ? kSplitJoin : 0.0);
            if (cost < best) best = cost, splits = s;
        }
    }
    int32_t chunk = (int32_t)std::max<int64_t>(least_chunk(p.many), (list + splits - 1) / splits);
    bool whole = chunk >= list;
    if (p.many) {
        const double parts = (double)(rows * b->n_seq * c->n_heads) * ((list + chunk - 1) / chunk);
        whole = whole || (list - chunk) * rows_block_us(c->d) < kRowsJoinUs + parts * c->d * 8 / kRowsJoinBytes;
    } else {
        whole = whole || list <= whole_list(c->d);
    }
    if (whole) chunk = p.entries;
    p.chunk = chunk;
    p.splits = (p.entries + chunk - 1) / chunk;
    // Parts that read the same blocks go to one die, where sequences, heads and splits are enough to keep all dies alike (one
    // sequence of 100000 tokens, 4 heads of 128, 64 rows: 48 us against 72).
    const int64_t sh = (int64_t)b->n_seq * c->n_heads, per = (int64_t)p.tiles * (n_sel > 0 ? b->max_tok : 1);
    const int64_t keys = sh * p.splits;
    p.dies = per > 1 && (keys % kDies == 0 || keys >= 8 * kDies) ? kDies : 1;
    p.grid = st::round_up(keys, p.dies) * per;
    // (calls of one history in us, a wavefront to a row against four: 8 splits 11.9 against 12.2, 16 12.4 and 12.5, 32 13.2 and 12.4, 63 15.6 and 13.5)
    p.join_waves = p.splits >= 16 ? 4 : p.splits > 1 ? 1 : 0;
    // (one workgroup to each sequence and head writes the weights itself, unless there are no tokens)
    const bool whole_pairs = n_sel == 0 && !p.many && p.tiles == 1 && p.splits == 1 && !b->dev_offsets && b->max_tok > 0;
    p.sum_lanes = !mass || b->n_seq == 0 || whole_pairs ? 0 : p.rows_pad > 16 ? 64 : 16;
    const int of = p.sum_lanes ? st::kKvThreads / p.sum_lanes : 1;
    p.sum_grid = p.sum_lanes == 0 ? 0 : n_sel > 0 ? sh : sh * ((b->max_blocks + of - 1) / of);
    const int64_t uh = p.units * c->n_heads;
    const int64_t parts = p.splits > 1 ? uh * p.splits * p.rows_pad : 0;
    p.o_bytes = st::round_up(parts * c->d * 4, 256);
    p.ml_bytes = st::round_up(parts * 16, 256);
    p.block_bytes = mass ? st::round_up(uh * p.entries * p.rows_pad * 8, 256) : 0;
    p.row_bytes = mass ? st::round_up(uh * p.rows_pad * 8, 256) : 0;
    return p;
}

template <int D, bool kSelected>
int launch_attend(const st::KvAttendArgs& a, const AttendPlan& p, hipStream_t stream)
{
    {
        TimedLaunch t(0, stream);
        const dim3 grid((unsigned)p.grid);
        if (p.many && a.exact) hipLaunchKernelGGL((st::kv_attend_rows_kernel<D, row_waves(D), true>), grid, dim3(row_waves(D) * 64), 0, stream, a);
        else if (p.many) hipLaunchKernelGGL((st::kv_attend_rows_kernel<D, row_waves(D), false>), grid, dim3(row_waves(D) * 64), 0, stream, a);
        else if (p.waves == 1) hipLaunchKernelGGL((st::kv_attend_kernel<D, kSelected, 1>), grid, dim3(64), 0, stream, a);
        else hipLaunchKernelGGL((st::kv_attend_kernel<D, kSelected, 4>), grid, dim3(256), 0, stream, a);
    }
    if (p.join_waves) {
        TimedLaunch t(1, stream);
        const int64_t rows = (int64_t)a.b.n_tok * a.c.n_heads * a.group;
        if (p.join_waves == 4) hipLaunchKernelGGL((st::kv_join_kernel<D, kSelected, 4>), dim3((unsigned)rows), dim3(st::kKvThreads), 0, stream, a);
        else hipLaunchKernelGGL((st::kv_join_kernel<D, kSelected, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(st::kKvThreads), 0, stream, a);
    }
    return ST_OK;
}

int64_t select_stride(const st_kv_batch* b) { return st::round_up(std::max(1, blocks_of(b->max_len)), 16); }

struct SelectPlan {
    bool one;              // the workgroup that scores also chooses
    int32_t chunks, rounds;  // workgroups to the blocks of a tile of tokens, and rounds of kKvScoreBlocks of each
    int32_t keys;          // that a lane holds where a wavefront chooses; 0: a workgroup chooses
    int64_t groups;
};

SelectPlan select_plan(const st_kv_cache* c, const st_kv_batch* b)
{
    const int32_t blocks = std::max(1, blocks_of(b->max_len)), tiles = (b->max_tok + 15) / 16;
    const int64_t pairs = (int64_t)b->n_seq * c->n_heads;
    SelectPlan p = {false, 1, 1, blocks <= 256 ? 4 : blocks <= 512 ? 8 : blocks <= 1024 ? 16 : 0, 0};
    // One token to a sequence: the workgroup that scores also chooses, as long as its blocks are few enough to be read by one
    // (or there are as many sequences and heads as compute units anyway).  Selection and attention in us, one kernel against two: 8 sequences and
    // heads of 512 blocks 22.6 against 24.5, of 1024 25.0 and 24.8, of 1500 31.2 and 27.2; 32 of 2500 45 and 35; 256 of 100 blocks 23.6 and
    // 27.1, of 1500 27.7 and 35.1.
    p.one = b->max_tok == 1 && (blocks <= 1024 || pairs >= st::kComputeUnits);
    if (!p.one) {
        // rounds of 256 blocks to a workgroup: as many as still leave two workgroups to a compute unit
        const int all = (blocks + st::kKvScoreBlocks - 1) / st::kKvScoreBlocks;
        const int64_t want = std::max<int64_t>(1, 2ll * st::kComputeUnits / std::max<int64_t>(1, pairs * tiles));
        p.chunks = (int32_t)std::min<int64_t>(all, want);
        p.rounds = (all + p.chunks - 1) / p.chunks;
    }
    p.groups = pairs * tiles * p.chunks;
    return p;
}

// Kernels whose dynamic LDS may pass the default limit: the limit is raised once.
template <class K>
int allow_lds(K kernel, int bytes)
{
    if (bytes > 32 * 1024) ST_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024));
    return ST_OK;
}

}  // namespace

extern "C" {

int st_kv_append(const st_kv_cache* cache, const st_kv_batch* batch, const void* dev_k_new, int64_t k_stride,
                 const void* dev_v_new, int64_t v_stride, int32_t dtype, void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if ((rc = check_cache(cache, true, true)) || (rc = check_batch(batch)) || (rc = check_dtype(dtype))) return rc;
    const int64_t width = (int64_t)cache->n_heads * cache->d;
    if ((rc = check_rows("keys", dev_k_new, k_stride, width, batch->n_tok)) ||
        (rc = check_rows("values", dev_v_new, v_stride, width, batch->n_tok)))
        return rc;
    if (batch->n_tok == 0 || batch->max_tok == 0) return ST_OK;
    st::KvAppendArgs a = {view(cache), view(batch), dev_k_new, dev_v_new, k_stride, v_stride, dtype == ST_BF16,
                          (batch->max_tok + ST_KV_BLOCK - 2) / ST_KV_BLOCK + 1};
    const int64_t groups = 2ll * batch->n_seq * a.touched * cache->n_heads;
    if ((rc = check_grid(groups))) return rc;
    hipStream_t stream = (hipStream_t)hip_stream;
    with_dim(cache->d, [&](auto d) -> int {
        TimedLaunch t(0, stream);
        hipLaunchKernelGGL((st::kv_append_kernel<decltype(d)::value>), dim3((unsigned)groups), dim3(st::kKvThreads), 0, stream, a);
        return ST_OK;
    });
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

int st_kv_read(const st_kv_cache* cache, const st_kv_batch* batch, int32_t n_blocks, float* dev_out_k,
               float* dev_out_v, float* dev_out_bounds, void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if ((rc = check_cache(cache, true, true)) || (rc = check_batch(batch))) return rc;
    if (n_blocks < 1 || n_blocks > ST_KV_MAX_BLOCKS) return fail(ST_EINVAL, "n_blocks=%d out of range", n_blocks);
    if (misaligned(dev_out_k) || misaligned(dev_out_v) || misaligned(dev_out_bounds)) return fail(ST_EINVAL, "misaligned output (16 B)");
    const int64_t groups = 2ll * batch->n_seq * n_blocks * cache->n_heads;
    if ((rc = check_grid(groups))) return rc;
    if (groups == 0 || (!dev_out_k && !dev_out_v && !dev_out_bounds)) return ST_OK;
    st::KvReadArgs a = {view(cache), view(batch), n_blocks, dev_out_k, dev_out_v, dev_out_bounds};
    hipStream_t stream = (hipStream_t)hip_stream;
    with_dim(cache->d, [&](auto d) -> int {
        TimedLaunch t(0, stream);
        hipLaunchKernelGGL((st::kv_read_kernel<decltype(d)::value>), dim3((unsigned)groups), dim3(st::kKvThreads), 0, stream, a);
        return ST_OK;
    });
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

int st_kv_copy(const st_kv_cache* from, const st_kv_cache* to, const int32_t* dev_src, const int32_t* dev_dst, int32_t n,
               void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if ((rc = check_cache(from, true, true)) || (rc = check_cache(to, true, true))) return rc;
    if (from->n_heads != to->n_heads || from->d != to->d)
        return fail(ST_EINVAL, "pages of %d heads of %d do not fit a cache of %d heads of %d", from->n_heads, from->d, to->n_heads, to->d);
    if (n < 0) return fail(ST_EINVAL, "negative size");
    if (n == 0) return ST_OK;
    if (!dev_src || !dev_dst) return fail(ST_EINVAL, "null argument");
    if (((uintptr_t)dev_src & 3) || ((uintptr_t)dev_dst & 3)) return fail(ST_EINVAL, "misaligned list of pages (4 B)");
    st::KvCopyArgs a = {view(from), view(to), dev_src, dev_dst, 0, from->n_heads * from->d * (ST_KV_BLOCK / 16), from->n_heads * from->d / 8};
    a.parts = (a.rows16 + st::kKvThreads * st::kCopyLoads - 1) / (st::kKvThreads * st::kCopyLoads);
    const int64_t groups = (int64_t)n * (2 * a.parts + 1);
    if (groups > 0xFFFFFFll) return fail(ST_EINVAL, "too many pages for one call: %lld workgroups of at most 16777215", (long long)groups);
    {
        TimedLaunch t(0, (hipStream_t)hip_stream);
        hipLaunchKernelGGL(st::kv_copy_kernel, dim3((unsigned)groups), dim3(st::kKvThreads), 0, (hipStream_t)hip_stream, a);
    }
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

int64_t st_kv_attend_workspace_bytes(const st_kv_cache* cache, const st_kv_batch* batch, int32_t n_q_heads,
                                     int32_t n_sel, int32_t with_mass)
{
    int rc;
    if (!cache || !batch) return fail(ST_EINVAL, "null argument");
    if (!known_dim(cache->d) || cache->n_heads < 1 || cache->n_heads > ST_KV_MAX_HEADS) return fail(ST_EINVAL, "bad cache");
    if ((rc = check_batch(batch)) || (rc = check_heads(cache, n_q_heads))) return rc;
    if (n_sel < 0 || n_sel > ST_KV_MAX_BLOCKS) return fail(ST_EINVAL, "n_sel=%d out of range", n_sel);
    return std::max<int64_t>(256, attend_plan(cache, batch, n_q_heads, n_sel, with_mass != 0).bytes());
}

int st_kv_attend(const st_kv_cache* cache, const st_kv_batch* batch, const void* dev_q, int64_t q_stride,
                 int32_t dtype, int32_t n_q_heads, float softmax_scale, int32_t causal, const uint64_t* dev_mask,
                 int32_t mask_words, const int32_t* dev_blocks, int32_t n_sel, void* dev_out, float* dev_lse,
                 const float* dev_mass_in, float decay, float* dev_mass_out, void* dev_workspace,
                 int64_t workspace_bytes, void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if ((rc = check_cache(cache, true, true)) || (rc = check_batch(batch)) || (rc = check_dtype(dtype)) ||
        (rc = check_heads(cache, n_q_heads)) || (rc = check_mask(dev_mask, mask_words, batch)) ||
        (rc = check_rows("queries", dev_q, q_stride, (int64_t)n_q_heads * cache->d, batch->n_tok)))
        return rc;
    if (!std::isfinite(softmax_scale) || !std::isfinite(decay)) return fail(ST_EINVAL, "softmax_scale and decay have to be finite");
    if (dev_blocks ? n_sel < 1 || n_sel > ST_KV_MAX_BLOCKS : n_sel != 0) return fail(ST_EINVAL, "n_sel=%d out of range", n_sel);
    if (batch->n_tok > 0 && !dev_out) return fail(ST_EINVAL, "null argument");
    if (misaligned(dev_out) || ((uintptr_t)dev_lse & 3) || ((uintptr_t)dev_blocks & 3)) return fail(ST_EINVAL, "misaligned buffer (output 16 B)");
    if (dev_mass_in && !dev_mass_out) return fail(ST_EINVAL, "dev_mass_in without dev_mass_out");
    const bool mass = dev_mass_out != nullptr;
    const AttendPlan p = attend_plan(cache, batch, n_q_heads, n_sel, mass);
    if (p.bytes() > 0 && (!dev_workspace || workspace_bytes < p.bytes()))
        return fail(ST_EWORKSPACE, "workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)p.bytes());
    if ((uintptr_t)dev_workspace & 255) return fail(ST_EINVAL, "misaligned workspace (256 B)");
    if ((rc = check_grid(p.grid)) || (rc = check_grid((int64_t)batch->n_tok * n_q_heads))) return rc;
    char* ws = (char*)dev_workspace;
    st::KvAttendArgs a = {view(cache), view(batch), dev_q, q_stride, dtype == ST_BF16, n_q_heads / cache->n_heads, causal != 0,
                          softmax_scale * 1.44269504089f, dev_mask, mask_words, n_sel, dev_blocks, dev_out, dev_lse, mass || dev_lse,
                          p.chunk, p.splits, p.tiles, p.tile_rows, p.dies, (uint32_t)(batch->n_seq * cache->n_heads), p.rows_pad, (float*)ws, (float4*)(ws + p.o_bytes),
                          mass ? (float2*)(ws + p.o_bytes + p.ml_bytes) : nullptr, p.entries,
                          mass ? (float2*)(ws + p.o_bytes + p.ml_bytes + p.block_bytes) : nullptr, dev_mass_in, decay, dev_mass_out};
    // all that can be refused is, before anything is written
    if ((rc = check_grid(p.sum_grid))) return rc;
    if (p.sum_lanes && n_sel > 0 && (rc = allow_lds(&st::kv_mass_selected_kernel, batch->max_blocks * 4))) return rc;
    hipStream_t stream = (hipStream_t)hip_stream;
    if (batch->n_tok > 0 && batch->max_tok > 0)
        with_dim(cache->d, [&](auto d) -> int {
            return n_sel > 0 ? launch_attend<decltype(d)::value, true>(a, p, stream) : launch_attend<decltype(d)::value, false>(a, p, stream);
        });
    if (p.sum_lanes) {
        TimedLaunch t(1, stream);
        const dim3 groups((unsigned)p.sum_grid);
        if (n_sel > 0) hipLaunchKernelGGL(st::kv_mass_selected_kernel, groups, dim3(st::kKvThreads), batch->max_blocks * 4, stream, a);
        else if (p.sum_lanes == 64) hipLaunchKernelGGL(st::kv_mass_kernel<64>, groups, dim3(st::kKvThreads), 0, stream, a);
        else hipLaunchKernelGGL(st::kv_mass_kernel<16>, groups, dim3(st::kKvThreads), 0, stream, a);
    }
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

int64_t st_kv_select_workspace_bytes(const st_kv_cache* cache, const st_kv_batch* batch, int32_t n_q_heads, int32_t n_sel)
{
    int rc;
    if (!cache || !batch) return fail(ST_EINVAL, "null argument");
    if (!known_dim(cache->d) || cache->n_heads < 1 || cache->n_heads > ST_KV_MAX_HEADS) return fail(ST_EINVAL, "bad cache");
    if ((rc = check_batch(batch)) || (rc = check_heads(cache, n_q_heads))) return rc;
    if (n_sel < 1 || n_sel > ST_KV_MAX_BLOCKS) return fail(ST_EINVAL, "n_sel=%d out of range", n_sel);
    return std::max<int64_t>(256, st::round_up((int64_t)batch->n_tok * cache->n_heads * select_stride(batch) * 4, 256));
}

int st_kv_select(const st_kv_cache* cache, const st_kv_batch* batch, const void* dev_q, int64_t q_stride, int32_t dtype,
                 int32_t n_q_heads, int32_t causal, const uint64_t* dev_mask, int32_t mask_words, int32_t n_sel,
                 int32_t sink, int32_t recent, int32_t* dev_out_blocks, void* dev_workspace, int64_t workspace_bytes,
                 void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if ((rc = check_cache(cache, false, false)) || (rc = check_batch(batch)) || (rc = check_dtype(dtype)) ||
        (rc = check_heads(cache, n_q_heads)) || (rc = check_mask(dev_mask, mask_words, batch)) ||
        (rc = check_rows("queries", dev_q, q_stride, (int64_t)n_q_heads * cache->d, batch->n_tok)))
        return rc;
    if (n_sel < 1 || n_sel > ST_KV_MAX_BLOCKS) return fail(ST_EINVAL, "n_sel=%d out of range", n_sel);
    if (sink < 0 || recent < 0 || (int64_t)sink + recent > n_sel) return fail(ST_EINVAL, "sink=%d and recent=%d exceed n_sel=%d", sink, recent, n_sel);
    if (batch->n_tok > 0 && !dev_out_blocks) return fail(ST_EINVAL, "null argument");
    if ((uintptr_t)dev_out_blocks & 3) return fail(ST_EINVAL, "misaligned output (4 B)");
    const int64_t need = st_kv_select_workspace_bytes(cache, batch, n_q_heads, n_sel);
    if (need < 0) return (int)need;
    if (!dev_workspace || workspace_bytes < need)
        return fail(ST_EWORKSPACE, "workspace has %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
    if ((uintptr_t)dev_workspace & 255) return fail(ST_EINVAL, "misaligned workspace (256 B)");
    if (batch->n_tok == 0 || batch->max_tok == 0) return ST_OK;
    const SelectPlan p = select_plan(cache, batch);
    st::KvSelectArgs a = {view(cache), view(batch), dev_q, q_stride, dtype == ST_BF16, n_q_heads / cache->n_heads, causal != 0,
                          dev_mask, mask_words, n_sel, sink, recent, (batch->max_tok + 15) / 16, p.chunks, p.rounds, select_stride(batch),
                          (uint32_t*)dev_workspace, dev_out_blocks};
    const int64_t rows = (int64_t)batch->n_tok * cache->n_heads;
    if ((rc = check_grid(p.groups)) || (rc = check_grid(rows))) return rc;
    hipStream_t stream = (hipStream_t)hip_stream;
    const int lds = (int)select_stride(batch) * 4;
    rc = with_dim(cache->d, [&](auto d) -> int {
        constexpr int D = decltype(d)::value;
        int rc2;
        // (256 threads for 8 x 1024 blocks 28.2 us against 25.0, 256 x 1500 34.1 against 27.7; 1024 threads 25.1 and 27.4)
        constexpr int kOneThreads = 512;
        if (p.one && (rc2 = allow_lds(&st::kv_score_kernel<D, true, kOneThreads>, lds))) return rc2;
        TimedLaunch t(0, stream);
        if (p.one) hipLaunchKernelGGL((st::kv_score_kernel<D, true, kOneThreads>), dim3((unsigned)p.groups), dim3(kOneThreads), lds, stream, a);
        else hipLaunchKernelGGL((st::kv_score_kernel<D, false, st::kKvThreads>), dim3((unsigned)p.groups), dim3(st::kKvThreads), 0, stream, a);
        return ST_OK;
    });
    if (rc != ST_OK) return rc;
    if (!p.one) {
        if (p.keys == 0 && (rc = allow_lds(&st::kv_choose_kernel, lds))) return rc;
        TimedLaunch t(1, stream);
        const dim3 waves((unsigned)((rows + 3) / 4));
        if (p.keys == 4) hipLaunchKernelGGL(st::kv_choose_wave_kernel<4>, waves, dim3(st::kKvThreads), 0, stream, a);
        else if (p.keys == 8) hipLaunchKernelGGL(st::kv_choose_wave_kernel<8>, waves, dim3(st::kKvThreads), 0, stream, a);
        else if (p.keys == 16) hipLaunchKernelGGL(st::kv_choose_wave_kernel<16>, waves, dim3(st::kKvThreads), 0, stream, a);
        else hipLaunchKernelGGL(st::kv_choose_kernel, dim3((unsigned)rows), dim3(st::kKvThreads), lds, stream, a);
    }
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

int st_kv_host_plan(const st_kv_cache* cache, const st_kv_batch* batch, int32_t n_q_heads, int32_t n_sel, int32_t with_mass,
                    int32_t* host_out_plan)
{
    return guarded([&]() -> int {
    int rc;
    if (!host_out_plan) return fail(ST_EINVAL, "null argument");
    if ((rc = check_cache(cache, false, false)) || (rc = check_batch(batch)) || (rc = check_heads(cache, n_q_heads))) return rc;
    if (n_sel < 0 || n_sel > ST_KV_MAX_BLOCKS) return fail(ST_EINVAL, "n_sel=%d out of range", n_sel);
    const AttendPlan a = attend_plan(cache, batch, n_q_heads, n_sel, with_mass != 0);
    const SelectPlan s = select_plan(cache, batch);
    const int32_t plan[10] = {a.many ? 0 : a.waves, a.tiles, a.chunk, a.splits, a.join_waves, a.sum_lanes, s.one, s.chunks, s.rounds, s.keys};
    std::copy(plan, plan + 10, host_out_plan);
    return ST_OK;
    });
}

int st_kv_evict(const st_kv_batch* batch, const float* dev_mass, int32_t n_heads, int32_t budget, int32_t sink,
                int32_t recent, int32_t* dev_out_tables, int32_t* dev_out_lengths, float* dev_out_mass,
                int32_t* dev_out_freed, int32_t* dev_out_n_freed, void* hip_stream)
{
    return guarded([&]() -> int {
    int rc;
    if ((rc = check_batch(batch))) return rc;
    if (n_heads < 1 || n_heads > ST_KV_MAX_HEADS) return fail(ST_EINVAL, "n_heads=%d out of range", n_heads);
    if (recent < 1 || sink < 0 || (int64_t)sink + recent > budget)
        return fail(ST_EINVAL, "budget=%d, sink=%d, recent=%d: recent is at least 1 and both fit the budget", budget, sink, recent);
    if (batch->n_seq == 0) return ST_OK;
    if (!dev_mass || !dev_out_tables || !dev_out_lengths || !dev_out_mass || !dev_out_freed || !dev_out_n_freed)
        return fail(ST_EINVAL, "null argument");
    st::KvEvictArgs a = {view(batch), dev_mass, n_heads, budget, sink, recent, dev_out_tables, dev_out_lengths, dev_out_mass,
                         dev_out_freed, dev_out_n_freed};
    const int lds = batch->max_blocks * 8;
    if ((rc = allow_lds(&st::kv_evict_kernel, lds))) return rc;
    {
        TimedLaunch t(1, (hipStream_t)hip_stream);
        hipLaunchKernelGGL(st::kv_evict_kernel, dim3((unsigned)batch->n_seq), dim3(st::kKvEvictThreads), lds, (hipStream_t)hip_stream, a);
    }
    ST_HIP(hipGetLastError());
    return ST_OK;
    });
}

}  // extern "C"
