// Attention of many rows of a sequence (candidates, a prompt's chunk) over its cached history.
//
// Bound by the matrix units and the vector units beside them: 4 d operations to a row and token for the products, some five
// vector instructions to a weight.  A workgroup's wavefronts hold 32 rows each; a block's integers are turned into 16-bit floats
// once for all of them, on their way into the LDS (two blocks deep, the next one's integers in flight behind the products).
// As in the kernel for few rows a lane holds one row's logits, and weights go from one product to the other as they lie.  The
// products of the next block's keys stand beside the exponentials of this one's weights.  The value scale of a block is part of
// its weights, relative to a reference that each row has for itself and that follows the scales of the blocks it sees at a distance, so
// that the products accumulate into the outputs.
//
// 500 candidates to each of 16 histories of 1216 to 4096 tokens, 2 query heads to each of 4 heads of 128: 132 us, 660 TFLOP/s;
// with histories of one length 843 (a large product of matrices in 16 bits reaches 1390), since one round of workgroups lasts
// as long as the longest history.  2047 tokens over 15001, 5 query heads to each of 3 heads of 96, under a mask: 274 us and 19 to
// join.  With one part left out, 138 us (on another card) become 131 (exponentials), 120 (stores to the LDS), 127 (loads), 106 or 104 (either product):
// the parts hide behind each other about as far as two wavefronts of a SIMD let them.  256 rows to a workgroup of 8 wavefronts
// rather than 128 to one of 4: 132 against 152; two tiles of 32 rows to a wavefront, 4 wavefronts: 219; products and weights
// in turn on the two wavefronts of a SIMD, with a barrier between: 154.
#pragma once
#include "st_kv_attend_kernels.h"

namespace st {

typedef float float16v __attribute__((ext_vector_type(16)));

// A block's value scale over the row's reference is part of its weights between these two; beyond them the reference moves to the
// block's.  The least: weights are still of 11 significant bits down to 2^-20 of the row's largest, and rounding takes at
// most 2^-31 of the largest from the sum for each lighter token.  The most: a weight of 2^15 stays a 16-bit number.  The reference does
// not fall below kFall of the largest that the row has met (a smaller scale counts as that, off by 2^-73 of the largest
// value): outputs of 2^20 tokens stay below 2^124.  (A reference to each row rather than to the wavefront: 131.7 us against 130.6, 292
// against 284 with a mask.)
constexpr float kRhoLeast = 0.25f, kRhoMost = 1.875f, kFall = 0x1p-80f;

// kExact: lse or the blocks' weights are asked for (the case above: 16 us more for both).
template <int D, int kWaves, bool kExact>
__global__ __launch_bounds__(kWaves * 64, D > 128 ? 1 : 2) void kv_attend_rows_kernel(KvAttendArgs a)
{
    constexpr int kThreads = kWaves * 64, kRows = kWaves * 32, kSteps = D / 16, kCh = D / 32;
    constexpr int kKeyBytes = 2 * D + 16, kValBytes = 2 * kKvBlock + 16;  // rows of the LDS, an odd number of 16 bytes apart
    constexpr int kPieces = (4 * D + kThreads - 1) / kThreads;            // 16 bytes of keys, and of values, of a thread
    __shared__ __align__(16) char s_k[2][kKvBlock * kKeyBytes];
    __shared__ __align__(16) char s_v[2][D * kValBytes];
    __shared__ uint64_t s_any[kWaves][64];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const KvPlace at = kv_place<false>(a);
    if (at.unit < 0) return;
    const int split = at.split, head = at.head, unit = at.unit, row0 = at.tile * kRows;
    const KvTile t = kv_tile<false>(a, at.seq, unit, row0, kRows);
    if (row0 >= t.rows) return;
    const int jb = split * a.chunk, je = min(jb + a.chunk, t.n_list);
    if (split > 0 && jb >= je) return;
    const int64_t uh = (int64_t)unit * a.c.n_heads + head, heads_all = (int64_t)a.c.n_heads * a.group;
    const bool bf16 = a.bf16 != 0;

    const int row = row0 + w * 32 + n;
    const bool valid = row < t.rows;
    const KvRow of = kv_row(valid ? row : row0, t.tok_unit, head, a.group);
    const int lim = valid ? t.limit(of.i) : 0;
    half8 q[kSteps];
    float factor;
    const uint16_t* src = (const uint16_t*)a.q + of.tok * a.q_stride + of.q_head * D + h * 8;
    uint4 raw[kSteps];
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        raw[k] = make_uint4(0, 0, 0, 0);
        if (valid) raw[k] = *(const uint4*)(src + k * 16);
    }
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        float f[8];
        eight_floats(raw[k], bf16, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
    }
    float up;
    kv_query_unit(max_over_32(top), a.scale_log2, &up, &factor);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        float f[8];
        eight_floats(raw[k], bf16, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[k][j] = (_Float16)(f[j] * up);
    }
    float m = -__builtin_inff(), l = 0.0f, l_exact = 0.0f;
    float16v o[kCh];
#pragma unroll
    for (int c = 0; c < kCh; ++c) o[c] = float16v(0.0f);
    const bool busy = row0 + w * 32 < t.rows;                              // this wavefront has rows; all help with the blocks
    const int lim_all = t.limit(t.token(min(row0 + w * 32, t.rows - 1)));  // its rows see at least the positions below this one
    uint64_t far = 0;                                                      // rows of large logits (kv_far)
    float v_unit = 0.0f, v_top = 0.0f;                                     // outputs are in units of this value scale; the largest it was

    for (int j0 = jb; j0 < je; j0 += 64) {
        // up to 64 blocks: page and scales, one to a lane (the same in all wavefronts)
        const int j = j0 + lane;
        int page = j < je ? kv_page(a.c, a.b, t.seq, j) : -1;
        if (a.mask) {  // a block that no row of the tile sees is not read
            uint64_t any = 0;
            if (page >= 0)
                for (int64_t i = t.tok_first + w; i <= t.tok_last; i += kWaves) any |= a.mask[i * a.mask_words + j];
            __syncthreads();
            s_any[w][lane] = any;
            __syncthreads();
            for (int i = 0; i < kWaves; ++i) any |= s_any[i][lane];
            if (any == 0) page = -1;
        }
        const uint64_t all = ballot(j < je);
        uint64_t todo = ballot(page >= 0);
        if (a.block_ml)
            for (uint64_t dead = all & ~todo; dead; dead &= dead - 1)
                for (int r = tid; r < kRows && row0 + r < a.rows_pad; r += kThreads)
                    a.block_ml[(uh * a.entries + j0 + __builtin_ctzll(dead)) * a.rows_pad + row0 + r] = make_float2(0.0f, 0.0f);
        if (todo == 0) continue;
        const int64_t ph_l = (int64_t)max(page, 0) * a.c.n_heads + head;
        const float ks_l = page >= 0 ? a.c.k_scale[ph_l] : 0.0f, vs_l = page >= 0 ? a.c.v_scale[ph_l] : 0.0f;
        uint4 kraw[kPieces], vraw[kPieces];
        auto load = [&](const int8_t* from, int block, uint4* raw) {
            const int64_t ph = (int64_t)(int)lane_value((uint32_t)page, block) * a.c.n_heads + head;
            const uint4* src = (const uint4*)(from + ph * (D * kKvBlock));
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (4 * D % kThreads == 0 || i * kThreads + tid < 4 * D) raw[i] = src[i * kThreads + tid];
        };
        auto put_keys = [&](int buf) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int p = i * kThreads + tid;
                if (4 * D % kThreads == 0 || p < 4 * D) {
                    char* to = s_k[buf] + p / (D / 16) * kKeyBytes + p % (D / 16) * 32;
                    *(half8*)to = eight_halves(kraw[i].x, kraw[i].y);
                    *(half8*)(to + 16) = eight_halves(kraw[i].z, kraw[i].w);
                }
            }
        };
        auto put_values = [&](int buf, int block) {
            // (integers under a scale of zero are zeros)
            const uint32_t some = lane_value(__float_as_uint(vs_l), block) << 1 ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int p = i * kThreads + tid;
                if (4 * D % kThreads == 0 || p < 4 * D) {
                    // four neighbouring tokens to a word: half of the 8 that a lane's fragment of 16 tokens holds
                    char* to = s_v[buf] + p / 4 * kValBytes + (p & 1) * 16 + (p >> 1 & 1) * 8;
                    *(uint2*)to = halves_of_bytes(vraw[i].x & some);
                    *(uint2*)(to + 32) = halves_of_bytes(vraw[i].y & some);
                    *(uint2*)(to + 64) = halves_of_bytes(vraw[i].z & some);
                    *(uint2*)(to + 96) = halves_of_bytes(vraw[i].w & some);
                }
            }
        };
        auto products = [&](int buf, float16v (&x)[2]) {
            const char* bk = s_k[buf] + n * kKeyBytes + h * 16;
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                x[tt] = float16v(0.0f);
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    const half8 f = *(const half8*)(bk + tt * 32 * kKeyBytes + k * 32);
                    x[tt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, q[k], x[tt], 0, 0, 0);
                }
            }
        };
        // One block: x holds its products with the keys; next is filled with those of the block behind it.
        auto step = [&](int buf, int cur, int next, int third, float16v (&x)[2], float16v (&xn)[2]) {
            const int b = j0 + cur;
            load(a.c.k, third, kraw);
            load(a.c.v, next, vraw);
            // the scale of the values against the row's reference, which follows the blocks that the row sees
            const float vs = __uint_as_float(lane_value(__float_as_uint(vs_l), cur));
            const float ratio = vs != 0.0f ? vs * __builtin_amdgcn_rcpf(v_unit) : 1.0f;  // (an ulp or two off; exact divisions: 137 us against 134)
            float rho = fminf(fmaxf(ratio, kRhoLeast), kRhoMost);
            float rho_inv = __builtin_amdgcn_rcpf(rho), rho_log = __builtin_amdgcn_logf(rho);
            if (a.mask || (b + 1) * kKvBlock > lim_all) {
                const int left = lim - b * kKvBlock;
                uint64_t see = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0ull;
                if (a.mask && see) see &= a.mask[of.tok * a.mask_words + b];
                see >>= h * 4;
#pragma unroll
                for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[tt][i] = kv_seen(x[tt][i], (uint32_t)(see >> (tt * 32)), (i >> 2) * 8 + (i & 3));
            }
            float ks = fmaxf(__uint_as_float(lane_value(__float_as_uint(ks_l), cur)) * factor, 1e-37f);
            float top = x[0][0];
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, x[tt][i]);
            top = max_over_32(top) * ks;
            // seldom: the maximum or the reference moves, or logits are large
            const bool rises = top - m > kKvSlack, moves = top > -__builtin_inff() && ratio != rho;
            float shift = m == -__builtin_inff() ? 0.0f : m;
            if ((ballot(rises || moves) | far) != 0) {
                const float alpha = rises ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
                m = rises ? top : m;
                shift = m == -__builtin_inff() ? 0.0f : m;
                if (moves) v_top = fmaxf(v_top, v_unit);
                const float to = vs < v_top * kFall ? v_top * kFall : vs, f = moves ? v_unit / to * alpha : alpha;
                v_unit = moves ? to : v_unit;
                rho = moves ? 1.0f : rho;
                rho_inv = moves ? 1.0f : rho_inv;
                rho_log = moves ? 0.0f : rho_log;
                l *= alpha;
                if (kExact) l_exact *= alpha;
#pragma unroll
                for (int c = 0; c < kCh; ++c) o[c] *= f;
                far = ballot(kv_far(m));
                if (far) {
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[tt][i] = __fmul_rn(x[tt][i], ks) - shift;
                    ks = 1.0f;
                    shift = 0.0f;
                }
            }
            const float base = kKvLift + rho_log - shift;
            products(buf ^ 1, xn);
            half8 p[4];
            float sum = 0.0f;
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tt][i], ks, base));
                    if (kExact) sum += e;
                    p[tt * 2 + (i >> 3)][i & 7] = (_Float16)e;
                }
            float rounded = 0.0f;
#pragma unroll
            for (int u = 0; u < 4; ++u) rounded = add_halves(p[u], rounded);
            l = __builtin_fmaf(rounded, rho_inv, l);
            const float sums = sum * rho_inv;
            l_exact += sums;
            const char* bv = s_v[buf] + n * kValBytes + h * 16;
#pragma unroll
            for (int c = 0; c < kCh; ++c)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const half8 f = *(const half8*)(bv + c * 32 * kValBytes + u * 32);
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, p[u], o[c], 0, 0, 0);
                }
            put_keys(buf);
            put_values(buf ^ 1, next);
            if (kExact && a.block_ml) {
                const float both = sum_over_32(sums);
                if (h == 0 && row < t.rows) a.block_ml[(uh * a.entries + b) * a.rows_pad + row] = make_float2(m, both);
            }
            __syncthreads();
        };
        // the walk over the blocks to do: the last one again where there is none
        auto after = [&](int* it) {
            if (todo) {
                *it = __builtin_ctzll(todo);
                todo &= todo - 1;
                return 1;
            }
            return 0;
        };
        float16v xa[2], xb[2];
        int left = __builtin_popcountll(todo);
        int first = 0, second, third;
        after(&first);
        second = first;
        after(&second);
        third = second;
        after(&third);
        load(a.c.k, first, kraw);
        load(a.c.v, first, vraw);
        put_keys(0);
        put_values(0, first);
        load(a.c.k, second, kraw);
        put_keys(1);
        __syncthreads();
        if (busy) products(0, xa);
        __syncthreads();  // (the first step writes other keys where these were)
        // (loops of their own: with the choice inside the step its products and its stores are no longer interleaved)
        if (!busy) {
            for (int buf = 0; left > 0; --left, buf ^= 1) {
                load(a.c.k, third, kraw);
                load(a.c.v, second, vraw);
                put_keys(buf);
                put_values(buf ^ 1, second);
                second = third;
                after(&third);
                __syncthreads();
            }
            continue;
        }
        for (; left > 0; left -= 2) {
            step(0, first, second, third, xa, xb);
            first = second;
            second = third;
            after(&third);
            if (left == 1) break;
            step(1, first, second, third, xb, xa);
            first = second;
            second = third;
            after(&third);
        }
    }

    const float sum = sum_over_32(l), exact = kExact ? sum_over_32(l_exact) : 0.0f;
    if (row >= t.rows) return;
    if (t.n_list > a.chunk) {
        const int64_t part = (uh * a.splits + split) * a.rows_pad + row;
#pragma unroll
        for (int c = 0; c < kCh; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float4v y;
#pragma unroll
                for (int u = 0; u < 4; ++u) y[u] = o[c][4 * i + u];
                *(float4v*)(a.part_o + part * D + c * 32 + i * 8 + h * 4) = y;
            }
        if (h == 0) a.part_ml[part] = make_float4(m, sum, exact, v_unit);
        return;
    }
    const KvRow to = kv_row(row, t.tok_unit, head, a.group);  // (kept through the walk it would cost registers: 140 us against 133)
    const int64_t place = to.tok * heads_all + to.q_head;
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int c = 0; c < kCh; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t r[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) r[u] = to_16_bits(o[c][4 * i + u] * inv * v_unit, bf16);
            *(uint2*)((uint16_t*)a.out + place * D + c * 32 + i * 8 + h * 4) = make_uint2(r[0] | r[1] << 16, r[2] | r[3] << 16);
        }
    if (kExact && h == 0) {
        if (a.lse) a.lse[place] = exact == 0.0f ? -__builtin_inff() : (m - kKvLift + log2f(exact)) * 0.69314718056f;
        if (a.row_ml) a.row_ml[uh * a.rows_pad + row] = make_float2(m, exact);
    }
}

}  // namespace st
