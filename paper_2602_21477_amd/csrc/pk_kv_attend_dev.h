// Attention over a paged key/value cache: softmax(scale q k) v over the keys that a query sees, for chunks of new tokens
// and for single ones, over all of a sequence's pages or over listed blocks of them, with scores as they are or capped and biased.
// The kernels and the rules that choose them; pk_kv_attend*.hip compile them, a storage each.
#pragma once

#include <algorithm>
#include <cmath>

#include "pk_kv.h"

namespace pk {
namespace {


// How the second product's operands are scaled.  The largest weight is 2^top: in half precision that type has the more of its range
// below it (2^-39 of it is the smallest), in bfloat16 it keeps the products with denormal codes where 32 bits are normal, and small weights that
// alone make a channel which all heavy keys' 4 bits have as zero.  Each time a
// value's scale goes into the weight in units of the largest seen, so that no size of them overflows.
// One rounding of a weight is of the size of the result's own: against 64 bits a result is off by 2.1e-3, with weights of 32 bits by 1.6e-3
// (one bfloat16 token), by 2.9e-4 and 2.1e-4 (half precision over e4m3).  A second part would be the second product once more: only where
// bfloat16 has fewer bits than the codes are worth, which those of 4 bits are not.
template <int S, int T>
struct KvScaling {
    static constexpr bool CODED = kv_coded<S>, HALF = T == PK_F16;
    static constexpr bool TWICE = CODED && !HALF && S != PK_F4; // a weight is the sum of two numbers
    static constexpr bool UNITS = CODED && (HALF || S != PK_F8);
    static constexpr float top = HALF ? 15.f : S == PK_I8 ? 127.f : S == PK_F4 ? 16.f : 0.f;
    static constexpr float l_unit = !HALF && S == PK_I8 ? 0x1p-27f : 1.f; // of the sum of weights: it does not overflow
    // sums of weights, and of products (before the unit, of 2^-100 at least), in the end: both as if the largest weight were 1
    static constexpr float l_back = HALF ? 0x1p-15f : S == PK_I8 ? 0x1p-100f : S == PK_F4 ? 0x1p-16f : 1.f;
    static constexpr float o_back = S != PK_I8 ? l_back : HALF ? 0x1p9f : 0x1p6f;
};

// A query's part of the scores' scale.  PK_I8: the query times a power of two that keeps its products with denormal codes where 32 bits are
// normal (half precision needs none), and the start value of a product, from the sum of the scaled query.
template <int S, int T>
struct KvQueryScale {
    float near = 1.f, back = 1.f;
    __device__ __forceinline__ void largest(float most)
    {
        if constexpr (S == PK_I8 && T == PK_F16) back = 0x1p24f;
        if constexpr (S == PK_I8 && T == PK_BF16) {
            const int e = (int)((__float_as_uint(most) >> 23) & 0xffu) - 127, f = min(max(100 - e, 6), 127);
            near = __uint_as_float((uint32_t)(127 + f) << 23);
            back = __uint_as_float((uint32_t)(127 + 133 - f) << 23);
        }
    }
    __device__ __forceinline__ float start(float sum) const { return S != PK_I8 ? 0.f : -sum * (T == PK_F16 ? 0x1p-17f : 0x1p-126f); }
};
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A weight is 2^((x - m) qscale + top) for a score x and the largest m.  As x qscale - (m qscale - top), one operation less, it is off by the
// rounding of m qscale: 2^-16 at this size of it (powers of two), from 2^24 on more than the type of the weights has room for above top.
constexpr float kNear = 512.f;

// acc += A (16 rows x 32) B (32 x 16 columns), 16-bit operands
template <bool HALF>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 acc)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), acc, 0, 0, 0);
}

// Sixteen bytes of a row as operands of a product: one of 8 elements, two of 8 codes each, or (keys) four of 8 codes in 4 bits.
template <int S> constexpr int kv_operands = 16 / kv_bits<S>;
template <int S, int T, bool VALUES, int N>
__device__ __forceinline__ void operands(u32x4 w, float power, u32x4 (&to)[N])
{
    if constexpr (S == PK_F4) {
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = eight_of_4<T>(w[i], power);
    } else if constexpr (kv_coded<S>) {
        static_assert(N == 2, "");
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t lo, hi;
            codes_to<S, T, VALUES>(w[2 * i], lo, hi);
            to[i][0] = lo, to[i][1] = hi;
            codes_to<S, T, VALUES>(w[2 * i + 1], lo, hi);
            to[i][2] = lo, to[i][3] = hi;
        }
    } else {
        to[0] = w;
    }
}

// What a run of 16 tokens of channel tile d is in a lane's 16-byte loads of values: in 16 bits two loads, of which each is an operand; in 8 one; in
// 4 bits half a load, words of 8 tokens.
template <int S> constexpr int kv_value_loads = kv_bits<S> == 16 ? 2 : 1;
template <int S, int DT> constexpr int kv_value_words = S == PK_F4 ? DT / 2 : DT * kv_value_loads<S>;
template <int S, int T, int N>
__device__ __forceinline__ void value_operands(const u32x4 (&w)[N], int d, u32x4 &first, u32x4 &second)
{
    if constexpr (S == PK_F4) {
        first = eight_of_4<T>(w[d / 2][(d & 1) * 2], 1.f);
        second = eight_of_4<T>(w[d / 2][(d & 1) * 2 + 1], 1.f);
    } else if constexpr (kv_coded<S>) {
        u32x4 f[2];
        operands<S, T, true>(w[d], 1.f, f);
        first = f[0], second = f[1];
    } else {
        first = w[2 * d], second = w[2 * d + 1];
    }
}
// The bits of word i of such a load whose tokens, of the lane's 16, come before `held`.
template <int S>
__device__ __forceinline__ uint32_t held_bits(int word, int load, int held)
{
    constexpr int B = kv_bits<S>, EACH = 32 / B;
    const int first = (S == PK_F4 ? (word & 1) : kv_bits<S> == 8 ? word : load * 4 + word) * EACH;
    uint32_t keep = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) keep |= first + e < held ? ((1u << B) - 1) << (B * e) : 0u;
    return keep;
}

__device__ __forceinline__ float over_quarters_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float over_quarters_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// The largest of three (without the rounds that fmaxf makes for signalling NaNs).
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The largest of a number's values in 16 neighbouring lanes.
__device__ __forceinline__ float over_row_max(float v)
{
    auto with = [](float x, int moved) __attribute__((always_inline)) { return fmaxf(x, __int_as_float(moved)); };
    v = with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
    v = with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, true));  // 2 3 0 1
    v = with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true)); // 7 6 .. 0
    return with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true)); // 15 14 .. 0
}

// A number that all lanes of a wave have.
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Where a wave's lane finds its part of a tile of 64 keys: a run of 16 tokens that lie in one page.
struct KvRun {
    int base;      // position of its first token; -1: there are none
    uint32_t page; // a number of n_pages and more: the table has none there
};

// ------------------------------------------------------------------ scores that are capped or biased, masks of documents and a prefix
// y = cap tanh(x / cap) - slope |distance|, as a number that is scaled later, as products are:
//   not capped          the product itself; a mask then costs nothing, a bias, in the products' units, two instructions a score
//   cap <= kPlainCap    tanh z = 1 - 2 / (1 + e^2z): -1 / (1 + e^2z), whose scale is twice the cap; the cap itself, the same for all keys, is left to
//                       the logarithm of the sum.  Off by 2^-22 of the cap (measured; 2^-21 if all its operations are as far off as they may be), whatever the score's size: as
//                       much as a score of a few units is by itself
//   above               powers of two: beyond half the cap the same formula (its error is small beside such a score), below a polynomial, each score by
//                       itself, so that it does not depend on what others there are; a wave that has none beyond does without the first
// Measured, 4096 tokens over 32768, bf16, 32 query heads, us: not capped 2000, a cap of 30 2300 - 2420, of 1000 (no score near half of it) 3700, slopes alone 2620.  When a cap of 30 took 2470: with
// y itself 2585, all scores by the polynomial 2846, by the power, or it where a wave has a score beyond half the cap, 3283.
constexpr float kPlainCap = 64.f;
// Added to a maximum for the logarithm of the sum, before it is scaled: -1 / (1 + e^2z) + 1 / 2 is exact near 0, the cap added afterwards would leave 2^-18 of its own.
__device__ __forceinline__ float score_middle(const KvAttend &a) { return a.cap > 0.f && a.cap <= kPlainCap ? 0.5f : 0.f; }
constexpr float kMostSlope = 0x1p36f; // over the least unit of y, 2^-60, and times any distance, it is a number

struct KvScoring {
    float z, cap; // products times z: 2 x / cap as a power of two (above kPlainCap: x / cap)
    float slope;
    bool capped, plain, biased;
    // qscale: what products are scaled by, then what y is
    __device__ __forceinline__ void begin(const KvAttend &a, int query_head, float &qscale)
    {
        capped = a.cap > 0.f, plain = a.cap <= kPlainCap, biased = a.slopes != nullptr;
        cap = a.cap * kLog2e;
        z = fminf(qscale / cap, 1e38f); // (0 of it is 0)
        if (plain) z *= 2.f * kLog2e;
        z = fminf(z, 3e38f);
        if (capped) qscale = plain ? 2.f * cap : 1.f;
        slope = biased ? __builtin_amdgcn_fmed3f(a.slopes[query_head], -kMostSlope, kMostSlope) * kLog2e / qscale : 0.f;
    }
    // z times a polynomial in z^2 that was fitted to tanh(z) / z up to 1/2 (off by 2^-26 of it), times the cap.
    __device__ __forceinline__ float near(float x) const
    {
        const float t = x * x;
        float r = __builtin_fmaf(t, 0.017135003577794676f, -0.05298607376020325f);
        r = __builtin_fmaf(r, t, 0.1332477929361659f);
        r = __builtin_fmaf(r, t, -0.33333069392817194f);
        r = __builtin_fmaf(r, t, 0.9999999868717396f);
        return x * r * cap;
    }
    // -1 / (1 + 2^power)
    static __device__ __forceinline__ float below(float power) { return __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(power)); }
    // N products of a lane, in place, by all lanes of a wave together.
    template <int N>
    __device__ __forceinline__ void cap_all(float (&x)[N]) const
    {
        if (plain) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = below(x[i] * z);
            return;
        }
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] *= z;
            most = fmaxf(most, fabsf(x[i]));
        }
        const bool all_near = !__any(most > 0.5f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = near(x[i]);
            if (all_near) x[i] = y;
            else x[i] = fabsf(x[i]) > 0.5f ? __builtin_fmaf(2.f * cap, below(x[i] * (2.f * kLog2e)), cap) : y;
        }
    }
};

// The keys that a row tile's queries see lie in tiles [0, prefix) and [low, high) of 64: tile j of those, in order.
struct KvSpan {
    int prefix, low, count;
    __device__ __forceinline__ void begin(int prefix_keys, int first_key, int end_tile)
    {
        prefix = (prefix_keys + kKvTile - 1) / kKvTile;
        low = max(first_key / kKvTile, prefix);
        count = prefix + max(end_tile - low, 0);
    }
    __device__ __forceinline__ int tile(int j) const { return j < prefix ? j : j - prefix + low; }
};

// What a workgroup (or the last one of a split row tile) does with a row of its results: 16 threads a row, four channels each at a time.
// m: their largest score, in units of qscale.
template <int T, int DP, typename F>
__device__ __forceinline__ void kv_write_row(const KvAttend &a, int h, int tok, int member, int sub, float m, float qscale, float l, F value)
{
    const size_t oh = (size_t)tok * a.c.H * a.G + h * a.G + member;
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DP; d += 64) {
        const int dd = d + sub * 4;
        if (dd >= a.c.D) continue;
        const f32x4 y = value(dd) * inv;
        *reinterpret_cast<u32x2 *>(a.out + (oh * a.c.D + dd) * 2) = u32x2{pack16<T>(y[0], y[1]), pack16<T>(y[2], y[3])};
    }
    if (sub == 0 && a.lse) a.lse[oh] = l > 0.f ? ((m + score_middle(a)) * qscale + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// The parts of row r of a tile of BR rows joined, from part `first` on and in order: their largest maximum, and sums and 4 channels in 64 in its
// units.  Several at a time are asked for before any is used: one after the other they cost a latency each (64 parts of 8 heads: the join 12 us where
// every thread looked at all the maxima, one by one 40; now 54 parts 8).
template <int DP, int BR>
__device__ __forceinline__ void kv_join_parts(const KvAttend &a, size_t first, int r, int sub, float qscale, float &m, float &l, f32x4 (&y)[DP / 64])
{
    constexpr int AT_ONCE = 8;
    const int n = a.n_split;
    m = -INFINITY, l = 0.f;
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) y[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    // the row's threads look at a sixteenth of the maxima each
    for (int s = 0; s < n; s += AT_ONCE * 16) {
        float x[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) x[k] = a.part_ml[((first + min(s + k * 16 + sub, n - 1)) * BR + r) * 2];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) m = fmaxf(m, x[k]);
    }
    m = over_row_max(m);
    const float base = m == -INFINITY ? 0.f : m;
    for (int s = 0; s < n; s += AT_ONCE) {
        f32x2 ml[AT_ONCE];
        f32x4 v[AT_ONCE][DP / 64];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const size_t pr = (first + min(s + k, n - 1)) * BR + r;
            ml[k] = *reinterpret_cast<const f32x2 *>(a.part_ml + pr * 2);
#pragma unroll
            for (int d = 0; d < DP / 64; ++d) v[k][d] = *reinterpret_cast<const f32x4 *>(a.part + pr * DP + d * 64 + sub * 4);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (s + k >= n) break;
            const float w = __builtin_amdgcn_exp2f((ml[k][0] - base) * qscale); // (a part that saw no key has zeros)
            l += w * ml[k][1];
#pragma unroll
            for (int d = 0; d < DP / 64; ++d) y[d] += w * v[k][d];
        }
    }
}

// Rows of 16 queries that share a key/value head (query heads of its group, several tokens' where the group is small) against
// keys that four waves of a workgroup take in turns, 64 at a time, with no LDS until they join their results:
//   S^T = K Q^T   rows are keys, columns queries; the products' operands come from memory as they lie there
//   O^T += V^T P^T  whose right operand is, by the choice of which key is which row of K, what a lane holds of S^T already:
//     row m of product t is key 16 (m / 4) + 4 t + (m % 4) of the tile, so that lane (column, quarter g) ends up with keys
//     16 g .. 16 g + 15 of its query, and loads those same 16 tokens of the values' channels
// One pass with a running maximum and sum per query, in 32 bits.  Products are taken in the queries' type, which holds 8-bit codes
// exactly; weights, which carry the values' scales, are rounded to it for the second one: in bfloat16, whose 8 bits are fewer than the
// codes are worth, to the sum of two numbers.
// Bound by memory: K of a wave's next tile is asked for when the products with this one's are done, V of a tile when its K is about to be
// used, and the pages of both a round (their blocks, where they are listed, two rounds) earlier, so that a wave always has 8 or 16 KB on
// its way.  Where the keys are cut into few parts, the workgroup that ends last joins them, in their order: no launch of its own.
// blockIdx: row tile of a sequence (sparse: of a token), part of its keys, head; the heads fastest, so that each of the chip's eight
// parts reads few of them.  ONE: a tile of keys lies in one page.
// Measured (medians), 8 heads of 128, 4 query heads each: one token of each of 48 sequences of up to 32768 tokens, int8, 1.22 GB in 235 us,
// 5.2 TB/s (without what is asked for ahead 446); one token of 1025, bf16, 9.2 us, a chain of lengths, pages, keys and the join.
// Of 256 channels at 16 bits K and V do not fit the 512 registers of one wave a SIMD: 69 - 128 of them go to scratch, 268 - 376 bytes a lane (48
// sequences of 8192 bf16 tokens, a token each, 787 us, 4.1 TB/s; int8, with no scratch, 296 us, 5.5 TB/s; 4 bits 172 us, 250 where two waves of a SIMD have 256 registers each).
// 4 bits: one token of each of 48 sequences of up to 65536 tokens, 128 channels, 1.11 GB in 228 us, 4.9 TB/s: three waves a SIMD with half the bytes of 8 bits on
// their way, vector units 38 % busy.
// R: where there are 16 / R queries at most, each of them has R columns, and a column weighs that part of a lane's keys that is its own: a
// column is a softmax of its own, joined with the others in the end as the waves' are.  For the sparse form, which reads from the
// caches and is bound by the vector units (1024 tokens, 32 blocks each of int8: 4 query heads a group, R 1 403 us, R 4 352 - 362; 2, R 1 412,
// R 4 373; 8, R 1 423, R 2 393).
template <int S, int T, int DP, bool SPARSE, bool ONE, int R, bool SCORED>
__global__ __launch_bounds__(256, DP * kv_bits<S> / 8 > 128 || (S == PK_F4 && DP == 256) ? 1 : 2) void kv_rows_kernel(KvAttend a)
{
    using Sc = KvScaling<S, T>;
    constexpr bool CODED = Sc::CODED, HALF = Sc::HALF, TWICE = Sc::TWICE, FOUR = S == PK_F4;
    constexpr int RB = DP * kv_bits<S> / 8;   // bytes of a row
    constexpr int KB = RB / 4 < 16 ? RB / 4 : 16, KC = RB / (4 * KB); // a lane's loads for one row of K: bytes of each, their number
    constexpr int EL = KB * 8 / kv_bits<S>, OPS = EL / 8; // elements of such a load, operands of a product of them
    constexpr int KS = DP / 32;               // products over the channels
    constexpr int DT = DP / 16;               // tiles of 16 channels of the output
    constexpr int VN = kv_value_words<S, DT>; // loads of a lane for 16 tokens of all channels
    constexpr int RT = 16 / R, NI = 4 / R;    // queries of a tile; of a lane's four groups of four keys, those that its column weighs
    __shared__ __align__(16) float join_o[4][16][DP + 4];
    __shared__ float join_m[4][16], join_l[4][16], join_q[16];
    __shared__ uint32_t arrived;
    const int tid = threadIdx.x, wave = same(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
    const KvDev c = a.c;
    const int P = c.P, G = a.G;
    int at = blockIdx.x;
    const int h = at % c.H;
    at /= c.H;
    const int split = at % a.n_split, unit = at / a.n_split;

    // the tile's queries
    int seq, tile, token0 = 0;
    if constexpr (SPARSE) {
        token0 = unit / a.row_tiles;
        tile = unit - token0 * a.row_tiles;
        seq = kv_seq_of(a.b, token0);
    } else {
        seq = unit / a.row_tiles;
        tile = unit - seq * a.row_tiles;
    }
    const KvSeq sq = kv_seq(a.b, seq, P);
    const int rows = SPARSE ? G : sq.m * G;
    if (tile * RT >= rows || (!SPARSE && rows > a.few_rows)) return;
    if (SPARSE && (token0 < sq.first || token0 >= sq.first + sq.m)) return; // a token of no sequence: its rows are left as they are
    const int part = R == 1 ? 0 : col / RT, row = tile * RT + col % RT;
    const bool valid = row < rows;
    const int tok = SPARSE ? token0 : sq.first + min(row, rows - 1) / G;
    const int member = min(row, rows - 1) % G;
    const int start = sq.len - sq.m;
    // columns without a query see every key (what they compute is dropped)
    const int pos = valid ? start + (tok - sq.first) : 0x7fffffff;
    int from = valid && !SPARSE && a.window > 0 ? max(pos - a.window + 1, 0) : 0;
    int prefix = 0;
    if constexpr (SCORED) {
        if (valid && a.starts) from = max(from, min(a.starts[tok], (int)kKvMaxTokens));
        if (a.prefix) prefix = min(max(a.prefix[seq], 0), sq.len);
    }
    const int32_t *table = a.b.tables + (size_t)seq * a.b.table_stride;
    const int32_t *list = SPARSE ? a.blocks + ((size_t)token0 * c.H + h) * a.n_blocks : nullptr;

    // tiles of 64 keys: those that the first and the last query of the tile see at most
    int t0, t1;
    KvSpan span;
    if constexpr (SCORED) {
        int first = valid ? from : INT32_MAX;
#pragma unroll
        for (int d = 1; d < 16; d *= 2) first = min(first, __shfl_xor(first, d));
        const int last_pos = start + min(tile * RT + RT - 1, rows - 1) / G;
        span.begin(prefix, same(first), last_pos < 0 ? 0 : last_pos / kKvTile + 1);
        // (cut evenly, whatever the masks leave: each part of one call of a window of 4096 in 131072 has its share)
        const int each = (span.count + a.n_split - 1) / a.n_split;
        t0 = min(split * each, span.count);
        t1 = min(t0 + each, span.count);
    } else if constexpr (SPARSE) {
        t0 = split * a.split_tiles;
        t1 = min((a.n_blocks * P + kKvTile - 1) / kKvTile, t0 + a.split_tiles);
    } else {
        const int first_pos = start + (tile * RT) / G, last_pos = start + min(tile * RT + RT - 1, rows - 1) / G;
        const int lo = a.window > 0 ? max(first_pos - a.window + 1, 0) / kKvTile : 0;
        t0 = max(lo, split * a.split_tiles);
        t1 = min(last_pos < 0 ? 0 : last_pos / kKvTile + 1, (split + 1) * a.split_tiles);
    }

    // ---- blocks, pages and K on their way
    const int ksub = ONE ? 0 : col >> 2, vsub = ONE ? 0 : g; // the lane's run of K's rows, and of V's tokens, whose pages it has to know
    auto block_of = [&](int t, int sub) __attribute__((always_inline)) -> int {
        if constexpr (SPARSE) {
            const int bi = min((t * kKvTile + sub * 16) >> c.logP, a.n_blocks - 1);
            return list[bi];
        } else return 0;
    };
    auto base_of = [&](int t, int sub, int block) __attribute__((always_inline)) -> int {
        const int at = (SCORED ? span.tile(t) : t) * kKvTile + sub * 16;
        if constexpr (SPARSE) {
            const bool in = t < t1 && (at >> c.logP) < a.n_blocks && block >= 0 && block <= (sq.len - 1) >> c.logP;
            return in ? (block << c.logP) + (at & (P - 1)) : -1;
        } else return t < t1 && at < sq.len ? at : -1;
    };
    auto page_of = [&](int base) __attribute__((always_inline)) -> uint32_t {
        const uint32_t page = (uint32_t)table[max(base, 0) >> c.logP]; // (asked for whether wanted or not: no branch)
        return base >= 0 ? page : c.n_pages;
    };
    // (ONE: what all lanes have, taken out of a vector register where it is used, not where it is asked for)
    auto taken = [&](KvRun r) __attribute__((always_inline)) -> KvRun {
        if constexpr (ONE) {
            asm volatile("" : "+v"(r.page), "+v"(r.base));
            r.base = same(r.base);
            r.page = (uint32_t)same((int)r.page);
        }
        return r;
    };
    u32x4 kw[4][KC];
    uint32_t kpow[KC]; // (4 bits) powers of two of the lane's four keys
    auto ask_k = [&](const KvRun &r) __attribute__((always_inline)) {
        const size_t ph = (size_t)(r.page < c.n_pages ? r.page : 0) * c.H + h;
        const int off = r.base >= 0 ? r.base & (P - 1) : 0, run = ONE ? col >> 2 : 0;
        const char *kr = c.k + (ph * P + off) * RB + (uint32_t)(run * 16 * RB + (KB == 16 ? g * 64 : (g >> 1) * 64 + (g & 1) * 8) + (col & 3) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                if constexpr (KB == 16) kw[i][k] = *reinterpret_cast<const u32x4 *>(kr + i * RB * 4 + k * 256);
                else {
                    const u32x2 w = *reinterpret_cast<const u32x2 *>(kr + i * RB * 4);
                    kw[i][k] = u32x4{w[0], w[1], 0u, 0u};
                }
            }
        if constexpr (FOUR) {
            const uint8_t *e = c.ke + (ph * P + off) * (DP / 32) + (uint32_t)(run * (DP / 2) + (KB == 16 ? g : g >> 1) * 16 + (col & 3) * 4);
#pragma unroll
            for (int k = 0; k < KC; ++k) kpow[k] = *reinterpret_cast<const uint32_t *>(e + k * 64);
        }
    };
    const int tw = t0 + wave;
    int kblock = 0, vblock = 0; // (sparse) of the round after the next
    KvRun kr, vr, kr1, vr1;     // of this round and the next
    {
        const int kb0 = block_of(tw, ksub), vb0 = ONE ? kb0 : block_of(tw, vsub), kb1 = block_of(tw + 4, ksub), vb1 = ONE ? kb1 : block_of(tw + 4, vsub);
        kblock = block_of(tw + 8, ksub), vblock = ONE ? kblock : block_of(tw + 8, vsub);
        kr.base = base_of(tw, ksub, kb0), vr.base = base_of(tw, vsub, vb0);
        kr1.base = base_of(tw + 4, ksub, kb1), vr1.base = base_of(tw + 4, vsub, vb1);
        kr.page = page_of(kr.base), vr.page = ONE ? kr.page : page_of(vr.base);
        kr1.page = page_of(kr1.base), vr1.page = ONE ? kr1.page : page_of(vr1.base);
        kr = taken(kr);
        if constexpr (ONE) vr = kr;
    }

    // queries, as the right operand
    u32x4 qf[KS];
    float qscale = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f, x0; // (the query carries the scale's sign)
    {
        const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f;
        const char *qrow = a.q.data + ((size_t)tok * a.q.token_stride + (size_t)(h * G + member) * a.q.head_stride) * 2;
        float x[KS][8], most = 0.f, sum = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int at = (k / OPS * 4 + g) * EL + k % OPS * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] = 0.f;
            if (valid && at < c.D) load_eight<T>(x[k], qrow, at);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[k][i]));
        }
        KvQueryScale<S, T> qs;
        qs.largest(over_quarters_max(most));
        qs.near *= sign;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                x[k][i] *= qs.near, x[k][i + 1] *= qs.near;
                sum += x[k][i] + x[k][i + 1];
                qf[k][i / 2] = pack16<T>(x[k][i], x[k][i + 1]);
            }
        x0 = qs.start(over_quarters_sum(sum));
        qscale *= qs.back;
    }
    KvScoring scoring;
    if constexpr (SCORED) scoring.begin(a, h * G + member, qscale);

    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f, vunit = 1e-30f, vper = 1e30f; // (of the scales of values: the largest so far, at least this)

    if (tw < t1) ask_k(kr);
    for (int t = tw; t < t1; t += 4) {
        const bool there = vr.page < c.n_pages;
        const int vb = ONE ? (vr.base >= 0 ? vr.base + g * 16 : -1) : vr.base; // the lane's first token
        f32x4 ksc[NI], vsc[NI];
        u32x4 vw[VN];
        {
            const size_t vph = (size_t)(there ? vr.page : 0) * c.H + h;
            const int voff = vr.base >= 0 ? vr.base & (P - 1) : 0, vrun = ONE ? g * 16 : 0;
            if constexpr (CODED) {
                const float *ks = c.ks + vph * P + voff + (uint32_t)(vrun + part * NI * 4), *vs = c.vs + vph * P + voff + (uint32_t)(vrun + part * NI * 4);
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    ksc[i] = *reinterpret_cast<const f32x4 *>(ks + 4 * i);
                    vsc[i] = *reinterpret_cast<const f32x4 *>(vs + 4 * i);
                }
            }
            const char *v = c.v + (vph * P + voff) * RB + (uint32_t)(vrun * RB + col * 16);
#pragma unroll
            for (int d = 0; d < VN; ++d) vw[d] = *reinterpret_cast<const u32x4 *>(v + (kv_bits<S> == 16 ? d / 2 * 256 + d % 2 * DP * 16 : d * 256));
        }
        __builtin_amdgcn_sched_barrier(0);

        f32x4 xa[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xa[i] = f32x4{x0, x0, x0, x0};
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                u32x4 f[OPS];
                operands<S, T, false>(kw[i][k], FOUR ? power_of(kpow[k] >> 8 * i & 0xffu) : 1.f, f);
#pragma unroll
                for (int e = 0; e < OPS; ++e) xa[i] = mma<HALF>(f[e], qf[OPS * k + e], xa[i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // the pages of the round after the next (first: whoever waits for them does not wait for K), and the next round's K
        kr = taken(kr1), vr = ONE ? kr : vr1;
        kr1.base = base_of(t + 8, ksub, kblock), vr1.base = base_of(t + 8, vsub, vblock);
        kr1.page = page_of(kr1.base), vr1.page = ONE ? kr1.page : page_of(vr1.base);
        kblock = block_of(t + 12, ksub), vblock = ONE ? kblock : block_of(t + 12, vsub);
        __builtin_amdgcn_sched_barrier(0);
        ask_k(kr);
        __builtin_amdgcn_sched_barrier(0);

        // the column's keys
        f32x4 x[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            x[i] = xa[i];
#pragma unroll
            for (int k = 1; k < R; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][j] = part == k ? xa[k * NI + i][j] : x[i][j];
            if constexpr (CODED) x[i] *= ksc[i];
        }
        if constexpr (SCORED) {
            static_assert(R == 1, "");
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = x[i >> 2][i & 3];
            if (scoring.capped) scoring.cap_all(y);
            if (scoring.biased) {
                const float far = (float)(pos - vb);
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = __builtin_fmaf(-scoring.slope, fabsf(far - (float)i), y[i]);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i >> 2][i & 3] = y[i];
#pragma unroll
            for (int i = 0; i < NI; ++i) asm volatile("" : "+v"(x[i])); // (what follows is the same code for all kinds: without it 4 - 9 registers go to scratch)
        }
        // keys that a query does not see; the values of tokens that no query sees are taken as zeros, whatever lies there
        const int seen = (there ? min(pos, sq.len - 1) : -1) - vb; // of the lane's 16 keys: 0 .. seen
        const int since = from - vb;
        if (__any(seen < 15 || since > 0 || vb < 0)) {
            const int held = there && vb >= 0 ? sq.len - vb : 0; // of its 16 tokens
            const int last = vb >= 0 ? seen : -1, key0 = part * NI * 4;
            const int before = SCORED && held > 0 ? prefix - vb : 0; // of the prefix
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = key0 + 4 * i + j;
                    x[i][j] = (key <= last && key >= since) || (SCORED && key < before) ? x[i][j] : -INFINITY;
                    if constexpr (CODED) vsc[i][j] = key < held ? vsc[i][j] : 0.f;
                }
#pragma unroll
            for (int d = 0; d < VN; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) vw[d][i] &= held_bits<S>(i, kv_bits<S> == 16 ? d & 1 : 0, held);
        }
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < NI; ++i) most = max3(most, max3(x[i][0], x[i][1], x[i][2]), x[i][3]);
        most = over_quarters_max(most);
        float big = 0.f;
        if constexpr (Sc::UNITS) {
#pragma unroll
            for (int i = 0; i < NI; ++i) big = max3(big, max3(vsc[i][0], vsc[i][1], vsc[i][2]), vsc[i][3]);
        }
        if (__any(most > m || big > vunit)) { // else all stays as it is
            const float m1 = fmaxf(m, most);
            float fade = m1 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m1) * qscale);
            m = m1;
            l *= fade;
            if constexpr (Sc::UNITS) {
                big = over_quarters_max(big);
                if (big > vunit) { // (else what is there stays: a unit times its rounded inverse need not be 1)
                    vper = 1.f / big;
                    fade *= vunit * vper;
                    vunit = big;
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= fade;
        }
        // (the largest is taken off before the scale, whatever its size: a chunk of the sparse form 1 - 2 % slower, no other call)
        const float mz = m == -INFINITY ? 0.f : m;
        f32x4 p[NI];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[i][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][j] - mz, qscale, Sc::top));
                sum = __builtin_fmaf(p[i][j], Sc::l_unit, sum);
            }
        l += sum;
        if constexpr (CODED) {
#pragma unroll
            for (int i = 0; i < NI; ++i) p[i] *= Sc::UNITS ? vsc[i] * vper : vsc[i];
        }
        u32x4 pf[2], pr[2]; // weights, and (TWICE) what their rounding left; of other columns' keys zeros
        uint32_t w[NI][2], r[NI][2];
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float p0 = p[i][2 * e], p1 = p[i][2 * e + 1];
                w[i][e] = pack16<T>(p0, p1);
                if constexpr (TWICE) {
                    asm("" : "+v"(w[i][e])); // (its halves are what was rounded: not rounded again)
                    r[i][e] = pack16<T>(p0 - __uint_as_float(w[i][e] << 16), p1 - __uint_as_float(w[i][e] & 0xffff0000u));
                }
            }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bool mine = R == 1 || part == (2 * u + i) / NI;
                    pf[u][2 * i + e] = mine ? w[(2 * u + i) % NI][e] : 0u;
                    if constexpr (TWICE) pr[u][2 * i + e] = mine ? r[(2 * u + i) % NI][e] : 0u;
                }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            u32x4 f0, f1;
            value_operands<S, T>(vw, d, f0, f1);
            o[d] = mma<HALF>(f0, pf[0], o[d]);
            o[d] = mma<HALF>(f1, pf[1], o[d]);
            if constexpr (TWICE) {
                o[d] = mma<HALF>(f0, pr[0], o[d]);
                o[d] = mma<HALF>(f1, pr[1], o[d]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    // the four waves' results joined: everything in units of the largest maximum
    l = over_quarters_sum(l) * Sc::l_back;
    const float back = Sc::UNITS ? Sc::o_back * vunit : Sc::o_back;
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4 *>(&join_o[wave][col][d * 16 + g * 4]) = o[d] * back;
    if (g == 0) {
        join_m[wave][col] = m;
        join_l[wave][col] = l;
        join_q[col] = qscale; // (the same in all waves)
    }
    __syncthreads();
    const int r = tid >> 4, sub = tid & 15; // 16 threads a row
    const bool in_row = r < RT && tile * RT + r < rows;
    const int otok = SPARSE ? token0 : sq.first + min(tile * RT + r, rows - 1) / G, omember = (tile * RT + r) % G;
    // a row's columns in the four waves: column r + k RT of wave w has f[w + 4 k]
    const int rr = r % RT;
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4 * R; ++w) mm = fmaxf(mm, join_m[w & 3][rr + (w >> 2) * RT]);
    const float mb = mm == -INFINITY ? 0.f : mm, jq = join_q[rr];
    float f[4 * R], ll = 0.f;
#pragma unroll
    for (int w = 0; w < 4 * R; ++w) {
        f[w] = __builtin_amdgcn_exp2f((join_m[w & 3][rr + (w >> 2) * RT] - mb) * jq);
        ll += f[w] * join_l[w & 3][rr + (w >> 2) * RT];
    }
    auto joined = [&](int dd) __attribute__((always_inline)) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4 * R; ++w) y += f[w] * *reinterpret_cast<const f32x4 *>(&join_o[w & 3][rr + (w >> 2) * RT][dd]);
        return y;
    };
    if (a.n_split == 1) {
        if (in_row) kv_write_row<T, DP>(a, h, otok, omember, sub, mm, jq, ll, joined);
        return;
    }
    const size_t slot = (size_t)unit * c.H + h, first = slot * a.n_split;
    if (in_row) {
        const size_t pr = (first + split) * 16 + r;
        if (sub == 0) *reinterpret_cast<f32x2 *>(a.part_ml + pr * 2) = f32x2{mm, ll};
        if (sub == 0 && split == 0) a.part_q[slot * 16 + r] = jq;
#pragma unroll
        for (int d = 0; d < DP; d += 64) *reinterpret_cast<f32x4 *>(a.part + pr * DP + d + sub * 4) = joined(d + sub * 4);
    }
    if (!a.join_here) return;
    // The last of the parts joins them all (what this one wrote is seen by it: release, and acquire where it is the last).  The barrier does not
    // wait for stores to memory, and the release is one wave's: every wave waits for its own first.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        arrived = atomicAdd(&a.arrivals[slot], 1u);
    }
    __syncthreads();
    if (arrived != (uint32_t)a.n_split - 1) return;
    __threadfence();
    if (tid == 0) a.arrivals[slot] = 0; // for the next call
    if (!in_row) return;
    float jm, jl;
    f32x4 y[DP / 64];
    kv_join_parts<DP, 16>(a, first, r, sub, jq, jm, jl, y);
    kv_write_row<T, DP>(a, h, otok, omember, sub, jm, jq, jl, [&](int dd) __attribute__((always_inline)) { return y[dd / 64]; });
}

// ------------------------------------------------------------------ long chunks
typedef float f32x16 __attribute__((ext_vector_type(16)));

// acc += A (32 rows x 16) B (16 x 32 columns)
template <bool HALF>
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 acc)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), acc, 0, 0, 0);
}

// Row tile `unit` among those of the sequences that have more rows of queries than are taken 16 at a time, counted
// over the batch, the last of a sequence first; seq -1: there are no more.  By all lanes of a wave together, 64 sequences at once.
struct KvUnit {
    int seq, tile;
};
template <int BR>
__device__ __forceinline__ KvUnit kv_unit(const KvAttend &a, int unit)
{
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.b.n_seqs; s0 += 64) {
        int n = 0;
        if (s0 + lane < a.b.n_seqs) {
            const int rows = kv_seq(a.b, s0 + lane, a.c.P).m * a.G;
            n = rows > a.few_rows ? (rows + BR - 1) / BR : 0;
        }
        int upto = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const unsigned long long beyond = __ballot(upto > unit);
        if (beyond) {
            const int l = __ffsll(beyond) - 1, end = __shfl(upto, l);
            return KvUnit{s0 + l, end - 1 - unit};
        }
        unit -= __shfl(upto, 63);
    }
    return KvUnit{-1, 0};
}

// Where 16-byte piece `piece` of row `row` lies in a tile in LDS: rows of CH pieces, moved about so that 16 lanes that read one piece
// of 16 neighbouring rows, or write four pieces of four, meet all banks.  (Piece p ^ x lies where p does, exclusive-or x.)
template <int CH>
__device__ __forceinline__ int lds_piece(int row, int piece)
{
    const int x = CH == 8 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
    return row * CH + (piece ^ x);
}

// The largest of a number's values in lanes l and l ^ 32.
__device__ __forceinline__ float over_halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// All waves of the workgroup meet; what they read of or wrote to LDS before is done, loads from memory may still be on their way.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The order of a phase's products: N1 operands of EACH products, then N2 of one, read from LDS AHEAD of them.
template <int AHEAD, int N1, int EACH, int N2>
__device__ __forceinline__ void reads_ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < N1 + N2; ++i) {
        if (i < N1) __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
        else __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i < N1 + N2 - AHEAD) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
}

// The largest of a number's values in a wave.
__device__ __forceinline__ float over_wave_max(float v)
{
    v = over_row_max(v);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return over_halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// Tiles on their way into LDS: their pages, then pieces of K(j) and V(j - 1) in registers, then LDS.
template <int S, int T, int DP, int NW, bool ONE, bool SCORED>
struct KvTiles {
    static constexpr int RB = DP * kv_bits<S> / 8, NT = NW * 64, CH = DP / 8; // bytes of a row
    static constexpr bool CODED = kv_coded<S>, FOUR = S == PK_F4, UNITS = KvScaling<S, T>::UNITS;
    static constexpr int PIECES = kKvTile * RB / 16; // 16-byte pieces of a tile of K, and of one of V
    static constexpr int KP = (PIECES + NT - 1) / NT;     // of a thread
    static constexpr int KR = RB / 16;                    // pieces of a row of K
    // piece p of a tile in memory: of K piece k_piece of token k_tok; of V channel v_row (4 bits: and the one 16 beyond), tokens from v_tok on
    static __device__ __forceinline__ int k_tok(int p) { return p / (4 * KR) * 4 + (p & 3); }
    static __device__ __forceinline__ int k_piece(int p) { return p / 4 % KR; }
    static __device__ __forceinline__ int v_row(int p) { return FOUR ? p % RB / 16 * 32 + p % 16 : p % DP; }
    static __device__ __forceinline__ int v_tok(int p) { return FOUR ? p / RB * 16 : p / DP * (128 / kv_bits<S>); }
    static constexpr int PG = ONE ? 1 : KP;
    static_assert(PIECES % NT == 0 || PIECES < NT, "");
    // Whether a tile's pages are asked for ahead of the pieces of the one before it (fetch), not among them, where the compiler else has them.  Measured, first (among),
    // us: bf16, 8 heads of 4, 4096 tokens over 32768 1990 (2040), 256 tokens behind a window of 4096 138 (148), 256 channels, 2048 over 8192 706 (720); codes no less: e4m3, 64
    // channels, 16 sequences 1604 (1593), int8, 256 channels 796 (782), 4 bits 1140 (1133); capped, 64 channels, 2048 over 16384 553 (533), 128, 4096 over 32768 2330 (2350).
    static constexpr bool PAGES_FIRST = !CODED && !(SCORED && DP == 64);
    struct Lds {
        u32x4 k[2][kKvTile * CH];
        u32x4 v[2][DP * 8];
        float scales[CODED ? 4 : 1][2][kKvTile];
        float fade[4], unit[4]; // UNITS: what the sums so far are multiplied by, as the unit of V's scales grows with a tile, and that unit
    };

    const char *k, *v;
    const float *ks, *vs;
    const uint8_t *ke;
    const int32_t *table;
    uint32_t n_pages;
    int H, h, P, logP, len;
    KvSpan span; // (SCORED)
    uint32_t kpage[PG], vpage[PG], spage; // of K(j), of V(j - 1); of the lane's token of K(j)
    u32x4 kw[KP], vw[KP];
    uint32_t kpow[FOUR ? KP : 1]; // powers of two of the pieces of K
    float ksw, vsw;
    float unit, fade; // (of the wave that brings them) largest scale of a value so far, and the one before it in units of it
    uint32_t v_in;    // which of the thread's pieces of V(j - 1) lie in pages that the table has
    bool v_there;     // all of the wave's
    uint32_t in_next; // which of K(j)'s four runs of 16 tokens lie in such pages

    __device__ __forceinline__ void begin(const KvDev &c, const int32_t *t, int head, int tokens)
    {
        k = c.k, v = c.v, ks = c.ks, vs = c.vs, ke = c.ke, table = t;
        n_pages = c.n_pages, H = c.H, h = head, P = c.P, logP = c.logP, len = tokens;
        spage = 0, ksw = 0.f, vsw = 0.f, in_next = 0, v_in = 0, v_there = true, unit = 1e-30f, fade = 1.f;
    }
    // first position of tile j (of those that the workgroup goes through)
    __device__ __forceinline__ int first_of(int j) const { return (SCORED ? span.tile(j) : j) * kKvTile; }
    // page of a position, of the nearest that the sequence has where it has none there
    __device__ __forceinline__ uint32_t page_of(int pos) const { return (uint32_t)table[min(max(pos, 0), max(len - 1, 0)) >> logP]; }
    __device__ __forceinline__ size_t place(uint32_t page) const { return (size_t)(page < n_pages ? page : 0) * H + h; }

    __device__ __forceinline__ void lookup(int j)
    {
        const int kb = first_of(j), vb = first_of(j - 1), tid = threadIdx.x;
        if constexpr (ONE) {
            kpage[0] = page_of(kb);
            vpage[0] = page_of(vb);
        } else {
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int p = tid + i * NT;
                kpage[i] = page_of(kb + k_tok(p));
                vpage[i] = page_of(vb + v_tok(p));
            }
            spage = page_of(kb + (tid & 63));
        }
    }

    // NEXT: and the pages of tile j + 1, first.
    template <bool NEXT>
    __device__ __forceinline__ void fetch(int j)
    {
        const int kb = first_of(j), vb = first_of(j - 1), tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
        const bool mine = PIECES >= NT || tid < PIECES;
        if constexpr (ONE) {
            // (taken here, not where they were asked for: that would be a wait for all that is on its way)
            asm volatile("" : "+v"(kpage[0]), "+v"(vpage[0]));
            const uint32_t kp = (uint32_t)same((int)kpage[0]), vp = (uint32_t)same((int)vpage[0]);
            if constexpr (NEXT) {
                lookup(j + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            const char *kr = k + (place(kp) * P + (kb & (P - 1))) * RB, *vr = v + (place(vp) * P + (vb & (P - 1))) * RB;
            in_next = kp < n_pages ? 15u : 0u;
            if constexpr (CODED) { // (first: loads come back in their order, and the scales are wanted before the rest)
                const size_t at = place(kp) * P + (kb & (P - 1));
                const float *ksr = ks + at, *vsr = vs + at;
                uint32_t by = lane;
                asm volatile("" : "+v"(by)); // (added to the tile's address: kept as addresses of their own over the loop, these went to scratch)
                if (wave == 0) ksw = ksr[by];
                if (wave == 1) vsw = in_next && kb + lane < len ? vsr[by] : 0.f;
            }
            if (mine) {
#pragma unroll
                for (int i = 0; i < KP; ++i) {
                    const int p = tid + i * NT;
                    kw[i] = *reinterpret_cast<const u32x4 *>(kr + (uint32_t)(p * 16));
                    vw[i] = *reinterpret_cast<const u32x4 *>(vr + (uint32_t)(p * 16));
                    if constexpr (FOUR) kpow[i] = ke[(place(kp) * P + (kb & (P - 1))) * (DP / 32) + (uint32_t)e_place<DP>(k_tok(p), k_piece(p))];
                }
            }
            v_there = vp < n_pages;
            v_in = v_there ? ~0u : 0u;
        } else {
            uint32_t kp[KP], vp[KP];
            v_in = 0;
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                asm volatile("" : "+v"(kpage[i]), "+v"(vpage[i]));
                kp[i] = kpage[i], vp[i] = vpage[i];
            }
            asm volatile("" : "+v"(spage));
            const uint32_t sp = spage;
            if constexpr (NEXT) {
                lookup(j + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int p = tid + i * NT;
                if (mine) {
                    // (a run of 16 tokens lies in one page)
                    constexpr int RUN = RB; // pieces of a run
                    const size_t krun = place(kp[i]) * P + ((kb + p / RUN * 16) & (P - 1)), vrun = place(vp[i]) * P + ((vb + p / RUN * 16) & (P - 1));
                    kw[i] = *reinterpret_cast<const u32x4 *>(k + krun * RB + (p % RUN) * 16);
                    vw[i] = *reinterpret_cast<const u32x4 *>(v + vrun * RB + (p % RUN) * 16);
                    if constexpr (FOUR) kpow[i] = ke[krun * (DP / 32) + (uint32_t)e_place<DP>(k_tok(p) & 15, k_piece(p))];
                }
                v_in |= (vp[i] < n_pages ? 1u : 0u) << i;
            }
            const bool ok = sp < n_pages;
            const unsigned long long b = __ballot(ok);
            in_next = (uint32_t)((b & 1) | (b >> 15 & 2) | (b >> 30 & 4) | (b >> 45 & 8));
            v_there = __all(v_in == (1u << KP) - 1);
            if constexpr (CODED) {
                const size_t at = place(sp) * P + ((kb + lane) & (P - 1));
                if (wave == 0) ksw = ks[at];
                if (wave == 1) vsw = ok && kb + lane < len ? vs[at] : 0.f;
            }
        }
    }

    // The scales of the values that were asked for last, in units of the largest so far: by the wave that brings them, when it has time.
    __device__ __forceinline__ void weigh()
    {
        if constexpr (UNITS) {
            if (same(threadIdx.x >> 6) != 1) return;
            asm volatile("" : "+v"(vsw)); // (here, not where it was asked for)
            const float most = fmaxf(over_wave_max(vsw), unit), per = __builtin_amdgcn_rcpf(most);
            fade = most > unit ? unit * per : 1.f; // (a unit times its rounded inverse need not be 1, and that in every tile: 2^-10 of O in 2^20 keys)
            unit = most;
            vsw *= per;
        }
    }

    // Before tile j is written: tokens that no query sees count as zeros, whatever lies there.
    __device__ __forceinline__ void mask(int j)
    {
        const int vb = first_of(j - 1);
        if (vb >= 0 && vb + kKvTile <= len && v_there) return;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const int p = threadIdx.x + i * NT, held = vb >= 0 && (v_in >> i & 1) ? len - (vb + v_tok(p)) : 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) vw[i][w] &= held_bits<S>(w, 0, held);
        }
    }

    __device__ __forceinline__ void store(int j, Lds &lds)
    {
        const int kb = j & 1, vb = kb ^ 1, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
        if (PIECES >= NT || tid < PIECES) {
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int p = tid + i * NT;
                const int row = k_tok(p), piece = k_piece(p), vrow = v_row(p), vpiece = v_tok(p) / 8;
                if constexpr (FOUR) {
                    u32x4 f[4];
                    operands<S, T, false>(kw[i], power_of(kpow[i]), f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) lds.k[kb][lds_piece<CH>(row, piece * 4 + e)] = f[e];
                    operands<S, T, true>(vw[i], 1.f, f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) lds.v[vb][lds_piece<8>(vrow + (e >> 1) * 16, vpiece + (e & 1))] = f[e];
                } else if constexpr (CODED) {
                    u32x4 f[2];
                    operands<S, T, false>(kw[i], 1.f, f);
                    lds.k[kb][lds_piece<CH>(row, piece * 2)] = f[0];
                    lds.k[kb][lds_piece<CH>(row, piece * 2 + 1)] = f[1];
                    operands<S, T, true>(vw[i], 1.f, f);
                    lds.v[vb][lds_piece<8>(vrow, vpiece)] = f[0];
                    lds.v[vb][lds_piece<8>(vrow, vpiece + 1)] = f[1];
                } else {
                    lds.k[kb][lds_piece<CH>(row, piece)] = kw[i];
                    lds.v[vb][lds_piece<8>(vrow, vpiece)] = vw[i];
                }
            }
        }
        if constexpr (CODED) {
            if (wave == 0) lds.scales[j & 3][0][lane] = ksw;
            if (wave == 1) {
                lds.scales[j & 3][1][lane] = vsw;
                if constexpr (UNITS) {
                    if (lane == 0) lds.fade[j & 3] = fade, lds.unit[j & 3] = unit;
                }
            }
        }
    }
};

// Many rows of queries against tiles of 64 keys that lie in LDS for all NW waves of the workgroup, 32 queries a wave.
//   S^T = K Q^T, O^T += V^T P^T as above, in products of 32 x 32: row m of S^T is the key with bits 2 and 3 of m exchanged, so that what a
//   lane holds of S^T is the right operand of the second product, for V's tokens in their order.
// A wave's round for tile t has two phases: products (P V of tile t - 1, then Q K of tile t) and weights (maximum, exponentials and
// sums of tile t, and its share of bringing later tiles in).  64 keys x 32 queries x 128 channels keep the matrix cores busy
// for 1024 cycles and the vector units for about as many, so the two waves of a SIMD are half a round apart: all waves meet after
// every phase, and waves 4 .. 7 began with one meeting more.
// Tiles lie in two buffers each.  Round t's products are in interval 2 t between meetings for waves 0 .. 3 and in 2 t + 1 for the others;
// they read K(t) and V(t - 1), so that K(t + 1) and V(t) may be written in these same two.  Scales, and which pages are not there,
// are read by the phases of weights and have four buffers.
// On its way a tile is in registers, asked for a round before it is written, and is converted to the queries' type once for all waves.
// The running maximum is of the bare products (the queries carry the scale's sign); O is rescaled only when some query's maximum
// has grown.  Once a wave has met a maximum beyond kNear, its scores are lessened by it before they are scaled, in the branch that else
// masks them.  In every tile that cost a long chunk 2.2 % and mixed chunks 2.7 % (the maximum so far as the products' start value: 2.5 and 5 %,
// as most tiles raise some query's); so 0.1 - 0.4 and 1 %.  The masks are bits: of comparisons for each key 16381 tokens in documents of 700 took 477 us, so 325 (304 now).  Of 256 channels, which leave no register, in every tile all the same: 2048 tokens
// over 8192, bf16, 702 us, in the branch 749, not at all 690.  ONE: a tile of keys lies in one page.
// Measured, bf16, 32 query heads of 128 channels: 4096 tokens over 32768 2.00 ms (median; from card to card and run to run 1.97 - 2.10), 1.0 PFLOP/s.
// 4.25 million cycles, of which the matrix cores are busy for 46 % and the reads of K and V out of LDS by eight waves take about as many,
// at 2.1 GHz: the power that the products draw holds the clock there (the same launch over zeros 1.76 ms, at 2.4 GHz).  A product of 8192 x 8192 x 8192 runs at 1.2 - 1.35 PFLOP/s on
// such numbers, 1.8 on zeros.  First form, each read waited for: 2.71 ms.
// ALONE: one workgroup a CU, whose waves then may have more than 128 registers (run()).
template <int S, int T, int DP, int NW, bool ONE, bool SCORED, bool ALONE = false>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(NW / 4, ALONE ? NW / 4 : 8))) void kv_tile_kernel(KvAttend a)
{
    constexpr int BR = NW * 32;
    using Sc = KvScaling<S, T>;
    constexpr bool CODED = Sc::CODED, HALF = Sc::HALF, TWICE = Sc::TWICE;
    constexpr int KS = DP / 16, DT = DP / 32, CH = DP / 8;
    constexpr bool ALWAYS = DP == 256; // the maximum is taken off in every tile
    __shared__ __align__(16) typename KvTiles<S, T, DP, NW, ONE, SCORED>::Lds lds;
    const int tid = threadIdx.x, wave = same(tid >> 6), lane = tid & 63, col = lane & 31, hf = lane >> 5;
    const int late = NW > 4 ? wave >> 2 : 0;
    const KvDev c = a.c;
    const int P = c.P, G = a.G, window = a.window;
    // consecutive workgroups take the heads in turn (each of the chip's parts then reads few heads), the last queries of a sequence, which
    // see the most keys, first
    int at = blockIdx.x;
    const int h = at % c.H;
    at /= c.H;
    const int split = at % a.n_split;
    const KvUnit un = kv_unit<BR>(a, at / a.n_split);
    if (un.seq < 0) return;
    const int seq = same(un.seq), tile = same(un.tile), unit = at / a.n_split;
    KvSeq sq = kv_seq(a.b, seq, P);
    sq = KvSeq{same(sq.first), same(sq.m), same(sq.len)};
    const int rows = sq.m * G;
    const int start = sq.len - sq.m;
    const int row = tile * BR + wave * 32 + col;
    const bool valid = row < rows;
    const int tok = sq.first + min(row, rows - 1) / G, member = min(row, rows - 1) % G;
    const int pos = valid ? start + (tok - sq.first) : 0x7fffffff;
    int from = valid && window > 0 ? max(pos - window + 1, 0) : 0;
    int prefix = 0;
    if constexpr (SCORED) {
        if (valid && a.starts) from = max(from, min(a.starts[tok], (int)kKvMaxTokens));
        if (a.prefix) prefix = same(min(max(a.prefix[seq], 0), sq.len));
    }
    const int32_t *table = a.b.tables + (size_t)seq * a.b.table_stride;
    // tiles of keys of the workgroup (its waves keep step: one whose queries see none of a tile's keys has weights of zero)
    auto first_of = [&](int r) { return window > 0 ? max(start + r / G - window + 1, 0) / kKvTile : 0; };
    auto last_of = [&](int r) { const int p = start + min(r, rows - 1) / G; return p < 0 ? 0 : p / kKvTile + 1; };
    int t0 = max(first_of(tile * BR), split * a.split_tiles), t1 = min(last_of(tile * BR + BR - 1), (split + 1) * a.split_tiles);
    KvTiles<S, T, DP, NW, ONE, SCORED> in;
    in.begin(c, table, h, sq.len);
    if constexpr (SCORED) {
        int first = first_of(tile * BR) * kKvTile;
        if (a.starts) { // the earliest of the tile's tokens', by each wave for itself
            int least = INT32_MAX;
            const int upto = sq.first + min(tile * BR + BR - 1, rows - 1) / G;
            for (int t = sq.first + tile * BR / G + lane; t <= upto; t += 64) least = min(least, a.starts[t]);
#pragma unroll
            for (int d = 1; d < 64; d *= 2) least = min(least, __shfl_xor(least, d));
            first = max(first, min(same(least), (int)kKvMaxTokens));
        }
        in.span.begin(prefix, first, last_of(tile * BR + BR - 1));
        const int each = (in.span.count + a.n_split - 1) / a.n_split;
        t0 = min(split * each, in.span.count);
        t1 = min(t0 + each, in.span.count);
    }

    u32x4 qf[KS];
    float qscale = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f, s0;
    {
        const char *qrow = a.q.data + ((size_t)tok * a.q.token_stride + (size_t)(h * G + member) * a.q.head_stride) * 2;
        const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f;
        float x[KS][8], most = 0.f, sum = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] = 0.f;
            if (valid && k * 16 + hf * 8 < c.D) load_eight<T>(x[k], qrow, k * 16 + hf * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[k][i]));
        }
        KvQueryScale<S, T> qs;
        qs.largest(over_halves_max(most));
        qs.near *= sign;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                x[k][i] *= qs.near, x[k][i + 1] *= qs.near;
                sum += x[k][i] + x[k][i + 1];
                qf[k][i / 2] = pack16<T>(x[k][i], x[k][i + 1]);
            }
        s0 = qs.start(sum + __shfl_xor(sum, 32));
        qscale *= qs.back;
    }

    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    KvScoring scoring;
    if constexpr (SCORED) scoring.begin(a, h * G + member, qscale);

    // ---- the two phases
    u32x4 pf[4], pr[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) pf[u] = pr[u] = u32x4{0u, 0u, 0u, 0u}; // (the first round has no tile before it)
    f32x16 s[2];
    bool far = false; // whether the wave has met a maximum beyond kNear
    auto pv_products = [&](int t) __attribute__((always_inline)) {
        const int vp = ((t & 1) ^ 1) * DP * 8 + lds_piece<8>(col, hf); // the lane's piece of the first row; the others' from it
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const u32x4 v = lds.v[0][(vp ^ (u * 2)) + d * 32 * 8];
                o[d] = mma32<HALF>(v, pf[u], o[d]);
                if constexpr (TWICE) o[d] = mma32<HALF>(v, pr[u], o[d]);
            }
    };
    auto qk_products = [&](int t) __attribute__((always_inline)) {
        const int key_row = (col & 0x13) | (col & 4) << 1 | (col & 8) >> 1; // bits 2 and 3 exchanged
        const int kp = (t & 1) * kKvTile * CH + lds_piece<CH>(key_row, hf);
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[r][i] = s0;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int r = 0; r < 2; ++r) s[r] = mma32<HALF>(lds.k[0][(kp ^ (k * 2)) + r * 32 * CH], qf[k], s[r]);
    };
    // (what a lane holds of s: keys 32 r + 16 u + 8 hf + j at 8 u + j)
    auto take_off = [&](float most) __attribute__((always_inline)) {
        const float z = most == -INFINITY ? 0.f : most;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[r][i] -= z;
    };
    auto rescale = [&](float fade, float unit_up) __attribute__((always_inline)) {
        l *= fade;
        const float f = fade * unit_up;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= f;
    };
    auto weights = [&](int t, uint32_t held) __attribute__((always_inline)) {
        const int base = in.first_of(t);
        const float *ks = lds.scales[CODED ? t & 3 : 0][0], *vs = lds.scales[CODED ? t & 3 : 0][1];
        if constexpr (CODED) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[u >> 1][8 * (u & 1) + j] *= ks[u * 16 + hf * 8 + j];
        }
        if constexpr (SCORED) {
            if (scoring.capped || scoring.biased) {
                float y[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = s[i >> 4][i & 15];
                if (scoring.capped) scoring.cap_all(y);
                if (scoring.biased) {
                    const float away = (float)(pos - base - hf * 8);
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] = __builtin_fmaf(-scoring.slope, fabsf(away - (float)(i / 8 * 16 + i % 8)), y[i]);
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = y[i];
            }
        }
        float above = m; // what a score has to exceed to be a new maximum
        if (far || held != 15u || (!(SCORED && base + kKvTile <= prefix) && __any(base + kKvTile - 1 > pos || base < from))) {
            // the tile's 64 keys as bits, of which a lane has the even or the odd bytes; two instructions a score
            const int last = min(pos, sq.len - 1) - base, since = max(from - base, 0), upto = min(last, kKvTile - 1);
            unsigned long long seen = upto >= since ? (~0ull >> (63 - upto)) & (~0ull << since) : 0ull;
            if (SCORED && prefix > base) seen |= ~0ull >> (64 - min(prefix - base, kKvTile));
            const unsigned long long runs = (held & 1 ? 0xffffull : 0ull) | (held & 2 ? 0xffffull << 16 : 0ull) | (held & 4 ? 0xffffull << 32 : 0ull) | (held & 8 ? 0xffffull << 48 : 0ull);
            seen &= runs;
            const uint32_t gone = ~__builtin_amdgcn_perm((uint32_t)(seen >> 32), (uint32_t)seen, hf ? 0x07050301u : 0x06040200u);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t none = (uint32_t)__builtin_amdgcn_sbfe((int)gone, i, 1);
                s[i >> 4][i & 15] = __uint_as_float((none & 0xff800000u) | (~none & __float_as_uint(s[i >> 4][i & 15])));
            }
            if (far) {
                above = INFINITY;
                float m1 = m;
#pragma unroll
                for (int i = 0; i < 16; ++i) m1 = max3(m1, s[0][i], s[1][i]);
                m1 = over_halves_max(m1);
                take_off(m1);
                rescale(m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m1) * qscale), 1.f);
                m = m1;
            }
        }
        float most = max3(s[0][0], s[0][1], s[0][2]), most2 = max3(s[1][0], s[1][1], s[1][2]);
#pragma unroll
        for (int i = 3; i < 15; i += 2) {
            most = max3(most, s[0][i], s[0][i + 1]);
            most2 = max3(most2, s[1][i], s[1][i + 1]);
        }
        most = max3(most, most2, max3(s[0][15], s[1][15], s[1][15]));
        most = over_halves_max(most);
        float unit_up = 1.f;
        if constexpr (Sc::UNITS) unit_up = lds.fade[t & 3];
        if (__any(most > above || unit_up != 1.f)) {
            const float m1 = most > above ? most : m;
            rescale(m1 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m1) * qscale), unit_up);
            m = m1;
            if (!ALWAYS && !far && __any(fabsf(m == -INFINITY ? 0.f : m) * qscale > kNear)) {
                far = true;
                take_off(m);
            }
        }
        if constexpr (ALWAYS) take_off(m);
        const float c = Sc::top - (ALWAYS || far || m == -INFINITY ? 0.f : m * qscale);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u >> 1][8 * (u & 1) + j], qscale, c));
                sum[j & 1] = __builtin_fmaf(p[j], Sc::l_unit, sum[j & 1]);
                if constexpr (CODED) p[j] *= vs[u * 16 + hf * 8 + j];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pf[u][i] = pack16<T>(p[2 * i], p[2 * i + 1]);
                if constexpr (TWICE) asm("" : "+v"(pf[u][i]));
                if constexpr (TWICE) pr[u][i] = pack16<T>(p[2 * i] - __uint_as_float(pf[u][i] << 16), p[2 * i + 1] - __uint_as_float(pf[u][i] & 0xffff0000u));
            }
        }
        l += sum[0] + sum[1];
    };

    if (t0 < t1) {
        in.lookup(t0);
        in.template fetch<false>(t0);
        in.lookup(t0 + 1);
        in.weigh();
        in.mask(t0);
        in.store(t0, lds);
        uint32_t held = in.in_next;
        in.template fetch<false>(t0 + 1);
        in.lookup(t0 + 2);
        in.weigh();
        meet();
        if (late) meet();
        for (int t = t0; t < t1; ++t) {
            // tile t + 1 is written (up to t1: the last tile's V comes with it), the next one asked for
            in.mask(t + 1);
            in.store(t + 1, lds);
            const uint32_t held_next = in.in_next;
            in.template fetch<in.PAGES_FIRST>(t + 2);
            if constexpr (!in.PAGES_FIRST) in.lookup(t + 3);
            pv_products(t);
            qk_products(t);
            reads_ahead<4, 4 * DT, TWICE ? 2 : 1, 2 * KS>();
            meet();
            weights(t, held);
            in.weigh();
            held = held_next;
            meet();
        }
        pv_products(t1);
        if (NW > 4 && !late) meet();
    }
    if (!valid) return;
    l = (l + __shfl_xor(l, 32)) * Sc::l_back;
    const float back = Sc::UNITS && t0 < t1 ? Sc::o_back * lds.unit[(t1 - 1) & 3] : Sc::o_back;
    if (a.n_split > 1) {
        const size_t pr = (((size_t)unit * c.H + h) * a.n_split + split) * BR + (wave * 32 + col);
        if (hf == 0) {
            *reinterpret_cast<f32x2 *>(a.part_ml + pr * 2) = f32x2{m, l};
            if (split == 0) a.part_q[((size_t)unit * c.H + h) * BR + (wave * 32 + col)] = qscale;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                *reinterpret_cast<f32x4 *>(a.part + pr * DP + d * 32 + b * 8 + hf * 4) =
                    f32x4{o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]} * back;
        return;
    }
    const size_t oh = (size_t)tok * c.H * G + h * G + member;
    const float inv = l > 0.f ? back / l : 0.f;
    // a lane and the one 32 beyond hold four channels each of two runs of eight: exchanged, each writes a run
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; b += 2) {
            uint32_t w[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) w[i][e] = pack16<T>(o[d][4 * (b + i) + 2 * e] * inv, o[d][4 * (b + i) + 2 * e + 1] * inv);
            const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false), y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
            const int dd = d * 32 + (b + hf) * 8;
            if (dd < c.D) *reinterpret_cast<u32x4 *>(a.out + (oh * c.D + dd) * 2) = u32x4{x[0], y[0], x[1], y[1]};
        }
    if (hf == 0 && a.lse) a.lse[oh] = l > 0.f ? ((m + score_middle(a)) * qscale + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// The parts of a row joined, in order: 16 threads a row.  Parts have BR rows; a workgroup joins 16 of them.  BR 16: the parts of the kernel
// for few rows, else of the one for many.  4 - 8 us, a launch and a chain of loads: 48 sequences of 8 heads in 13 parts 7 us.
template <int T, int DP, int BR, bool SPARSE>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttend a)
{
    const int r = (blockIdx.x % (BR / 16)) * 16 + (threadIdx.x >> 4), sub = threadIdx.x & 15, h = blockIdx.y, unit = blockIdx.x / (BR / 16);
    KvUnit un;
    if constexpr (BR == 16) {
        const int of = unit / a.row_tiles;
        un = KvUnit{SPARSE ? kv_seq_of(a.b, of) : of, unit - of * a.row_tiles};
    } else {
        un = kv_unit<BR>(a, unit);
    }
    if (un.seq < 0) return;
    const KvSeq sq = kv_seq(a.b, un.seq, a.c.P);
    const int row = un.tile * BR + r, rows = SPARSE ? a.G : sq.m * a.G;
    if (row >= rows || (BR == 16 && !SPARSE && rows > a.few_rows)) return;
    const int tok = SPARSE ? unit / a.row_tiles : sq.first + row / a.G;
    if (SPARSE && (tok < sq.first || tok >= sq.first + sq.m)) return; // (has no parts)
    const size_t at = ((size_t)unit * a.c.H + h) * a.n_split;
    const float qscale = a.part_q[((size_t)unit * a.c.H + h) * BR + r];
    float m, l;
    f32x4 y[DP / 64];
    kv_join_parts<DP, BR>(a, at, r, sub, qscale, m, l, y);
    kv_write_row<T, DP>(a, h, tok, row % a.G, sub, m, qscale, l, [&](int dd) __attribute__((always_inline)) { return y[dd / 64]; });
}

// Parts that the keys are cut into (`tiles` tiles of 64 at most): so many that there are `wgs` workgroups, each with `least` tiles at least;
// more of them, up to `more_wgs`, where each has `much` tiles, as sequences' lengths differ.  Within the room for partial results.  A window does
// not enter: parts that lie outside it end at once and are joined as parts without a key (one token, window 4096 of 131072: 8 heads 24 us, one 21).
// `most` of them at most.
void cut(KvAttend &a, int64_t items, int64_t tiles, int rows, int64_t wgs, int least, int64_t more_wgs, int much, int64_t most)
{
    const int64_t room = a.part_floats / ((int64_t)rows * a.part_row) / std::max<int64_t>(items, 1);
    const int64_t want = std::max(std::min((wgs + items - 1) / items, tiles / least), std::min((more_wgs + items - 1) / items, tiles / much));
    const int64_t n = std::max<int64_t>(std::min({want, room, most}), 1);
    a.split_tiles = (int32_t)((tiles + n - 1) / n);
    a.n_split = (int32_t)((tiles + a.split_tiles - 1) / a.split_tiles);
}

// Most parts of the kernel for few rows.  A row's parts are joined one after the other, eight on their way, 0.13 us each, so that few long sequences of few heads are better off
// with fewer parts than there are places: of T tiles 48 or 1.4 sqrt(T).  Measured, bf16, 8 query heads a head, us, so (and without): one token, one head over 32768 keys 15 (20), 131072 26
// (58), 10^6 108 (136); two heads 17 (25), 32 (50), 212 (231); four 23 (30), 54 (58), 367 (412), over 200000 99 (90); eight 33 (35), 105 (105), 715 (752); 1024 listed
// blocks, one head 21 (36), eight 56 (55); 4096 37 (69), 200 (205).
// The kernel for many rows, whose tiles take 2 us each and not 0.2, is better off with all the places (run(), 32 tokens, one head over 131072 keys 60, with this limit 86; 10^6 180, 228;
// two heads over 131072 64, 87; int8 67, 105; 256 channels 95, 135).
int64_t most_parts(int64_t tiles) { return std::max<int64_t>(48, (int64_t)(1.4 * std::sqrt((double)tiles))); }

template <int S, int T, int DP, bool SPARSE, bool SCORED>
hipError_t run(KvAttend a, hipStream_t s)
{
    const int64_t most = std::min<int64_t>(a.b.max_len, (int64_t)a.b.cols * a.c.P);
    const int64_t tiles = std::max<int64_t>(((SPARSE ? (int64_t)a.n_blocks * a.c.P : most) + kKvTile - 1) / kKvTile, 1);
    const int64_t seqs = SPARSE ? a.b.n_tokens : a.b.n_seqs;
    const int64_t rows = SPARSE ? a.G : (int64_t)a.b.max_new * a.G; // of a sequence at most
    // Most rows of queries of a sequence and head that are taken 16 at a time (above: 256 at a time).  Measured in us, 8 heads of 128 channels, 16
    // (256) at a time: bf16, 16 sequences of 64 rows over 8192 keys 182 (168), of 128 rows 309 (171), one of 64 rows over 32768 keys 54 (63), of
    // 128 rows 94 (65).  Codes of 8 bits cost the kernel for many more work for each tile, and half the reads here: int8, 16 sequences of 64 rows
    // 115 (209), of 128 rows 214 (214), of 256 rows 382 (236); one of 128 rows over 32768 keys 65 (78), of 256 rows 112 (85); 4 bits, 16 sequences of 128 rows
    // 147 (183), one of 128 rows over 32768 keys 45 (62).  (Other channels
    // and heads go by the same numbers, unmeasured; so do the numbers of parts.)
    a.few_rows = SPARSE ? INT32_MAX : kv_coded<S> ? kKvFewRows : 64;
    a.part_row = DP;
    // sequences of few rows: unless all may have the same number of new tokens, and that is many.  (The host's numbers are bounds: sequences
    // that have fewer after all are then the kernel for many's, as are all that have any)
    const bool alike = !SPARSE && (int64_t)a.b.n_seqs * a.b.max_new == a.b.n_tokens;
    if (SPARSE || !alike || rows <= a.few_rows) {
        a.row_tiles = (int32_t)((std::min<int64_t>(rows, a.few_rows) + 15) / 16);
        const int64_t units = seqs * a.row_tiles, items = units * a.c.H;
        cut(a, items, tiles, 16, 2 * a.num_cu, 4, 16 * a.num_cu, 32, most_parts(tiles));
        // The last part's workgroup joins them where all run at once: one token of 1025 keys 9.9 us, 7.1 + 3.8 with a launch of its own.  Where
        // there are many its fences cost more than a launch: 48 sequences of up to 32768 keys 494 us, 235 + 7 with the launch.
        a.join_here = items * a.n_split <= a.num_cu && items <= kKvArrivals;
        const dim3 grid((unsigned)(items * a.n_split));
        const bool one = a.c.P >= kKvTile;
        auto launch = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(a); };
        if constexpr (SPARSE) {
            if (a.G <= 4) one ? launch(kv_rows_kernel<S, T, DP, true, true, 4, SCORED>) : launch(kv_rows_kernel<S, T, DP, true, false, 4, SCORED>);
            else if (a.G <= 8) one ? launch(kv_rows_kernel<S, T, DP, true, true, 2, SCORED>) : launch(kv_rows_kernel<S, T, DP, true, false, 2, SCORED>);
            else one ? launch(kv_rows_kernel<S, T, DP, true, true, 1, SCORED>) : launch(kv_rows_kernel<S, T, DP, true, false, 1, SCORED>);
        } else {
            one ? launch(kv_rows_kernel<S, T, DP, false, true, 1, SCORED>) : launch(kv_rows_kernel<S, T, DP, false, false, 1, SCORED>);
        }
        if (a.n_split > 1 && !a.join_here) kv_join_kernel<T, DP, 16, SPARSE><<<dim3((unsigned)units, a.c.H), 256, 0, s>>>(a);
    }
    if constexpr (!SPARSE) {
        if (rows > a.few_rows) {
            // (a wave holds 32 x DP sums and the queries: of 256 channels these take all 512 registers, one wave a SIMD, and more over pages of
            // fewer than 64 tokens: 38 go to scratch at 16 bits, 53 with scores of other kinds; 2048 tokens over 8192 700 - 720 us at 16 bits, 1030 - 1040 over such pages, 907 at int8 under bf16.  Of 64 channels 4 waves a workgroup were slower: 16 ragged sequences 171 us, 143
            // with 8)
            constexpr int NW = DP == 256 ? 4 : 8, BR = NW * 32;
            // row tiles of the sequences that have more rows than the others' kernel takes: at most
            const int64_t all = a.b.n_tokens * (int64_t)a.G, longs = std::min<int64_t>(a.b.n_seqs, all / (a.few_rows + 1));
            const int64_t units = alike ? seqs * ((rows + BR - 1) / BR) : std::min(longs * ((rows + BR - 1) / BR), all / BR + longs);
            if (alike) a.few_rows = 0;
            cut(a, units * a.c.H, tiles, BR, a.num_cu, 8, (alike ? 1 : 4) * a.num_cu, 16, INT32_MAX);
            const dim3 grid((unsigned)(units * a.n_split * a.c.H));
            // Of 64 channels at bf16 the compiler gets by with 127 registers, so that two workgroups fit a CU: 15 % less time where there are workgroups for that, 17 % more where
            // there are not, as there the 140 that it takes when told of one workgroup give the better order.  8 heads of 4, us, as chosen (other): 2048 tokens over 16384, 256
            // workgroups, 334 (390); 4096 tokens 594 (588); 2100, 3000 tokens 529 (577), 544 (578); 16384 over 16384 1254 (1385).
            constexpr bool PAIRS = S == PK_BF16 && DP == 64 && !SCORED;
            if (a.c.P >= kKvTile && PAIRS && (int64_t)grid.x <= a.num_cu) kv_tile_kernel<S, T, DP, NW, true, SCORED, PAIRS><<<grid, NW * 64, 0, s>>>(a);
            else if (a.c.P >= kKvTile) kv_tile_kernel<S, T, DP, NW, true, SCORED><<<grid, NW * 64, 0, s>>>(a);
            else kv_tile_kernel<S, T, DP, NW, false, SCORED><<<grid, NW * 64, 0, s>>>(a);
            if (a.n_split > 1) kv_join_kernel<T, DP, BR, false><<<dim3((unsigned)(units * (BR / 16)), a.c.H), 256, 0, s>>>(a);
        }
    }
    return hipGetLastError();
}

template <int S, int T>
hipError_t run_dp(const KvAttend &a, int dp, hipStream_t s)
{
    if (a.blocks) return dp == 64 ? run<S, T, 64, true, false>(a, s) : dp == 128 ? run<S, T, 128, true, false>(a, s) : run<S, T, 256, true, false>(a, s);
    if (a.scored) return dp == 64 ? run<S, T, 64, false, true>(a, s) : dp == 128 ? run<S, T, 128, false, true>(a, s) : run<S, T, 256, false, true>(a, s);
    return dp == 64 ? run<S, T, 64, false, false>(a, s) : dp == 128 ? run<S, T, 128, false, false>(a, s) : run<S, T, 256, false, false>(a, s);
}

// A storage's calls, by the queries' type.
template <int S>
hipError_t run_storage(const KvAttend &a, int dp, int dtype, hipStream_t s)
{
    if constexpr (kv_coded<S>) return dtype == PK_F16 ? run_dp<S, PK_F16>(a, dp, s) : run_dp<S, PK_BF16>(a, dp, s);
    else return run_dp<S, S>(a, dp, s);
}

} // namespace
} // namespace pk
