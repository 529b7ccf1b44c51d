// Attention over a paged key/value cache: softmax(scale q k) v over the keys that a query sees, for chunks of new tokens
// and for single ones, over all of a sequence's pages or over listed blocks of them.
#include "pk_kv.h"

namespace pk {
namespace {

constexpr float kHalfTop = 15.f; // logarithm of the largest weight in half precision: 2^-39 of it is the smallest
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// acc += A (16 rows x 32) B (32 x 16 columns), 16-bit operands
template <bool HALF>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 acc)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), acc, 0, 0, 0);
}

// Sixteen bytes of a row as operands of a product: one of 8 elements, or two of 8 codes each.
template <int S, int T>
__device__ __forceinline__ void operands(u32x4 w, u32x4 &first, u32x4 &second)
{
    if constexpr (kv_coded<S>) {
        uint32_t lo, hi;
        codes_to<S, T>(w[0], lo, hi);
        first[0] = lo, first[1] = hi;
        codes_to<S, T>(w[1], lo, hi);
        first[2] = lo, first[3] = hi;
        codes_to<S, T>(w[2], lo, hi);
        second[0] = lo, second[1] = hi;
        codes_to<S, T>(w[3], lo, hi);
        second[2] = lo, second[3] = hi;
    } else {
        first = w;
    }
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

// Rows of 16 queries that share a key/value head (query heads of its group, several tokens' where the group is small) against
// keys that four waves of a workgroup take in turns, 64 at a time, with no LDS until they join their results:
//   S^T = K Q^T   rows are keys, columns queries; the products' operands come from memory as they lie there
//   O^T += V^T P^T  whose right operand is, by the choice of which key is which row of K, what a lane holds of S^T already:
//     row m of product t is key 16 (m / 4) + 4 t + (m % 4) of the tile, so that lane (column, quarter g) ends up with keys
//     16 g .. 16 g + 15 of its query, and loads those same 16 tokens of the values' channels
// One pass with a running maximum and sum per query, in 32 bits.  Products are taken in the queries' type, which holds 8-bit codes
// exactly; weights are rounded to it for the second one.  With codes a weight carries the value's scale.  In half precision that
// is in units of the largest scale seen, and the largest weight is 2^kHalfTop, as that type has the more of its range below it; in bfloat16,
// whose 8 bits are fewer than the codes are worth, a weight is the sum of two numbers, and its product two.  blockIdx: row tile of a sequence (sparse: of a token) and part of its keys, head.
template <int S, int T, int DP, bool SPARSE>
__global__ __launch_bounds__(256) void kv_rows_kernel(KvAttend a)
{
    constexpr int ES = KvBytes<S>::v;
    constexpr bool CODED = kv_coded<S>, HALF = T == PK_F16, TWICE = CODED && !HALF;
    constexpr int EL = 16 / ES;               // elements of a 16-byte load
    constexpr int KC = DP / (4 * EL);         // such loads of a lane for one row of K
    constexpr int KS = DP / 32;               // products over the channels
    constexpr int DT = DP / 16;               // tiles of 16 channels of the output
    constexpr int VC = CODED ? 1 : 2;         // loads of a lane for 16 tokens of a channel
    __shared__ float join_o[4][16][DP + 4];
    __shared__ float join_m[4][16], join_l[4][16];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g = lane >> 4;
    const int unit = blockIdx.x / a.n_split, split = blockIdx.x - unit * a.n_split, h = blockIdx.y;
    const KvDev &c = a.c;
    const int P = c.P, G = a.G;

    // the tile's queries
    int seq, tile;
    int token0 = 0;
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
    if (tile * 16 >= rows) return;
    const int row = tile * 16 + col;
    const bool valid = row < rows;
    const int tok = SPARSE ? token0 : sq.first + min(row, rows - 1) / G;
    const int member = min(row, rows - 1) % G;
    const int start = sq.len - sq.m;
    const int my_pos = start + (tok - sq.first);
    const bool stray = SPARSE && (tok < sq.first || tok >= sq.first + sq.m); // a token of no sequence
    // columns without a query see every key (what they compute is dropped)
    const int pos = valid ? (stray ? -1 : my_pos) : 0x7fffffff;
    const int from = valid && !SPARSE && a.window > 0 ? max(pos - a.window + 1, 0) : 0;
    const int32_t *table = a.b.tables + (size_t)seq * a.b.table_stride;
    const int32_t *list = SPARSE ? a.blocks + ((size_t)token0 * c.H + h) * a.n_blocks : nullptr;

    // tiles of 64 keys: those that the first and the last query of the tile see at most
    int t0, t1;
    if constexpr (SPARSE) {
        t0 = split * a.split_tiles;
        t1 = min((a.n_blocks * P + kKvTile - 1) / kKvTile, t0 + a.split_tiles);
    } else {
        const int first_pos = start + (tile * 16) / G, last_pos = start + min(tile * 16 + 15, rows - 1) / G;
        const int lo = a.window > 0 ? max(first_pos - a.window + 1, 0) / kKvTile : 0;
        t0 = max(lo, split * a.split_tiles);
        t1 = min(last_pos < 0 ? 0 : last_pos / kKvTile + 1, (split + 1) * a.split_tiles);
    }

    // queries, as the right operand
    u32x4 qf[KS];
    const float qscale = a.scale * kLog2e;
    {
        const char *qrow = a.q.data + ((size_t)tok * a.q.token_stride + (size_t)(h * G + member) * a.q.head_stride) * 2;
        float x[KS][8];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int at = CODED ? (k >> 1) * 64 + g * 16 + (k & 1) * 8 : k * 32 + g * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] = 0.f;
            if (valid && at < c.D) load_eight<T>(x[k], qrow, at);
        }
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[k][i] = pack16<T>(x[k][2 * i], x[k][2 * i + 1]);
    }

    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f, vunit = 1e-30f;

    // position and page of the 16 tokens `sub` of tile t; a page that is not there has number n_pages at least
    auto sub_base = [&](int t, int sub) -> int {
        if constexpr (SPARSE) {
            const int at = t * kKvTile + sub * 16, bi = at >> c.logP;
            const int block = bi < a.n_blocks ? list[bi] : -1;
            return block < 0 || block > (sq.len - 1) >> c.logP ? -1 : (block << c.logP) + (at & (P - 1));
        } else {
            const int base = t * kKvTile + sub * 16;
            return base < sq.len ? base : -1;
        }
    };
    for (int t = t0 + wave; t < t1; t += 4) {
        const int kb = sub_base(t, col >> 2), vb = sub_base(t, g);
        const uint32_t kpage = kb >= 0 ? kv_page(c, table, kb) : c.n_pages, vpage = vb >= 0 ? kv_page(c, table, vb) : c.n_pages;
        const bool there = vpage < c.n_pages;
        const size_t kph = (size_t)(kpage < c.n_pages ? kpage : 0) * c.H + h, vph = (size_t)(there ? vpage : 0) * c.H + h;
        const int koff = kb >= 0 ? kb & (P - 1) : 0, voff = vb >= 0 ? vb & (P - 1) : 0;
        const char *kr = c.k + (kph * P + koff + (col & 3)) * DP * ES + g * 16;
        const char *vr = c.v + ((vph * DP + col) * P + voff) * ES;

        u32x4 kw[4][KC];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < KC; ++k) kw[i][k] = *reinterpret_cast<const u32x4 *>(kr + i * 4 * DP * ES + k * 64);
        f32x4 ksc[4], vsc[4];
        if constexpr (CODED) {
            const float *ks = c.ks + vph * P + voff, *vs = c.vs + vph * P + voff;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ksc[i] = *reinterpret_cast<const f32x4 *>(ks + 4 * i);
                vsc[i] = *reinterpret_cast<const f32x4 *>(vs + 4 * i);
            }
        }
        u32x4 vw[DT][VC];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int k = 0; k < VC; ++k) vw[d][k] = *reinterpret_cast<const u32x4 *>(vr + (size_t)d * 16 * P * ES + k * 16);

        f32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                u32x4 f0, f1;
                operands<S, T>(kw[i][k], f0, f1);
                if constexpr (CODED) {
                    x[i] = mma<HALF>(f0, qf[2 * k], x[i]);
                    x[i] = mma<HALF>(f1, qf[2 * k + 1], x[i]);
                } else {
                    x[i] = mma<HALF>(f0, qf[k], x[i]);
                }
            }
            if constexpr (CODED) x[i] *= ksc[i];
            x[i] *= qscale;
        }
        // keys that a query does not see; the values of tokens that no query sees are taken as zeros, whatever lies there
        const int seen = min(there ? pos : -1, there ? sq.len - 1 : -1) - vb; // of the lane's 16 keys: 0 .. seen
        const int since = from - vb;
        if (__any(seen < 15 || since > 0 || vb < 0)) {
            const int held = there && vb >= 0 ? sq.len - vb : 0; // of its 16 tokens
            const int last = vb >= 0 ? seen : -1;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = 4 * i + j;
                    x[i][j] = key <= last && key >= since ? x[i][j] : -INFINITY;
                    if constexpr (CODED) vsc[i][j] = key < held ? vsc[i][j] : 0.f;
                }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int k = 0; k < VC; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int w = (k * 4 + i) * (4 / ES); // first token of the word
                        uint32_t keep = 0;
#pragma unroll
                        for (int e = 0; e < 4 / ES; ++e) keep |= w + e < held ? (ES == 1 ? 0xffu : 0xffffu) << (8 * ES * e) : 0u;
                        vw[d][k][i] &= keep;
                    }
        }
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3])));
        most = over_quarters_max(most);
        const float m1 = fmaxf(m, most);
        float fade = __builtin_amdgcn_exp2f(m - (m1 == -INFINITY ? 0.f : m1));
        m = m1;
        const float base = (m1 == -INFINITY ? 0.f : m1) - (HALF ? kHalfTop : 0.f);
        f32x4 p[4];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[i][j] = __builtin_amdgcn_exp2f(x[i][j] - base);
                sum += p[i][j];
            }
        l = l * fade + sum;
        if constexpr (TWICE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] *= vsc[i];
        } else if constexpr (CODED) {
            float big = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) big = fmaxf(big, fmaxf(fmaxf(vsc[i][0], vsc[i][1]), fmaxf(vsc[i][2], vsc[i][3])));
            big = fmaxf(over_quarters_max(big), vunit);
            const float per = 1.f / big;
            fade *= vunit * per;
            vunit = big;
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] *= vsc[i] * per;
        }
        u32x4 pf[2], pr[2]; // weights, and (TWICE) what their rounding left
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p0 = p[2 * u + (i >> 1)][(i & 1) * 2], p1 = p[2 * u + (i >> 1)][(i & 1) * 2 + 1];
                pf[u][i] = pack16<T>(p0, p1);
                if constexpr (TWICE) pr[u][i] = pack16<T>(p0 - __uint_as_float(pf[u][i] << 16), p1 - __uint_as_float(pf[u][i] & 0xffff0000u));
            }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            o[d] *= fade;
            u32x4 f0, f1;
            operands<S, T>(vw[d][0], f0, f1);
            if constexpr (!CODED) f1 = vw[d][VC - 1];
            o[d] = mma<HALF>(f0, pf[0], o[d]);
            o[d] = mma<HALF>(f1, pf[1], o[d]);
            if constexpr (TWICE) {
                o[d] = mma<HALF>(f0, pr[0], o[d]);
                o[d] = mma<HALF>(f1, pr[1], o[d]);
            }
        }
    }

    // the four waves' results joined: everything in units of the largest maximum
    l = over_quarters_sum(l);
    if constexpr (HALF) m -= kHalfTop;
    const float back = CODED && HALF ? vunit : 1.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) join_o[wave][col][d * 16 + g * 4 + i] = o[d][i] * back;
    if (g == 0) {
        join_m[wave][col] = m;
        join_l[wave][col] = l;
    }
    __syncthreads();
    const int r = tid >> 4, sub = tid & 15; // 16 threads a row
    float mm = join_m[0][r];
#pragma unroll
    for (int w = 1; w < 4; ++w) mm = fmaxf(mm, join_m[w][r]);
    const float mb = mm == -INFINITY ? 0.f : mm;
    float f[4], ll = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f[w] = __builtin_amdgcn_exp2f(join_m[w][r] - mb);
        ll += f[w] * join_l[w][r];
    }
    const int orow = tile * 16 + r;
    if (orow >= rows) return;
    if (a.n_split > 1) {
        const size_t at = ((size_t)unit * c.H + h) * a.n_split + split;
        if (sub == 0) {
            a.part_ml[(at * 16 + r) * 2] = mm;
            a.part_ml[(at * 16 + r) * 2 + 1] = ll;
        }
        float *po = a.part + (at * 16 + r) * DP;
#pragma unroll
        for (int d = 0; d < DP; d += 64) {
            const int dd = d + sub * 4;
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] += f[w] * join_o[w][r][dd + i];
            *reinterpret_cast<f32x4 *>(po + dd) = y;
        }
        return;
    }
    const int otok = SPARSE ? token0 : sq.first + orow / G, omember = orow % G;
    const size_t oh = (size_t)otok * c.H * G + h * G + omember;
    const float inv = ll > 0.f ? 1.f / ll : 0.f;
#pragma unroll
    for (int d = 0; d < DP; d += 64) {
        const int dd = d + sub * 4;
        if (dd >= c.D) continue;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] += f[w] * join_o[w][r][dd + i];
        y *= inv;
        *reinterpret_cast<u32x2 *>(a.out + (oh * c.D + dd) * 2) = u32x2{pack16<T>(y[0], y[1]), pack16<T>(y[2], y[3])};
    }
    if (sub == 0 && a.lse) a.lse[oh] = ll > 0.f ? (mm + __builtin_amdgcn_logf(ll)) * kLn2 : -INFINITY;
}

// The parts of a row joined, in order: 16 threads a row.
template <int T, int DP, bool SPARSE>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttend a)
{
    const int r = threadIdx.x >> 4, sub = threadIdx.x & 15, h = blockIdx.y;
    const KvDev &c = a.c;
    const int G = a.G;
    const int unit = blockIdx.x / a.row_tiles, tile = blockIdx.x - unit * a.row_tiles;
    const KvSeq sq = kv_seq(a.b, SPARSE ? kv_seq_of(a.b, unit) : unit, c.P);
    const int rows = SPARSE ? G : sq.m * G, row = tile * 16 + r;
    if (row >= rows) return;
    const size_t at = ((size_t)blockIdx.x * c.H + h) * a.n_split;
    float m = -INFINITY;
    for (int s = 0; s < a.n_split; ++s) m = fmaxf(m, a.part_ml[((at + s) * 16 + r) * 2]);
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 y[DP / 64];
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) y[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.n_split; ++s) {
        const float ms = a.part_ml[((at + s) * 16 + r) * 2], f = __builtin_amdgcn_exp2f(ms - base);
        if (ms == -INFINITY) continue;
        l += f * a.part_ml[((at + s) * 16 + r) * 2 + 1];
#pragma unroll
        for (int d = 0; d < DP / 64; ++d) y[d] += f * *reinterpret_cast<const f32x4 *>(a.part + ((at + s) * 16 + r) * DP + d * 64 + sub * 4);
    }
    const int tok = SPARSE ? unit : sq.first + row / G;
    const size_t oh = (size_t)tok * c.H * G + h * G + row % G;
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) {
        const int dd = d * 64 + sub * 4;
        if (dd >= c.D) continue;
        y[d] *= inv;
        *reinterpret_cast<u32x2 *>(a.out + (oh * c.D + dd) * 2) = u32x2{pack16<T>(y[d][0], y[d][1]), pack16<T>(y[d][2], y[d][3])};
    }
    if (sub == 0 && a.lse) a.lse[oh] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

template <int S, int T, int DP, bool SPARSE>
hipError_t run(const KvAttend &a, hipStream_t s)
{
    const unsigned units = (unsigned)((SPARSE ? a.b.n_tokens : a.b.n_seqs) * a.row_tiles);
    kv_rows_kernel<S, T, DP, SPARSE><<<dim3(units * a.n_split, a.c.H), 256, 0, s>>>(a);
    if (a.n_split > 1) kv_join_kernel<T, DP, SPARSE><<<dim3(units, a.c.H), 256, 0, s>>>(a);
    return hipGetLastError();
}

template <int S, int T>
hipError_t run_dp(const KvAttend &a, int dp, hipStream_t s)
{
    if (a.blocks) return dp == 64 ? run<S, T, 64, true>(a, s) : dp == 128 ? run<S, T, 128, true>(a, s) : run<S, T, 256, true>(a, s);
    return dp == 64 ? run<S, T, 64, false>(a, s) : dp == 128 ? run<S, T, 128, false>(a, s) : run<S, T, 256, false>(a, s);
}

} // namespace

hipError_t launch_kv_attend(const KvAttend &a, int storage, int dp, int dtype, hipStream_t s)
{
    switch (storage) {
    case PK_I8: return dtype == PK_F16 ? run_dp<PK_I8, PK_F16>(a, dp, s) : run_dp<PK_I8, PK_BF16>(a, dp, s);
    case PK_F8: return dtype == PK_F16 ? run_dp<PK_F8, PK_F16>(a, dp, s) : run_dp<PK_F8, PK_BF16>(a, dp, s);
    case PK_F16: return run_dp<PK_F16, PK_F16>(a, dp, s);
    default: return run_dp<PK_BF16, PK_BF16>(a, dp, s);
    }
}

} // namespace pk
