// Attention over a paged key/value cache: softmax(scale q k) v over the keys that a query sees, for chunks of new tokens
// and for single ones, over all of a sequence's pages or over listed blocks of them.
#include <algorithm>

#include "pk_kv.h"

namespace pk {
namespace {

constexpr int kFewRows = 64;     // most rows of queries of a sequence and head that are taken 16 at a time
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
    if (tile * 16 >= rows || (!SPARSE && rows > a.few_rows)) return;
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
// of 16 neighbouring rows meet all banks.  (Piece p ^ x lies where p does, exclusive-or x.)
template <int CH>
__device__ __forceinline__ int lds_piece(int row, int piece)
{
    return row * CH + (piece ^ (CH == 8 ? (row >> 1) & 7 : row & 15));
}

// A number that all lanes of a wave have.
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The largest of a number's values in lanes l and l ^ 32.
__device__ __forceinline__ float over_halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The largest of three (without the rounds that fmaxf makes for signalling NaNs).
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
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

// The order of N products' instructions: their operands are read from LDS AHEAD of them, and what brings the next tiles in (W writes to LDS,
// L loads) goes between them, one at a time.
template <int AHEAD, int N, int EACH, int W, int L>
__device__ __forceinline__ void in_between()
{
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
        if (i < N - AHEAD) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (i < W) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
        else if (i < W + L) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
}

// Tiles on their way into LDS: their pages, then pieces of K(j) and V(j - 1) in registers, then LDS.
template <int S, int T, int DP, int NW, bool ONE>
struct KvTiles {
    static constexpr int ES = KvBytes<S>::v, NT = NW * 64, CH = DP / 8;
    static constexpr bool CODED = kv_coded<S>;
    static constexpr int PIECES = kKvTile * DP * ES / 16; // 16-byte pieces of a tile of K, and of one of V
    static constexpr int KP = (PIECES + NT - 1) / NT;     // of a thread
    static constexpr int KR = DP * ES / 16;               // pieces of a row of K
    static constexpr int VR = kKvTile * ES / 16;          // pieces of a row of V
    static constexpr int PG = ONE ? 1 : KP;
    static_assert(PIECES % NT == 0 || PIECES < NT, "");
    struct Lds {
        u32x4 k[2][kKvTile * CH];
        u32x4 v[2][DP * 8];
        float scales[CODED ? 4 : 1][2][kKvTile];
    };

    const char *k, *v;
    const float *ks, *vs;
    const int32_t *table;
    uint32_t n_pages;
    int H, h, P, logP, len;
    uint32_t kpage[PG], vpage[PG], spage; // of K(j), of V(j - 1); of the lane's token of K(j)
    u32x4 kw[KP], vw[KP];
    float ksw, vsw;
    uint32_t v_in;    // which of the thread's pieces of V(j - 1) lie in pages that the table has
    bool v_there;     // all of the wave's
    uint32_t in_next; // which of K(j)'s four runs of 16 tokens lie in such pages

    __device__ __forceinline__ void begin(const KvDev &c, const int32_t *t, int head, int tokens)
    {
        k = c.k, v = c.v, ks = c.ks, vs = c.vs, table = t;
        n_pages = c.n_pages, H = c.H, h = head, P = c.P, logP = c.logP, len = tokens;
        spage = 0, ksw = 0.f, vsw = 0.f, in_next = 0, v_in = 0, v_there = true;
    }
    // page of a position, of the nearest that the sequence has where it has none there
    __device__ __forceinline__ uint32_t page_of(int pos) const { return (uint32_t)table[min(max(pos, 0), max(len - 1, 0)) >> logP]; }
    __device__ __forceinline__ size_t place(uint32_t page) const { return (size_t)(page < n_pages ? page : 0) * H + h; }

    __device__ __forceinline__ void lookup(int j)
    {
        const int kb = j * kKvTile, vb = kb - kKvTile, tid = threadIdx.x;
        if constexpr (ONE) {
            kpage[0] = page_of(kb);
            vpage[0] = page_of(vb);
        } else {
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int p = tid + i * NT;
                kpage[i] = page_of(kb + p / KR);
                vpage[i] = page_of(vb + (p % VR) * (16 / ES));
            }
            spage = page_of(kb + (tid & 63));
        }
    }

    __device__ __forceinline__ void fetch(int j)
    {
        const int kb = j * kKvTile, vb = kb - kKvTile, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
        const bool mine = PIECES >= NT || tid < PIECES;
        if constexpr (ONE) {
            // (taken here, not where they were asked for: that would be a wait for all that is on its way)
            asm volatile("" : "+v"(kpage[0]), "+v"(vpage[0]));
            const uint32_t kp = (uint32_t)same((int)kpage[0]), vp = (uint32_t)same((int)vpage[0]);
            const char *kr = k + (place(kp) * P + (kb & (P - 1))) * DP * ES, *vr = v + (place(vp) * DP * P + (vb & (P - 1))) * ES;
            if (mine) {
#pragma unroll
                for (int i = 0; i < KP; ++i) {
                    const int p = tid + i * NT;
                    kw[i] = *reinterpret_cast<const u32x4 *>(kr + (uint32_t)(p * 16));
                    vw[i] = *reinterpret_cast<const u32x4 *>(vr + (uint32_t)((p / VR) * P * ES + (p % VR) * 16));
                }
            }
            in_next = kp < n_pages ? 15u : 0u;
            v_there = vp < n_pages;
            v_in = v_there ? ~0u : 0u;
            if constexpr (CODED) {
                const size_t at = place(kp) * P + (kb & (P - 1));
                if (wave == 0) ksw = ks[at + lane];
                if (wave == NW - 1) vsw = in_next && kb + lane < len ? vs[at + lane] : 0.f;
            }
        } else {
            v_in = 0;
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int p = tid + i * NT;
                if (mine) {
                    kw[i] = *reinterpret_cast<const u32x4 *>(k + ((place(kpage[i]) * P + ((kb + p / KR) & (P - 1))) * DP) * ES + (p % KR) * 16);
                    vw[i] = *reinterpret_cast<const u32x4 *>(v + ((place(vpage[i]) * DP + p / VR) * P + ((vb + (p % VR) * (16 / ES)) & (P - 1))) * ES);
                }
                v_in |= (vpage[i] < n_pages ? 1u : 0u) << i;
            }
            const bool ok = spage < n_pages;
            const unsigned long long b = __ballot(ok);
            in_next = (uint32_t)((b & 1) | (b >> 15 & 2) | (b >> 30 & 4) | (b >> 45 & 8));
            v_there = __all(v_in == (1u << KP) - 1);
            if constexpr (CODED) {
                const size_t at = place(spage) * P + ((kb + lane) & (P - 1));
                if (wave == 0) ksw = ks[at];
                if (wave == NW - 1) vsw = ok && kb + lane < len ? vs[at] : 0.f;
            }
        }
    }

    // Before tile j is written: tokens that no query sees count as zeros, whatever lies there.
    __device__ __forceinline__ void mask(int j)
    {
        const int vb = (j - 1) * kKvTile;
        if (vb >= 0 && vb + kKvTile <= len && v_there) return;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const int p = threadIdx.x + i * NT, held = vb >= 0 && (v_in >> i & 1) ? len - (vb + (p % VR) * (16 / ES)) : 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t keep = 0;
#pragma unroll
                for (int e = 0; e < 4 / ES; ++e) keep |= w * (4 / ES) + e < held ? (ES == 1 ? 0xffu : 0xffffu) << (8 * ES * e) : 0u;
                vw[i][w] &= keep;
            }
        }
    }

    __device__ __forceinline__ void store(int j, Lds &lds) const
    {
        const int kb = j & 1, vb = kb ^ 1, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
        if (PIECES >= NT || tid < PIECES) {
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int p = tid + i * NT;
                if constexpr (CODED) {
                    u32x4 f0, f1;
                    operands<S, T>(kw[i], f0, f1);
                    lds.k[kb][lds_piece<CH>(p / KR, (p % KR) * 2)] = f0;
                    lds.k[kb][lds_piece<CH>(p / KR, (p % KR) * 2 + 1)] = f1;
                    operands<S, T>(vw[i], f0, f1);
                    lds.v[vb][lds_piece<8>(p / VR, (p % VR) * 2)] = f0;
                    lds.v[vb][lds_piece<8>(p / VR, (p % VR) * 2 + 1)] = f1;
                } else {
                    lds.k[kb][lds_piece<CH>(p / KR, p % KR)] = kw[i];
                    lds.v[vb][lds_piece<8>(p / VR, p % VR)] = vw[i];
                }
            }
        }
        if constexpr (CODED) {
            if (wave == 0) lds.scales[j & 3][0][lane] = ksw;
            if (wave == NW - 1) lds.scales[j & 3][1][lane] = vsw;
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
// has grown.  ONE: a tile of keys lies in one page.
template <int S, int T, int DP, int NW, bool ONE>
__global__ __launch_bounds__(NW * 64) void kv_tile_kernel(KvAttend a)
{
    constexpr int BR = NW * 32;
    constexpr bool CODED = kv_coded<S>, HALF = T == PK_F16, TWICE = CODED && !HALF;
    constexpr int KS = DP / 16, DT = DP / 32, CH = DP / 8;
    __shared__ __align__(16) typename KvTiles<S, T, DP, NW, ONE>::Lds lds;
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
    const int from = valid && window > 0 ? max(pos - window + 1, 0) : 0;
    const int32_t *table = a.b.tables + (size_t)seq * a.b.table_stride;
    // tiles of keys of the workgroup (its waves keep step: one whose queries see none of a tile's keys has weights of zero)
    auto first_of = [&](int r) { return window > 0 ? max(start + r / G - window + 1, 0) / kKvTile : 0; };
    auto last_of = [&](int r) { const int p = start + min(r, rows - 1) / G; return p < 0 ? 0 : p / kKvTile + 1; };
    const int t0 = max(first_of(tile * BR), split * a.split_tiles), t1 = min(last_of(tile * BR + BR - 1), (split + 1) * a.split_tiles);

    u32x4 qf[KS];
    {
        const char *qrow = a.q.data + ((size_t)tok * a.q.token_stride + (size_t)(h * G + member) * a.q.head_stride) * 2;
        const float sign = a.scale > 0.f ? 1.f : a.scale < 0.f ? -1.f : 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
            if (valid && k * 16 + hf * 8 < c.D) load_eight<T>(x, qrow, k * 16 + hf * 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[k][i] = pack16<T>(x[2 * i] * sign, x[2 * i + 1] * sign);
        }
    }
    const float qscale = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;

    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f, vunit = 1e-30f;

    KvTiles<S, T, DP, NW, ONE> in;
    in.begin(c, table, h, sq.len);

    // ---- the two phases
    u32x4 pf[4], pr[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) pf[u] = pr[u] = u32x4{0u, 0u, 0u, 0u}; // (the first round has no tile before it)
    f32x16 s[2];
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
            for (int i = 0; i < 16; ++i) s[r][i] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int r = 0; r < 2; ++r) s[r] = mma32<HALF>(lds.k[0][(kp ^ (k * 2)) + r * 32 * CH], qf[k], s[r]);
    };
    // (what a lane holds of s: keys 32 r + 16 u + 8 hf + j at 8 u + j)
    auto weights = [&](int t, uint32_t held) __attribute__((always_inline)) {
        const int base = t * kKvTile;
        const float *ks = lds.scales[CODED ? t & 3 : 0][0], *vs = lds.scales[CODED ? t & 3 : 0][1];
        if constexpr (CODED) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[u >> 1][8 * (u & 1) + j] *= ks[u * 16 + hf * 8 + j];
        }
        if (held != 15u || __any(base + kKvTile - 1 > pos || base < from)) {
            const int last = min(pos, sq.len - 1) - base, since = from - base;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = u * 16 + hf * 8 + j;
                    s[u >> 1][8 * (u & 1) + j] = key <= last && key >= since && (held >> u & 1) ? s[u >> 1][8 * (u & 1) + j] : -INFINITY;
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
        float unit_up = 1.f, per = 1.f;
        if constexpr (CODED && HALF) {
            float big = vs[lane];
#pragma unroll
            for (int d = 1; d < 64; d *= 2) big = fmaxf(big, __shfl_xor(big, d));
            big = fmaxf(big, vunit);
            per = 1.f / big;
            unit_up = vunit * per;
            vunit = big;
        }
        if (__any(most > m || unit_up != 1.f)) {
            const float m1 = fmaxf(m, most);
            const float fade = m1 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m1) * qscale);
            m = m1;
            l *= fade;
            const float f = fade * unit_up;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        const float base_m = (m == -INFINITY ? 0.f : m * qscale) - (HALF ? kHalfTop : 0.f);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u >> 1][8 * (u & 1) + j], qscale, -base_m));
                sum[j & 1] += p[j];
                if constexpr (CODED) p[j] *= vs[u * 16 + hf * 8 + j] * (HALF ? per : 1.f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pf[u][i] = pack16<T>(p[2 * i], p[2 * i + 1]);
                if constexpr (TWICE) pr[u][i] = pack16<T>(p[2 * i] - __uint_as_float(pf[u][i] << 16), p[2 * i + 1] - __uint_as_float(pf[u][i] & 0xffff0000u));
            }
        }
        l += sum[0] + sum[1];
    };

    if (t0 < t1) {
        in.lookup(t0);
        in.fetch(t0);
        in.lookup(t0 + 1);
        in.mask(t0);
        in.store(t0, lds);
        uint32_t held = in.in_next;
        in.fetch(t0 + 1);
        in.lookup(t0 + 2);
        meet();
        if (late) meet();
        for (int t = t0; t < t1; ++t) {
            // tile t + 1 is written (up to t1: the last tile's V comes with it), the next one asked for
            in.mask(t + 1);
            in.store(t + 1, lds);
            const uint32_t held_next = in.in_next;
            in.fetch(t + 2);
            in.lookup(t + 3);
            pv_products(t);
            qk_products(t);
            in_between<4, 4 * DT + 2 * KS, 1, 0, 0>();
            meet();
            weights(t, held);
            held = held_next;
            meet();
        }
        pv_products(t1);
        if (NW > 4 && !late) meet();
    }
    if (!valid) return;
    l += __shfl_xor(l, 32);
    const float back = CODED && HALF ? vunit : 1.f;
    const float mm = m * qscale - (HALF ? kHalfTop : 0.f); // logarithm of what the weights are in units of
    if (a.n_split > 1) {
        const size_t pr = (((size_t)unit * c.H + h) * a.n_split + split) * BR + (wave * 32 + col);
        if (hf == 0) {
            a.part_ml[pr * 2] = mm;
            a.part_ml[pr * 2 + 1] = l;
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
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int dd = d * 32 + b * 8 + hf * 4;
            if (dd < c.D)
                *reinterpret_cast<u32x2 *>(a.out + (oh * c.D + dd) * 2) =
                    u32x2{pack16<T>(o[d][4 * b] * inv, o[d][4 * b + 1] * inv), pack16<T>(o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv)};
        }
    if (hf == 0 && a.lse) a.lse[oh] = l > 0.f ? (mm + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// The parts of a row joined, in order: 16 threads a row.  Parts have BR rows; a workgroup joins 16 of them.
template <int T, int DP, bool SPARSE, int BR>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttend a)
{
    const int r = (blockIdx.x % (BR / 16)) * 16 + (threadIdx.x >> 4), sub = threadIdx.x & 15, h = blockIdx.y;
    const KvDev &c = a.c;
    const int G = a.G;
    const int at_unit = blockIdx.x / (BR / 16);
    int unit, tile;
    if constexpr (BR == 16) {
        unit = at_unit / a.row_tiles;
        tile = at_unit - unit * a.row_tiles;
    } else {
        const KvUnit un = kv_unit<BR>(a, at_unit);
        if (un.seq < 0) return;
        unit = un.seq;
        tile = un.tile;
    }
    const KvSeq sq = kv_seq(a.b, SPARSE ? kv_seq_of(a.b, unit) : unit, c.P);
    const int rows = SPARSE ? G : sq.m * G, row = tile * BR + r;
    if (row >= rows || (BR == 16 && !SPARSE && rows > a.few_rows)) return;
    const size_t at = ((size_t)at_unit * c.H + h) * a.n_split;
    float m = -INFINITY;
    for (int s = 0; s < a.n_split; ++s) m = fmaxf(m, a.part_ml[((at + s) * BR + r) * 2]);
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 y[DP / 64];
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) y[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.n_split; ++s) {
        const float ms = a.part_ml[((at + s) * BR + r) * 2], f = __builtin_amdgcn_exp2f(ms - base);
        if (ms == -INFINITY) continue;
        l += f * a.part_ml[((at + s) * BR + r) * 2 + 1];
#pragma unroll
        for (int d = 0; d < DP / 64; ++d) y[d] += f * *reinterpret_cast<const f32x4 *>(a.part + ((at + s) * BR + r) * DP + d * 64 + sub * 4);
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

// Parts that the keys are cut into: enough workgroups for the whole device, within the room for partial results, each of them with `least`
// tiles of keys.
void cut(KvAttend &a, int64_t items, int64_t tiles, int br, int num_wg, int least)
{
    const int64_t most = std::min<int64_t>((int64_t)kKvMaxPartials * 16 / br / std::max<int64_t>(items, 1), (num_wg + items - 1) / items);
    const int64_t want = std::max<int64_t>(std::min(most, tiles / least), 1);
    a.split_tiles = (int32_t)((tiles + want - 1) / want);
    a.n_split = (int32_t)((tiles + a.split_tiles - 1) / a.split_tiles);
}

template <int S, int T, int DP, bool SPARSE>
hipError_t run(KvAttend a, hipStream_t s)
{
    const int64_t most = std::min<int64_t>(a.b.max_len, (int64_t)a.b.cols * a.c.P);
    const int64_t tiles = std::max<int64_t>(((SPARSE ? (int64_t)a.n_blocks * a.c.P : most) + kKvTile - 1) / kKvTile, 1);
    const int64_t seqs = SPARSE ? a.b.n_tokens : a.b.n_seqs;
    const int64_t rows = SPARSE ? a.G : (int64_t)a.b.max_new * a.G; // of a sequence at most
    a.few_rows = SPARSE ? INT32_MAX : kFewRows;
    // sequences of few rows: unless all have the same number of new tokens, and that is many
    const bool alike = !SPARSE && (int64_t)a.b.n_seqs * a.b.max_new == a.b.n_tokens;
    if (SPARSE || !alike || rows <= a.few_rows) {
        a.row_tiles = (int32_t)((std::min<int64_t>(rows, a.few_rows) + 15) / 16);
        const int64_t units = seqs * a.row_tiles;
        cut(a, units * a.c.H, tiles, 16, 6 * a.num_cu, 4);
        kv_rows_kernel<S, T, DP, SPARSE><<<dim3((unsigned)(units * a.n_split), a.c.H), 256, 0, s>>>(a);
        if (a.n_split > 1) kv_join_kernel<T, DP, SPARSE, 16><<<dim3((unsigned)units, a.c.H), 256, 0, s>>>(a);
    }
    if constexpr (!SPARSE) {
        if (rows > a.few_rows) {
            constexpr int NW = DP == 256 ? 4 : 8, BR = NW * 32;
            // row tiles of the sequences that have more rows than the others' kernel takes: at most
            const int64_t all = a.b.n_tokens * (int64_t)a.G, longs = std::min<int64_t>(a.b.n_seqs, all / (a.few_rows + 1));
            const int64_t units = alike ? seqs * ((rows + BR - 1) / BR) : std::min(longs * ((rows + BR - 1) / BR), all / BR + longs);
            cut(a, units * a.c.H, tiles, BR, a.num_cu, 8);
            const dim3 grid((unsigned)(units * a.n_split * a.c.H));
            if (a.c.P >= kKvTile) kv_tile_kernel<S, T, DP, NW, true><<<grid, NW * 64, 0, s>>>(a);
            else kv_tile_kernel<S, T, DP, NW, false><<<grid, NW * 64, 0, s>>>(a);
            if (a.n_split > 1) kv_join_kernel<T, DP, false, BR><<<dim3((unsigned)(units * (BR / 16)), a.c.H), 256, 0, s>>>(a);
        }
    }
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
