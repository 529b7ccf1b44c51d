// Which blocks of a sequence a query attends to: the ones whose bounds promise the largest scores.
#include <algorithm>

#include "pk_kv.h"

namespace pk {
namespace {

// The scores' order as whole numbers: larger is better; 0 is for blocks that cannot be chosen, ~0 for those that are in any case.
constexpr uint32_t kAlways = 0xffffffffu;
constexpr int kTeam = 4; // most waves that choose for one token (2048 blocks: 1 wave 78, 4 waves 67, 16 waves 67 us)
__device__ __forceinline__ uint32_t score_key(float v)
{
    const uint32_t b = __float_as_uint(v);
    return max(b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u), 1u);
}

// The largest of `gp` neighbouring lanes (a power of two, 16 at most), in all of them.
__device__ __forceinline__ float group_max(float v, int gp)
{
    auto with = [](float x, int moved) __attribute__((always_inline)) { return fmaxf(x, __int_as_float(moved)); };
    if (gp > 1) v = with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
    if (gp > 2) v = with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, true));  // 2 3 0 1
    if (gp > 4) v = with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true)); // 7 6 .. 0
    if (gp > 8) v = with(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true)); // 15 14 .. 0
    return v;
}

// What `f`, whose order does not matter, makes of a number's values in a wave.
template <class F>
__device__ __forceinline__ uint32_t over_wave(uint32_t v, F f)
{
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));  // 2 3 0 1
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true)); // 7 6 .. 0
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true)); // 15 14 .. 0
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(r[0], r[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f(q[0], q[1]);
}
// The sum of the lanes above this one.
__device__ __forceinline__ uint32_t sum_above(uint32_t v)
{
    uint32_t s = v;
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x101, 0xf, 0xf, true); // of the next lane of 16, zero past the last
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x102, 0xf, 0xf, true);
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x104, 0xf, 0xf, true);
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x108, 0xf, 0xf, true);
    const uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)s, 16), c = (uint32_t)__builtin_amdgcn_readlane((int)s, 32);
    const uint32_t d = (uint32_t)__builtin_amdgcn_readlane((int)s, 48);
    const int g = (int)(threadIdx.x >> 4 & 3);
    return s - v + (g < 3 ? d : 0) + (g < 2 ? c : 0) + (g < 1 ? b : 0);
}
// Four of the keys at once, `step` apart: none (0) from `end` on.
__device__ __forceinline__ void four_keys(uint32_t (&key)[4], const uint32_t *k, int i, int step, int end)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) key[j] = i + j * step < end ? k[i + j * step] : 0;
}

// Groups of 2^log_tokens tokens counted over a batch: the first one of sequence s.  There is room between it and the next sequence's for all
// that the sequence can make: with o = a t + r and o' = a' t + r' its offset and the next one's, ceil((o' - o) / t) <= a' - a + 1.
__device__ __forceinline__ int first_group(const KvBatch &b, int s, int log_tokens)
{
    return (min(max(b.offsets[s], 0), b.n_tokens) >> log_tokens) + s;
}
// The sequence that group `unit` is one of, by all lanes of a wave: 64 at once, so that 4096 sequences take two steps.
__device__ __forceinline__ int group_seq(const KvBatch &b, int unit, int log_tokens)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = b.n_seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const bool upto = lane * step < n && first_group(b, lo + lane * step, log_tokens) <= unit;
        const int last = max(__popcll(__ballot(upto)) - 1, 0) * step;
        lo += last;
        n = min(step, n - last);
    }
    return lo;
}

struct KvSelect {
    KvDev c;
    KvBatch b;
    KvRows q;
    int32_t G, n, sink, local;
    int32_t gp, log_gp;         // columns of a token: its query heads, a power of two of 16 at most
    int32_t tokens, log_tokens; // of a workgroup: 16 / gp at most, a power of two
    int32_t groups; // of tokens: of one sequence at most; 0: counted over the batch, and looked up
    int32_t room;   // keys of a token in LDS
    int32_t *out;
};

// One workgroup: a few tokens of one sequence, one key/value head.
//   U[block, head] = sum_c max(q_c hi_c, q_c lo_c) = q+ hi + q- lo, whole numbers: int8 products of the rows [hi, lo] of 16 blocks' bounds with
//   [q+, q-] of 16 columns, the tokens' heads side by side
//   score[block] = max over a token's heads of U scale_q, times the bounds' scale
// No sum of it is rounded, so the choice is the same whatever computes it.  A load takes 64 bytes of a row by four neighbouring lanes and goes to
// the lanes that the product wants by way of LDS.  The keys of the scores stay there; a token's n-th largest is found by its
// bytes, from the first one in which its keys differ, one histogram each, by the waves that have the token (all of them, where it is the only one); each
// of these then has a stretch of the blocks, and what is chosen comes out in ascending order.
// Bound by reading the bounds where there are few tokens (16 waves then), by the steps of the choice where there are many.  Measured, 8 heads
// of 128, 4 query heads each: one token with 313 blocks 12.9 us, 16 tokens with 2048 each 26 us (67 MB of bounds, 13 us at the rate of a large
// copy), 1024 tokens with 512 52 us (8.3 G operations, 3.4 us at the rate of a large int8 product: the steps of the choice).
template <int T, int DP, int NW>
__global__ __launch_bounds__(NW * 64) void kv_select_kernel(KvSelect a)
{
    constexpr int KS = DP / 64; // products over a half of a row of bounds
    extern __shared__ uint32_t keys[];
    __shared__ __align__(16) u32x4 turn[NW][64];
    __shared__ uint32_t hist[NW][256];
    __shared__ uint32_t counts[NW][3], found[NW][2], few[NW][64];
    __shared__ uint32_t goes[3][NW]; // whether a token's waves have more to do
    const KvDev c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % c.H, unit = blockIdx.x / c.H;
    const int seq = a.groups > 0 ? unit / a.groups : group_seq(a.b, unit, a.log_tokens);
    const int first = (unit - (a.groups > 0 ? seq * a.groups : first_group(a.b, seq, a.log_tokens))) * a.tokens;
    const KvSeq sq = kv_seq(a.b, seq, c.P);
    if (first < 0 || first >= sq.m) return;
    const int32_t *table = a.b.tables + (size_t)seq * a.b.table_stride;
    const int start = sq.len - sq.m;
    const int last_pos = start + min(first + a.tokens, sq.m) - 1, nb = last_pos < 0 ? 0 : (last_pos >> c.logP) + 1; // blocks of its last token
    const int tk = col >> a.log_gp, member0 = col & (a.gp - 1);
    const int pos = start + first + tk, mine = pos >> c.logP; // (pos < 0: nothing is seen)
    const bool token_in = tk < a.tokens && first + tk < sq.m;

    for (int gt = 0; gt < a.G; gt += a.gp) {
        // the queries' codes: lane (column, g) has channels 64 k + 16 g .. + 15
        float x[KS][16], most = 0.f;
        const bool in = token_in && gt + member0 < a.G;
        const int tok = sq.first + min(first + tk, sq.m - 1);
        const char *qrow = a.q.data + ((size_t)tok * a.q.token_stride + (size_t)(h * a.G + min(gt + member0, a.G - 1)) * a.q.head_stride) * 2;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = 0.f;
                const int at = k * 64 + g * 16 + e;
                if (in && at < c.D) load_eight<T>(y, qrow, at);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[k][e + j] = y[j];
                    most = fmaxf(most, fabsf(y[j]));
                }
            }
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float up = code_factor(most, 127.f), qscale = most * (1.f / 127.f);
        i32x4 qp[KS], qm[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t p = 0, m = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int code = (int)rintf(fminf(fmaxf(x[k][4 * w + e] * up, -127.f), 127.f));
                    p |= (uint32_t)(uint8_t)(int8_t)max(code, 0) << (8 * e);
                    m |= (uint32_t)(uint8_t)(int8_t)min(code, 0) << (8 * e);
                }
                qp[k][w] = (int)p;
                qm[k][w] = (int)m;
            }
        // a lane loads piece `load_piece` of the bounds of block `load_row`, and has the scores of blocks 4 g .. 4 g + 3
        const int load_row = lane >> 2, load_piece = lane & 3;
        auto page_at = [&](int at) __attribute__((always_inline)) -> uint32_t { return (uint32_t)table[min(at, nb - 1)]; };
        uint32_t lpage = 0, pages[4] = {0, 0, 0, 0};
        auto ask = [&](int b0) __attribute__((always_inline)) {
            lpage = page_at(b0 + load_row);
#pragma unroll
            for (int j = 0; j < 4; ++j) pages[j] = page_at(b0 + g * 4 + j);
        };
        if (wave * 16 < nb) ask(wave * 16);
        for (int b0 = wave * 16; b0 < nb; b0 += NW * 16) {
            const size_t lph = (size_t)(lpage < c.n_pages ? lpage : 0) * c.H + h;
            const int8_t *row = c.bc + lph * 2 * DP + load_piece * 16;
            u32x4 w[2 * KS];
#pragma unroll
            for (int k = 0; k < 2 * KS; ++k) w[k] = *reinterpret_cast<const u32x4 *>(row + k * 64);
            float scale[4];
            bool there[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                there[j] = pages[j] < c.n_pages;
                scale[j] = c.bs[(size_t)(there[j] ? pages[j] : 0) * c.H + h];
            }
            ask(b0 + NW * 16); // (past the last block: the last one's again)
            // row r, piece p lies at 4 r + (p ^ (r / 4)): a quarter of a wave reads 16 rows from banks of their own, 2 at a time.  A wave's accesses
            // are in order: the next piece may be written as soon as this one's read is issued
            i32x4 f[2 * KS];
#pragma unroll
            for (int k = 0; k < 2 * KS; ++k) {
                turn[wave][load_row * 4 + (load_piece ^ (load_row >> 2))] = w[k];
                __builtin_amdgcn_wave_barrier();
                f[k] = __builtin_bit_cast(i32x4, turn[wave][col * 4 + (g ^ (col >> 2))]);
                __builtin_amdgcn_wave_barrier();
            }
            i32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 2 * KS; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(f[k], k < KS ? qp[k % KS] : qm[k % KS], acc, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = group_max(in ? (float)acc[j] * qscale : -INFINITY, a.gp);
                const int at = b0 + g * 4 + j;
                if (token_in && member0 == 0 && at < nb) {
                    uint32_t key = 0;
                    if (pos >= 0 && at <= mine && there[j])
                        key = at < a.sink || at > mine - a.local ? kAlways : score_key(v * scale[j] + 0.f); // (no zero of a sign)
                    uint32_t *k = keys + tk * a.room + at;
                    *k = gt == 0 ? key : max(*k, key);
                }
            }
        }
    }
    __syncthreads();

    // ---- the choice: waves `team` to `team + size - 1` have a token (more tokens than waves: several in turn, a wave each)
    constexpr int kLogWaves = NW == 16 ? 4 : 2, kLogTeam = kTeam == 4 ? 2 : 0;
    static_assert(NW == 1 << kLogWaves && kTeam == 1 << kLogTeam, "");
    const int log_size = min(max(kLogWaves - a.log_tokens, 0), kLogTeam), size = 1 << log_size, turns = max(a.tokens >> kLogWaves, 1);
    const int team = wave >> log_size, rank = wave & (size - 1), members = size * 64, me = rank * 64 + lane, teams = NW >> log_size;
    // where waves share a token, all of the workgroup meet: whether any token's have more to do
    auto meet = [&](int slot, bool go) __attribute__((always_inline)) {
        if (me == 0) goes[slot][team] = go;
        __syncthreads();
        const uint32_t v = lane < teams ? goes[slot][lane] : 0;
        return __ballot(v != 0) != 0;
    };
    for (int u = 0; u < turns; ++u) {
        const int t = team + u * NW; // (u > 0 only where a wave has tokens of its own)
        const bool have = t < a.tokens && first + t < sq.m;
        const uint32_t *k = keys + (have ? t : 0) * a.room;
        const int count = have ? nb : 0;
        // how many there are, how many of them in any case (both fit 16 bits, as LDS holds them), and the first bit in which the others differ
        uint32_t both = 0, low = 0xffffffffu, high = 0;
        for (int i = me; i < count; i += 4 * members) {
            uint32_t key[4];
            four_keys(key, k, i, members, count);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool other = key[j] && key[j] != kAlways;
                both += key[j] == kAlways ? 1u : other ? 1u << 16 : 0u;
                low = min(low, other ? key[j] : 0xffffffffu);
                high = max(high, other ? key[j] : 0u);
            }
        }
        both = over_wave(both, [](uint32_t x, uint32_t y) { return x + y; });
        low = over_wave(low, [](uint32_t x, uint32_t y) { return min(x, y); });
        high = over_wave(high, [](uint32_t x, uint32_t y) { return max(x, y); });
        if (size > 1) {
            if (lane == 0) counts[wave][0] = both, found[wave][0] = low, found[wave][1] = high;
            __syncthreads();
            both = high = 0, low = 0xffffffffu;
            for (int w = 0; w < size; ++w) {
                both += counts[team * size + w][0];
                low = min(low, found[team * size + w][0]);
                high = max(high, found[team * size + w][1]);
            }
        }
        const uint32_t always = both & 0xffff, others = both >> 16;
        uint32_t need = (uint32_t)a.n > always ? (uint32_t)a.n - always : 0;
        // of the keys that are not taken in any case: all where there are no more than that, else those above `bound` and `need` of those equal to it
        const bool all = others <= need, none = need == 0;
        int bits = all || none || low == high ? 0 : 32 - __clz((int)(low ^ high));
        uint32_t mask = bits == 32 ? 0u : ~0u << bits, bound = none ? kAlways : high & mask;
        uint32_t in_bin = others; // keys that agree with `bound` in `mask`
        for (int round = 0; round < 4; ++round) {
            const bool go = bits > 0 && in_bin > 64;
            if (size == 1 && !go) break;
            // (waves that share a token have two histograms in turn: one is cleared while some may still read the other)
            uint32_t *hs = hist[team * size + (size > 1 ? round & 1 : 0)];
            const int shift = max(bits - 8, 0), width = bits - shift;
            for (int i = me; i < 256; i += members) hs[i] = 0;
            if (size == 1) __builtin_amdgcn_wave_barrier();
            else if (!meet(round & 1, go)) break;
            if (go)
                for (int i = me; i < count; i += 4 * members) {
                    uint32_t key[4];
                    four_keys(key, k, i, members, count);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (key[j] && key[j] != kAlways && (key[j] & mask) == bound) atomicAdd(&hs[(key[j] >> shift) & ((1u << width) - 1)], 1u);
                }
            if (size > 1) __syncthreads();
            else __builtin_amdgcn_wave_barrier();
            // how many lie in bins above; a lane has four bins
            uint32_t own[4], sum = 0;
#pragma unroll
            for (int j = 3; j >= 0; --j) {
                own[j] = hs[lane * 4 + j];
                sum += own[j];
            }
            uint32_t above = sum_above(sum);
            int bin = -1;
            uint32_t left = 0, size_of = 0;
#pragma unroll
            for (int j = 3; j >= 0; --j) {
                if (bin < 0 && above < need && above + own[j] >= need) {
                    bin = lane * 4 + j;
                    left = need - above;
                    size_of = own[j];
                }
                above += own[j];
            }
            const unsigned long long has = __ballot(bin >= 0);
            if (go && has) {
                const int l = __ffsll(has) - 1;
                bound |= (uint32_t)__shfl(bin, l) << shift;
                need = (uint32_t)__shfl((int)left, l);
                in_bin = (uint32_t)__shfl((int)size_of, l);
                mask |= ((1u << width) - 1) << shift;
                bits = shift;
            }
        }
        // 64 keys at most are left: each lane has one and counts those above it
        const bool last = bits > 0;
        uint32_t *list = few[team * size], *listed = &counts[team * size][2];
        if (me == 0) *listed = 0;
        if (size == 1) __builtin_amdgcn_wave_barrier();
        if (size > 1 ? meet(2, last) : last) {
            if (last)
                for (int i = me; i < count; i += 4 * members) {
                    uint32_t key[4];
                    four_keys(key, k, i, members, count);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (key[j] && key[j] != kAlways && (key[j] & mask) == bound) list[atomicAdd(listed, 1u)] = key[j];
                }
            if (size > 1) __syncthreads();
            else __builtin_amdgcn_wave_barrier();
            if (last) {
                const uint32_t n = min(in_bin, 64u), own = (uint32_t)lane < n ? list[lane] : 0;
                uint32_t over = 0, equal = 0;
                for (uint32_t i = 0; i < n; ++i) {
                    const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)own, (int)i);
                    over += other > own ? 1u : 0u;
                    equal += other == own ? 1u : 0u;
                }
                const unsigned long long has = __ballot((uint32_t)lane < n && over < need && over + equal >= need);
                const int l = __ffsll(has) - 1;
                bound = (uint32_t)__shfl((int)own, l);
                need -= (uint32_t)__shfl((int)over, l);
            }
        }
        // each wave has a stretch of the blocks: what it takes before the equal ones, the equal ones, and where they go
        const int stretch = (((count + size - 1) >> log_size) + 63) & ~63, i0 = rank * stretch, i1 = min(i0 + stretch, count);
        uint32_t over = 0, equal = 0;
        for (int i = i0; i < i1; i += 256) {
            uint32_t key[4];
            four_keys(key, k, i + lane, 64, i1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                over += (uint32_t)__popcll(__ballot(key[j] == kAlways || (key[j] && (all || key[j] > bound))));
                equal += (uint32_t)__popcll(__ballot(key[j] && key[j] != kAlways && !all && key[j] == bound));
            }
        }
        uint32_t equal_before = 0, place = 0;
        if (size > 1) {
            if (lane == 0) counts[wave][0] = over, counts[wave][1] = equal;
            __syncthreads();
            for (int w = 0; w < size; ++w) {
                const uint32_t o = counts[team * size + w][0], e = counts[team * size + w][1];
                if (w < rank) {
                    place += o + (equal_before < need ? min(e, need - equal_before) : 0);
                    equal_before += e;
                }
            }
        }
        int32_t *o = a.out + ((size_t)(sq.first + min(first + t, sq.m - 1)) * c.H + h) * a.n;
        const unsigned long long below = (1ull << lane) - 1;
        for (int i = i0; i < i1; i += 256) {
            uint32_t key[4];
            four_keys(key, k, i + lane, 64, i1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool is = key[j] && key[j] != kAlways && !all && key[j] == bound;
                const unsigned long long eq = __ballot(is);
                const uint32_t nth = equal_before + (uint32_t)__popcll(eq & below);
                const bool take = key[j] == kAlways || (key[j] && !is && (all || key[j] > bound)) || (is && nth < need);
                const unsigned long long taken = __ballot(take);
                const uint32_t to = place + (uint32_t)__popcll(taken & below);
                if (take && to < (uint32_t)a.n) o[to] = i + j * 64 + lane;
                place += (uint32_t)__popcll(taken);
                equal_before += (uint32_t)__popcll(eq);
            }
        }
        // the last wave knows how many there are in all
        if (have && rank == size - 1)
            for (int i = (int)place + lane; i < a.n; i += 64) o[i] = -1;
    }
}

template <int T, int DP, int NW>
hipError_t run(const KvSelect &a, unsigned grid, size_t lds, hipStream_t s)
{
    if (lds > (32u << 10)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_select_kernel<T, DP, NW>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kv_select_kernel<T, DP, NW><<<dim3(grid), NW * 64, lds, s>>>(a);
    return hipGetLastError();
}

// How the batch is cut: tokens of a workgroup, and workgroups of a head.
int64_t cut(KvSelect &a)
{
    const int64_t most = ((int64_t)a.b.max_len + a.c.P - 1) / a.c.P;
    a.room = (int32_t)std::max<int64_t>(std::min<int64_t>(most, a.b.cols), 1);
    a.log_gp = 0;
    while ((1 << a.log_gp) < a.G && a.log_gp < 4) ++a.log_gp;
    a.gp = 1 << a.log_gp;
    // as many tokens as 16 columns have, as a sequence has, and as LDS has room for the keys of (two workgroups a CU at least, unless one
    // token alone takes more)
    a.tokens = 16 / a.gp;
    while (a.tokens > 1 && (a.tokens / 2 >= a.b.max_new || (int64_t)a.tokens * a.room * 4 > (48 << 10))) a.tokens /= 2;
    a.log_tokens = __builtin_ctz((unsigned)a.tokens);
    // the longest sequence's groups for every one, found by a division; or, where these are more than all tokens can make (a chunk among many
    // sequences), counted over the batch: 64 sequences, one with 4096 new tokens, 88 us, 290 by the longest; 1000, one with 512, 52 and 555
    const int64_t each = (int64_t)a.b.max_new / a.tokens + (a.b.max_new % a.tokens != 0), all = a.b.n_tokens / a.tokens + (int64_t)a.b.n_seqs;
    a.groups = a.b.n_seqs * each <= all ? (int32_t)each : 0;
    return std::min(a.b.n_seqs * each, all);
}

template <int T, int DP>
hipError_t run_waves(KvSelect a, int num_cu, hipStream_t s)
{
    const int64_t grid = cut(a) * a.c.H;
    const size_t lds = (size_t)a.tokens * a.room * 4;
    // few workgroups: 16 waves each, while LDS has room for what they need beside the keys (one token with 313 blocks 12.9 us, 4 waves 13.9; 16
    // with 2048 26.7, 4 waves 50.7; many workgroups: 1024 tokens with 512 122 us, 4 waves 52.9)
    if (grid <= 2 * num_cu && lds <= (120u << 10)) return run<T, DP, 16>(a, (unsigned)grid, lds, s);
    return run<T, DP, 4>(a, (unsigned)grid, lds, s);
}

} // namespace

int64_t kv_select_workgroups(const KvDev &c, const KvBatch &b, int G)
{
    KvSelect a{};
    a.c = c, a.b = b, a.G = G;
    return cut(a) * c.H;
}

hipError_t launch_kv_select(const KvDev &c, int dp, const KvBatch &b, const KvRows &q, int dtype, int G, int n_blocks, int sink, int local,
                            int num_cu, int32_t *out, hipStream_t s)
{
    KvSelect a{};
    a.c = c, a.b = b, a.q = q, a.G = G, a.n = n_blocks, a.sink = sink, a.local = local, a.out = out;
    if (dtype == PK_F16) return dp == 64 ? run_waves<PK_F16, 64>(a, num_cu, s) : dp == 128 ? run_waves<PK_F16, 128>(a, num_cu, s) : run_waves<PK_F16, 256>(a, num_cu, s);
    return dp == 64 ? run_waves<PK_BF16, 64>(a, num_cu, s) : dp == 128 ? run_waves<PK_BF16, 128>(a, num_cu, s) : run_waves<PK_BF16, 256>(a, num_cu, s);
}

} // namespace pk
