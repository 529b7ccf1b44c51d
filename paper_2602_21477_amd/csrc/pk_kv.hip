// Paged key/value cache: writing tokens into their pages, reading them back, and the host side of all its calls.
// See include/pancake.h for the contract and pk_kv.h for the layout.
#include <algorithm>
#include <cmath>
#include <new>

#include "pk_kv.h"

namespace pk {
namespace {

constexpr int kThreads = 256;
constexpr int kRowLanes = 16; // lanes that share a row: a quarter of a wave
constexpr int kRowsAtOnce = kThreads / kRowLanes;

// The larger and the smaller of two (without the rounds that fmaxf and fminf make for signalling NaNs: a quarter of an append's instructions).  In a wave that is in the IEEE
// mode, as it begins, a signalling NaN would come out as a quiet one, which the next maximum drops along with all before it; out of it a NaN of either
// kind gives the other number.
__device__ __forceinline__ void ignore_nans()
{
    __builtin_amdgcn_s_setreg(1 | 9 << 6 | 0 << 11, 0); // register MODE, from bit 9 (IEEE), one bit
}
__device__ __forceinline__ float larger(float a, float b)
{
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float smaller(float a, float b)
{
    float r;
    asm("v_min_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float larger_size(float a, float x) // of a, which is not negative, and the magnitude of x
{
    float r;
    asm("v_max_f32 %0, %1, |%2|" : "=v"(r) : "v"(a), "v"(x));
    return r;
}

// largest of 2, 4, 8 or 16 neighbouring lanes, in all of them, by lane moves (no LDS)
template <int N>
__device__ __forceinline__ float lanes_max(float x)
{
    auto with = [](float v, int moved) __attribute__((always_inline)) { return larger(v, __int_as_float(moved)); };
    x = with(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xb1, 0xf, 0xf, true));                         // lanes 1 0 3 2
    if constexpr (N >= 4) x = with(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4e, 0xf, 0xf, true));   // 2 3 0 1
    if constexpr (N >= 8) x = with(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true));  // 7 6 .. 0
    if constexpr (N >= 16) x = with(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x140, 0xf, 0xf, true)); // 15 14 .. 0
    return x;
}
// F(x of lanes l, l ^ 16, l ^ 32 and l ^ 48)
template <typename F>
__device__ __forceinline__ float over_quarters(float x, F both)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = both(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return both(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float quarter_max(float x) { return lanes_max<kRowLanes>(x); }

// E consecutive elements of a caller's row, zeros past its D.
template <int T, int E>
__device__ __forceinline__ void load_row(float (&x)[E], const char *row, int at, int D)
{
    if constexpr (E >= 8) {
#pragma unroll
        for (int j = 0; j < E; j += 8) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = 0.f;
            if (at + j < D) load_eight<T>(y, row, at + j);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[j + i] = y[i];
        }
    } else {
        static_assert(E == 4, "");
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = 0.f;
        if (at < D) load_four<T>(x, row, at);
    }
}

// A page's keys (or values) as they lie in memory, in LDS: values with 16 bytes more for every 8 channels, so that lanes that share
// a row write to banks of their own; values of 4 bits as a byte each.
template <int ES, int DP>
__device__ __forceinline__ int v_image(int tok, int d)
{
    return (tok * ES >> 4) * (DP * 18) + d * 16 + (d >> 3) * 16 + (tok * ES & 15);
}
template <int S> constexpr int kv_value_bytes = kv_bits<S> == 16 ? 2 : 1; // of an element there
template <int S, int DP>
constexpr size_t image_bytes(int P)
{
    return (size_t)P * DP * kv_bits<S> / 8 + (size_t)P * kv_value_bytes<S> / 16 * DP * 18;
}

// Sixteen tokens of 4 bits of a channel as bytes, and back.
__device__ __forceinline__ u32x4 unpack_run(uint32_t a, uint32_t b)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t w = i ? b : a, even = w & 0x0f0f0f0fu, odd = w >> 4 & 0x0f0f0f0fu;
        r[2 * i] = __builtin_amdgcn_perm(odd, even, 0x05010400u);
        r[2 * i + 1] = __builtin_amdgcn_perm(odd, even, 0x07030602u);
    }
    return r;
}
__device__ __forceinline__ uint32_t pack_run(uint32_t a, uint32_t b) // eight of them
{
    a &= 0x0f0f0f0fu, b &= 0x0f0f0f0fu; // (what has not been written may be anything)
    a |= a >> 4, b |= b >> 4;           // bytes 0 and 2 hold two codes each
    return __builtin_amdgcn_perm(b, a, 0x06040200u);
}

// What a workgroup does: one page that the batch touches, one head.
struct KvPage {
    KvSeq q;
    int h, lp, base, p0, p1; // the head; the page's number in the sequence, its first position, the rows of the batch's new tokens in it
    uint32_t page;
};
// Heads of a page one after the other, where a grid has that many: rows of a token, heads side by side, are then read (and written) at about
// the same time.
dim3 page_grid(const KvDev &c, const KvBatch &b)
{
    const int64_t pages = kv_touched(c, b);
    return pages * c.H <= kKvMaxGroups ? dim3((unsigned)(pages * c.H), 1, b.n_seqs) : dim3((unsigned)pages, c.H, b.n_seqs);
}
__device__ __forceinline__ bool kv_page_of(const KvDev &c, const KvBatch &b, KvPage &g)
{
    const int s = blockIdx.z;
    g.q = kv_seq(b, s, c.P);
    const int begin = max(g.q.len - g.q.m, 0);
    const bool flat = gridDim.y == 1;
    g.h = flat ? blockIdx.x % c.H : blockIdx.y;
    g.lp = (begin >> c.logP) + (int)(flat ? blockIdx.x / c.H : blockIdx.x);
    if (g.q.m == 0 || ((long long)g.lp << c.logP) >= g.q.len) return false;
    g.page = (uint32_t)b.tables[(size_t)s * b.table_stride + g.lp];
    g.base = g.lp << c.logP;
    g.p0 = max(begin - g.base, 0);
    g.p1 = min(g.q.len - g.base, c.P);
    return true;
}

// Bytes of a lane's E elements of a row: of values in 4 bits, a byte for each.
template <int S, int E, bool VALUES> constexpr int kv_part = S == PK_F4 && VALUES ? E : E * kv_bits<S> / 8;

// E consecutive elements of a row as they are stored: codes with a scale (keys in 4 bits: and the byte of their power of two), or 16 bits.
template <int S, int E, bool VALUES>
__device__ __forceinline__ float encode(const float (&x)[E], char (&codes)[kv_part<S, E, VALUES>], uint32_t &power)
{
    if constexpr (S == PK_F4) {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) most = larger_size(most, x[i]);
        const float group = lanes_max<32 / E>(most); // of 32 channels
        most = quarter_max(most);
        const float up = code_factor(most, kv_largest<S>);
        // (the conversion divides by a power of two before it rounds, and gives 6 for what is beyond: no more than a rounding of the product)
        if constexpr (VALUES) {
#pragma unroll
            for (int i = 0; i < E; i += 4) {
                uint32_t w = 0;
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i] * up, 0.f, 1.f, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i + 1] * up, 0.f, 1.f, 1);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i + 2] * up, 0.f, 1.f, 2);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i + 3] * up, 0.f, 1.f, 3);
                __builtin_memcpy(codes + i, &w, 4);
            }
        } else {
            power = 127u - min((__float_as_uint(most) - __float_as_uint(group)) >> 23, 15u);
            const float unit = power_of(power);
#pragma unroll
            for (int i = 0; i < E; i += 4) {
                uint32_t w = 0;
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i] * up, x[i + 1] * up, unit, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[i + 2] * up, x[i + 3] * up, unit, 1);
                __builtin_memcpy(codes + i / 2, &w, 2);
            }
        }
        return most * (1.f / kv_largest<S>);
    } else if constexpr (kv_coded<S>) {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) most = larger_size(most, x[i]);
        most = quarter_max(most);
        const float up = code_factor(most, kv_largest<S>);
#pragma unroll
        for (int i = 0; i < E; ++i) codes[i] = (char)to_code<S, VALUES>(x[i], up);
        return most * (1.f / kv_largest<S>);
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const uint32_t w = pack16<S>(x[i], x[i + 1]);
            __builtin_memcpy(codes + 2 * i, &w, 4);
        }
        return 1.f;
    }
}
template <int S, bool VALUES>
__device__ __forceinline__ float decode(const char *codes, int i)
{
    if constexpr (S == PK_F4 && !VALUES) return code_value<S, VALUES>((uint8_t)codes[i >> 1] >> 4 * (i & 1) & 15);
    else if constexpr (kv_coded<S>) return code_value<S, VALUES>((uint8_t)codes[i]);
    else {
        uint16_t w;
        __builtin_memcpy(&w, codes + 2 * i, 2);
        if constexpr (S == PK_BF16) return __uint_as_float((uint32_t)w << 16);
        else return (float)__builtin_bit_cast(_Float16, w);
    }
}

// One workgroup: one page that the batch touches, one head.  A row is read by 16 lanes, its largest magnitude found by four
// exchanges; the page's new parts are put together in LDS and go out 16 bytes a lane, in order.  The bounds of the page's
// keys are made of the rows that the cache holds once the call is over: those of this call from registers, older ones
// read back.  They depend on the rows alone, not on the calls that brought them.  Every row is read once
// and its codes written once, in the order of memory: without the page put together in LDS first, values went out a byte at a time (a
// prompt of 65536 tokens with its reading back 245 us, with it 199).  Measured (medians): 65536 tokens of 8 heads of 128 from half precision to int8,
// 403 MB in 99 us, 4.1 TB/s, the vector units (maxima, codes, bounds) two thirds busy; to 4 bits, 341 MB in 100 us, 3.4 TB/s; from bf16 to bf16, 537 MB in
// 122 us, 4.4 TB/s; of 64 channels 49 - 57 us (166 - 174 where two lanes each read the eight elements that they share).  One token of each of 64 sequences 7.1 us, of which most is the older rows of 512 pages read
// back for their bounds, after two dependent loads.
template <int S, int T, int DP>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvDev c, KvBatch b, KvRows kin, KvRows vin)
{
    constexpr int RB = DP * kv_bits<S> / 8, ES = kv_value_bytes<S>;
    constexpr int E = DP / kRowLanes; // elements of a lane
    constexpr int KB = kv_part<S, E, false>, N = KB < 16 ? KB : 16; // its bytes of a key, which lie in pieces of 16, or in one
    constexpr bool FOUR = S == PK_F4;
    extern __shared__ __align__(16) char image[];
    __shared__ float red[4][2][DP];
    const int tid = threadIdx.x;
    KvPage g;
    if (!kv_page_of(c, b, g) || g.page >= c.n_pages) return;
    if constexpr (kv_coded<S>) ignore_nans(); // (a row that is only rounded has no maximum, and a signalling NaN is quiet from then on; not before the page's loads, which wait for it: 2 - 3 % of an append, 8 - 10 % over pages of 16 tokens)
    const int h = g.h, p0 = g.p0, p1 = g.p1;
    char *kimg = image, *vimg = image + c.P * RB;
    const size_t ph = (size_t)g.page * c.H + h;
    char *kp = c.k + ph * c.P * RB;
    char *vp = c.v + ph * c.P * RB;
    uint8_t *ke = FOUR ? c.ke + ph * c.P * (DP / 32) : nullptr;
    const int sub = tid & (kRowLanes - 1), at = sub * E;

    float hi[E], lo[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        hi[i] = -INFINITY;
        lo[i] = INFINITY;
    }
    auto bound = [&](const char *codes, float scale, uint32_t power) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            float z;
            if constexpr (FOUR) {
                const f32x2 both = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)(uint8_t)codes[i / 2], power_of(power), 0);
                z = both[i & 1];
            } else {
                z = decode<S, false>(codes, i);
            }
            if constexpr (kv_coded<S>) z *= scale;
            hi[i] = larger(hi[i], z);
            lo[i] = smaller(lo[i], z);
        }
    };
    // rows that were there, several asked for at once
    constexpr int AHEAD = 4;
    for (int r0 = 0; r0 < p0; r0 += AHEAD * kRowsAtOnce) {
        char codes[AHEAD][KB];
        float scale[AHEAD];
        uint32_t power[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int r = min(r0 + k * kRowsAtOnce + tid / kRowLanes, p0 - 1); // (a row twice is no other bound)
#pragma unroll
            for (int i = 0; i < KB; i += N) __builtin_memcpy(codes[k] + i, kp + k_place<RB>(r, sub * KB + i), N);
            scale[k] = kv_coded<S> ? c.ks[ph * c.P + r] : 1.f;
            power[k] = FOUR ? ke[e_place<DP>(r, at / 32)] : 0;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) bound(codes[k], scale[k], power[k]);
    }
    // new rows
    for (int r0 = p0 / kRowsAtOnce * kRowsAtOnce; r0 < p1; r0 += kRowsAtOnce) {
        const int r = r0 + tid / kRowLanes;
        if (r < p0 || r >= p1) continue;
        const int t = g.q.first + (g.base + r - (g.q.len - g.q.m));
        char codes[KB], vcodes[kv_part<S, E, true>];
        uint32_t power = 0;
        float x[E], y[E];
        load_row<T, E>(x, kin.data + ((size_t)t * kin.token_stride + (size_t)h * kin.head_stride) * (T == PK_F32 ? 4 : 2), at, c.D);
        load_row<T, E>(y, vin.data + ((size_t)t * vin.token_stride + (size_t)h * vin.head_stride) * (T == PK_F32 ? 4 : 2), at, c.D);
        const float vscale = encode<S, E, true>(y, vcodes, power);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (ES == 1) vimg[v_image<ES, DP>(r, at + i)] = vcodes[i];
            else __builtin_memcpy(vimg + v_image<ES, DP>(r, at + i), vcodes + 2 * i, 2);
        }
        const float scale = encode<S, E, false>(x, codes, power);
#pragma unroll
        for (int i = 0; i < KB; i += N) __builtin_memcpy(kimg + k_place<RB>(r, sub * KB + i), codes + i, N);
        if constexpr (FOUR) {
            if (at % 32 == 0) ke[e_place<DP>(r, at / 32)] = (uint8_t)power;
        }
        if constexpr (kv_coded<S>) {
            if (sub == 0) {
                c.ks[ph * c.P + r] = scale;
                c.vs[ph * c.P + r] = vscale;
            }
        }
        bound(codes, scale, power);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
        hi[i] = over_quarters(hi[i], larger);
        lo[i] = over_quarters(lo[i], smaller);
        if ((tid & 63) < kRowLanes) {
            red[tid >> 6][0][at + i] = hi[i];
            red[tid >> 6][1][at + i] = lo[i];
        }
    }
    __syncthreads();
    if (tid < kRowLanes) {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
#pragma unroll
            for (int w = 1; w < 4; ++w) {
                hi[i] = larger(hi[i], red[w][0][at + i]);
                lo[i] = smaller(lo[i], red[w][1][at + i]);
            }
            most = larger_size(larger_size(most, hi[i]), lo[i]);
        }
        most = quarter_max(most);
        const float up = code_factor(most, 127.f);
        constexpr float kSlack = 1.f / 1024.f; // of a step: a bound this little beyond a whole number is that number
        int8_t *bc = c.bc + ph * 2 * DP;
        char bh[E], bl[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            bh[i] = (char)(int)fminf(fmaxf(ceilf(__fsub_rn(__fmul_rn(hi[i], up), kSlack)), -127.f), 127.f);
            bl[i] = (char)(int)fminf(fmaxf(floorf(__fadd_rn(__fmul_rn(lo[i], up), kSlack)), -127.f), 127.f);
        }
        __builtin_memcpy(bc + at, bh, E);
        __builtin_memcpy(bc + DP + at, bl, E);
        if (tid == 0) c.bs[ph] = most * (1.f / 127.f);
    }
    // keys: a piece is part of one token; values: 16 or 8 tokens of a channel, one by one where not all of them are new
    constexpr int VN = 16 / ES, PIECES = RB / 16;
    for (int i = (p0 >> 2) * 4 * PIECES + tid; i < ((p1 + 3) >> 2) * 4 * PIECES; i += kThreads) {
        const int tok = i / (4 * PIECES) * 4 + (i & 3);
        if (tok >= p0 && tok < p1) *reinterpret_cast<u32x4 *>(kp + (size_t)i * 16) = *reinterpret_cast<const u32x4 *>(kimg + i * 16);
    }
    if constexpr (FOUR) { // 16 tokens of two channels a piece; what is not new is kept
        for (int i = (p0 >> 4) * (DP / 2) + tid; i < ((p1 + 15) >> 4) * (DP / 2); i += kThreads) {
            const int tok = i / (DP / 2) * 16, d = i % (DP / 2) / 16 * 32 + i % 16;
            if (d >= c.D) continue;
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const char *from = vimg + v_image<1, DP>(tok + (j & 1) * 8, d + (j >> 1) * 16);
                w[j] = pack_run(reinterpret_cast<const uint32_t *>(from)[0], reinterpret_cast<const uint32_t *>(from)[1]);
            }
            u32x4 *to = reinterpret_cast<u32x4 *>(vp + (size_t)i * 16);
            if (tok < p0 || tok + 16 > p1) {
                const u32x4 old = *to;
                const unsigned long long upto = p1 - tok >= 16 ? ~0ull : (1ull << 4 * (p1 - tok)) - 1, fresh = upto & (~0ull << 4 * max(p0 - tok, 0));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t keep = ~(uint32_t)(fresh >> 32 * (j & 1));
                    w[j] = (w[j] & ~keep) | (old[j] & keep);
                }
            }
            *to = w;
        }
        return;
    }
    for (int i = p0 / VN * DP + tid; i < (p1 + VN - 1) / VN * DP; i += kThreads) {
        const int tok = i / DP * VN, d = i % DP;
        if (d >= c.D) continue;
        const char *from = vimg + v_image<ES, DP>(tok, d);
        if (tok >= p0 && tok + VN <= p1) {
            *reinterpret_cast<u32x4 *>(vp + (size_t)i * 16) = *reinterpret_cast<const u32x4 *>(from);
        } else {
            for (int j = max(tok, p0); j < min(tok + VN, p1); ++j) {
                if constexpr (ES == 1) vp[(size_t)i * 16 + (j - tok)] = from[j - tok];
                else reinterpret_cast<uint16_t *>(vp + (size_t)i * 16)[j - tok] = reinterpret_cast<const uint16_t *>(from)[j - tok];
            }
        }
    }
}

// One workgroup: one page of the batch's tokens, one head: the page into LDS as it lies in memory, out of it by rows, 16 lanes each.
// Bound by memory: 131071 tokens of 8 heads of 128 from e4m3 to half precision, 805 MB in 168 us (median), 4.8 TB/s; 65536 from bf16 to bf16,
// 537 MB in 118 us, 4.5 TB/s.
template <int S, int T, int DP>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvDev c, KvBatch b, char *kout, char *vout)
{
    constexpr int RB = DP * kv_bits<S> / 8, ES = kv_value_bytes<S>, TS = T == PK_F32 ? 4 : 2, E = DP / kRowLanes, KB = kv_part<S, E, false>;
    constexpr bool FOUR = S == PK_F4;
    extern __shared__ __align__(16) char image[];
    const int tid = threadIdx.x;
    KvPage g;
    if (!kv_page_of(c, b, g)) return;
    const int h = g.h;
    const bool there = g.page < c.n_pages;
    char *kimg = image, *vimg = image + c.P * RB;
    const size_t ph = (size_t)(there ? g.page : 0) * c.H + h;
    const char *kp = c.k + ph * c.P * RB, *vp = c.v + ph * c.P * RB;
    constexpr int N = 16 / ES, PIECES = RB / 16;
    for (int i = (g.p0 >> 2) * 4 * PIECES + tid; i < ((g.p1 + 3) >> 2) * 4 * PIECES; i += kThreads)
        *reinterpret_cast<u32x4 *>(kimg + i * 16) = *reinterpret_cast<const u32x4 *>(kp + (size_t)i * 16);
    if constexpr (FOUR) {
        for (int i = (g.p0 >> 4) * (DP / 2) + tid; i < ((g.p1 + 15) >> 4) * (DP / 2); i += kThreads) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(vp + (size_t)i * 16);
            char *to = vimg + v_image<1, DP>(i / (DP / 2) * 16, i % (DP / 2) / 16 * 32 + i % 16);
            *reinterpret_cast<u32x4 *>(to) = unpack_run(w[0], w[1]);
            *reinterpret_cast<u32x4 *>(to + v_image<1, DP>(0, 16)) = unpack_run(w[2], w[3]);
        }
    } else {
        for (int i = g.p0 / N * DP + tid; i < (g.p1 + N - 1) / N * DP; i += kThreads)
            *reinterpret_cast<u32x4 *>(vimg + v_image<ES, DP>(i / DP * N, i % DP)) = *reinterpret_cast<const u32x4 *>(vp + (size_t)i * 16);
    }
    __syncthreads();
    const int sub = tid & (kRowLanes - 1), at = sub * E;
    if (at >= c.D) return;
    for (int r = g.p0 + tid / kRowLanes; r < g.p1; r += kRowsAtOnce) {
        float ks = there ? 1.f : 0.f, vs = ks;
        if constexpr (kv_coded<S>) {
            ks = there ? c.ks[ph * c.P + r] : 0.f;
            vs = there ? c.vs[ph * c.P + r] : 0.f;
        }
        const size_t t = (size_t)(g.q.first + (g.base + r - (g.q.len - g.q.m)));
        const size_t o = ((t * c.H + h) * c.D + at) * TS;
        char codes[KB];
        constexpr int M = KB < 16 ? KB : 16;
#pragma unroll
        for (int i = 0; i < KB; i += M) __builtin_memcpy(codes + i, kimg + k_place<RB>(r, sub * KB + i), M);
        float power = 1.f;
        if constexpr (FOUR) power = !there ? 1.f : power_of(c.ke[ph * c.P * (DP / 32) + e_place<DP>(r, at / 32)]);
        float x[E], y[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            x[i] = there ? decode<S, false>(codes, i) : 0.f;
            y[i] = there ? decode<S, true>(vimg + v_image<ES, DP>(r, at + i), 0) : 0.f;
            if constexpr (FOUR) x[i] *= power;
            if constexpr (kv_coded<S>) {
                x[i] *= ks;
                y[i] *= vs;
            }
        }
        // (D is a multiple of 8: a lane of 4 or 8 elements has all of them or none, one of 16 its first 8 at least)
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            if (at + i >= c.D) continue;
            if constexpr (T == PK_F32) {
                *reinterpret_cast<f32x4 *>(kout + o + i * 4) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
                *reinterpret_cast<f32x4 *>(vout + o + i * 4) = f32x4{y[i], y[i + 1], y[i + 2], y[i + 3]};
            } else if constexpr (E == 4) {
                *reinterpret_cast<u32x2 *>(kout + o) = u32x2{pack16<T>(x[0], x[1]), pack16<T>(x[2], x[3])};
                *reinterpret_cast<u32x2 *>(vout + o) = u32x2{pack16<T>(y[0], y[1]), pack16<T>(y[2], y[3])};
            } else if (i % 8 == 0) {
                *reinterpret_cast<u32x4 *>(kout + o + i * 2) = u32x4{pack16<T>(x[i], x[i + 1]), pack16<T>(x[i + 2], x[i + 3]), pack16<T>(x[i + 4], x[i + 5]), pack16<T>(x[i + 6], x[i + 7])};
                *reinterpret_cast<u32x4 *>(vout + o + i * 2) = u32x4{pack16<T>(y[i], y[i + 1]), pack16<T>(y[i + 2], y[i + 3]), pack16<T>(y[i + 4], y[i + 5]), pack16<T>(y[i + 6], y[i + 7])};
            }
        }
    }
}

// The bounds of listed pages as numbers, a page a workgroup (and every kMaxBounds-th after it: a grid has 32 bits for its threads).  Small: 64
// pages of 8 heads 3.0 us, which is a launch and two loads, 1024 pages 5.8 us.
constexpr int64_t kMaxBounds = 1 << 20;
__global__ __launch_bounds__(kThreads) void kv_bounds_kernel(KvDev c, int dp, const int32_t *pages, int64_t n_listed, float *hi, float *lo)
{
    for (size_t n = blockIdx.x; n < (size_t)n_listed; n += kMaxBounds) {
        const uint32_t page = (uint32_t)pages[n];
        const bool there = page < c.n_pages;
        for (int i = threadIdx.x * 4; i < c.H * c.D; i += kThreads * 4) { // (D is a multiple of 8: four channels are of one head)
            const int h = i / c.D, d = i - h * c.D;
            const size_t ph = (size_t)(there ? page : 0) * c.H + h;
            const float s = there ? c.bs[ph] : 0.f;
            char bh[4], bl[4];
            __builtin_memcpy(bh, c.bc + ph * 2 * dp + d, 4);
            __builtin_memcpy(bl, c.bc + (ph * 2 + 1) * dp + d, 4);
            f32x4 x, y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = there ? (float)(int8_t)bh[j] * s : 0.f;
                y[j] = there ? (float)(int8_t)bl[j] * s : 0.f;
            }
            *reinterpret_cast<f32x4 *>(hi + n * c.H * c.D + i) = x;
            *reinterpret_cast<f32x4 *>(lo + n * c.H * c.D + i) = y;
        }
    }
}

// A launch with LDS for a page's keys and values.
template <typename K, typename... A>
hipError_t with_image(K kernel, size_t lds, dim3 grid, hipStream_t s, A... args)
{
    if (lds > (48u << 10)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kernel<<<grid, kThreads, lds, s>>>(args...);
    return hipGetLastError();
}

template <int S, int T>
hipError_t append_dp(const KvDev &c, int dp, const KvBatch &b, const KvRows &k, const KvRows &v, hipStream_t s)
{
    const dim3 grid = page_grid(c, b);
    if (dp == 64) return with_image(kv_append_kernel<S, T, 64>, image_bytes<S, 64>(c.P), grid, s, c, b, k, v);
    if (dp == 128) return with_image(kv_append_kernel<S, T, 128>, image_bytes<S, 128>(c.P), grid, s, c, b, k, v);
    return with_image(kv_append_kernel<S, T, 256>, image_bytes<S, 256>(c.P), grid, s, c, b, k, v);
}

template <int S>
hipError_t append_s(const KvDev &c, int dp, const KvBatch &b, const KvRows &k, const KvRows &v, int dtype, hipStream_t s)
{
    if (dtype == PK_F32) return append_dp<S, PK_F32>(c, dp, b, k, v, s);
    if (dtype == PK_F16) return append_dp<S, PK_F16>(c, dp, b, k, v, s);
    return append_dp<S, PK_BF16>(c, dp, b, k, v, s);
}

template <int S, int T>
hipError_t read_dp(const KvDev &c, int dp, const KvBatch &b, char *k, char *v, hipStream_t s)
{
    const dim3 grid = page_grid(c, b);
    if (dp == 64) return with_image(kv_read_kernel<S, T, 64>, image_bytes<S, 64>(c.P), grid, s, c, b, k, v);
    if (dp == 128) return with_image(kv_read_kernel<S, T, 128>, image_bytes<S, 128>(c.P), grid, s, c, b, k, v);
    return with_image(kv_read_kernel<S, T, 256>, image_bytes<S, 256>(c.P), grid, s, c, b, k, v);
}

template <int S>
hipError_t read_s(const KvDev &c, int dp, const KvBatch &b, char *k, char *v, int dtype, hipStream_t s)
{
    if (dtype == PK_F32) return read_dp<S, PK_F32>(c, dp, b, k, v, s);
    if (dtype == PK_F16) return read_dp<S, PK_F16>(c, dp, b, k, v, s);
    return read_dp<S, PK_BF16>(c, dp, b, k, v, s);
}

} // namespace

hipError_t launch_kv_append(const KvDev &c, int storage, int dp, const KvBatch &b, const KvRows &k, const KvRows &v, int dtype, hipStream_t s)
{
    switch (storage) {
    case PK_I8: return append_s<PK_I8>(c, dp, b, k, v, dtype, s);
    case PK_F8: return append_s<PK_F8>(c, dp, b, k, v, dtype, s);
    case PK_F4: return append_s<PK_F4>(c, dp, b, k, v, dtype, s);
    case PK_F16: return append_s<PK_F16>(c, dp, b, k, v, dtype, s);
    default: return append_s<PK_BF16>(c, dp, b, k, v, dtype, s);
    }
}

hipError_t launch_kv_read(const KvDev &c, int storage, int dp, const KvBatch &b, void *k, void *v, int dtype, hipStream_t s)
{
    char *ko = static_cast<char *>(k), *vo = static_cast<char *>(v);
    switch (storage) {
    case PK_I8: return read_s<PK_I8>(c, dp, b, ko, vo, dtype, s);
    case PK_F8: return read_s<PK_F8>(c, dp, b, ko, vo, dtype, s);
    case PK_F4: return read_s<PK_F4>(c, dp, b, ko, vo, dtype, s);
    case PK_F16: return read_s<PK_F16>(c, dp, b, ko, vo, dtype, s);
    default: return read_s<PK_BF16>(c, dp, b, ko, vo, dtype, s);
    }
}

hipError_t launch_kv_bounds(const KvDev &c, int dp, const int32_t *pages, int64_t n, float *hi, float *lo, hipStream_t s)
{
    kv_bounds_kernel<<<dim3((unsigned)std::min(n, kMaxBounds)), kThreads, 0, s>>>(c, dp, pages, n, hi, lo);
    return hipGetLastError();
}

} // namespace pk

// ------------------------------------------------------------------ host side

using namespace pk;

namespace {

constexpr float kLeastBiasedScale = 0x1p-60f; // of products, or of capped scores: what a bias is made one of
constexpr int kMaxHeads = 1024; // key/value heads of a cache, and query heads of one of them

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

int padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

bool valid(const pk_kv_config *g)
{
    return g && g->n_pages >= 1 && g->n_pages <= 0x7fffffff && g->n_heads >= 1 && g->n_heads <= kMaxHeads && g->head_dim >= 8 &&
           g->head_dim <= PK_KV_MAX_DIM && g->head_dim % 8 == 0 && g->page_tokens >= 16 && g->page_tokens <= kKvMaxPage &&
           (g->page_tokens & (g->page_tokens - 1)) == 0 && (kv_is_coded(g->storage) || g->storage == PK_F16 || g->storage == PK_BF16);
}

// Regions of the arena; base may be null (sizes only).
size_t lay_out(const pk_kv_config &g, char *base, KvDev *c)
{
    const int dp = padded(g.head_dim);
    const size_t row = kv_row_bytes(g.storage, dp), ph = (size_t)g.n_pages * g.n_heads;
    size_t off = 0;
    auto take = [&](size_t n) {
        char *p = base ? base + off : nullptr;
        off = up256(off + n);
        return p;
    };
    c->k = take(ph * g.page_tokens * row);
    c->v = take(ph * g.page_tokens * row);
    const size_t scales = kv_is_coded(g.storage) ? ph * g.page_tokens * sizeof(float) : 0;
    c->ks = reinterpret_cast<float *>(take(scales));
    c->vs = reinterpret_cast<float *>(take(scales));
    c->ke = reinterpret_cast<uint8_t *>(take(g.storage == PK_F4 ? ph * g.page_tokens * (dp / 32) : 0));
    c->bc = reinterpret_cast<int8_t *>(take(ph * 2 * dp));
    c->bs = reinterpret_cast<float *>(take(ph * sizeof(float)));
    c->n_pages = (uint32_t)g.n_pages;
    c->H = g.n_heads;
    c->D = g.head_dim;
    c->P = g.page_tokens;
    c->logP = __builtin_ctz((unsigned)g.page_tokens);
    return off;
}

bool row_type(int32_t t) { return t == PK_F32 || t == PK_F16 || t == PK_BF16; }

int take_rows(const pk_rows *r, KvRows *o)
{
    if (!r || !r->data || !row_type(r->dtype) || r->token_stride < 0 || r->head_stride < 0) return PK_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(r->data) % (r->dtype == PK_F32 ? 4 : 2)) return PK_ERR_INVALID_ARG;
    *o = KvRows{static_cast<const char *>(r->data), r->token_stride, r->head_stride};
    return PK_OK;
}

// Queries of a 16-bit type; a cache of a 16-bit storage takes its own type only.
int take_queries(const pk_kv *kv, const pk_rows *q, int32_t n_q_heads, KvRows *o, int *group)
{
    const int rc = take_rows(q, o);
    if (rc != PK_OK) return rc;
    if (n_q_heads < 1 || n_q_heads % kv->cfg.n_heads) return PK_ERR_INVALID_ARG;
    *group = n_q_heads / kv->cfg.n_heads;
    if (*group > kMaxHeads || q->dtype == PK_F32) return PK_ERR_UNSUPPORTED;
    if ((kv->cfg.storage == PK_F16 || kv->cfg.storage == PK_BF16) && q->dtype != kv->cfg.storage) return PK_ERR_UNSUPPORTED;
    return PK_OK;
}

int attend(pk_kv *kv, const pk_kv_batch *batch, const pk_rows *q, int32_t n_q_heads, float scale, int32_t window, const int32_t *blocks,
           int32_t n_blocks, const pk_kv_scores *scores, void *out, float *lse, hipStream_t s)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    KvAttend a{};
    bool none;
    int rc = kv_take_batch(kv, batch, &a.b, &none);
    if (rc != PK_OK) return rc;
    if (window < 0 || !std::isfinite(scale)) return PK_ERR_INVALID_ARG;
    if (scores && !(scores->cap >= 0.f && std::isfinite(scores->cap))) return PK_ERR_INVALID_ARG;
    if (none) return PK_OK;
    rc = take_queries(kv, q, n_q_heads, &a.q, &a.G);
    if (rc != PK_OK) return rc;
    if (!out || reinterpret_cast<uintptr_t>(out) % 16) return PK_ERR_INVALID_ARG;
    a.c = kv->dev;
    a.scale = scale;
    a.window = (int32_t)std::min<int64_t>(window, kKvMaxTokens); // (a position before the first one less the window fits 32 bits too)
    a.blocks = blocks;
    a.n_blocks = n_blocks;
    if (scores && (scores->cap > 0.f || scores->slopes || scores->starts || scores->prefix)) {
        // (a bias is made one of the products that the scale multiplies)
        if (scores->slopes && scale != 0.f && std::fabs(scale) < kLeastBiasedScale) return PK_ERR_UNSUPPORTED;
        a.scored = 1;
        // (nothing, and no cap at all, in 32 bits: a product over the cap, in the units of the scale, is a normal number)
        const float most = std::min(std::fabs(scale), 1.f) * 0x1p126f;
        a.cap = scores->cap > 0.f ? std::min({std::max(scores->cap, kLeastBiasedScale), scale != 0.f ? std::max(most, 128.f) : 1e37f, 1e37f}) : 0.f;
        a.slopes = scores->slopes;
        a.starts = scores->starts;
        a.prefix = scores->prefix;
    }
    a.out = static_cast<char *>(out);
    a.lse = lse;
    a.num_cu = kv->num_cu;
    const int64_t H = kv->cfg.n_heads, rows = (int64_t)a.b.n_tokens * a.G;
    const int64_t few = blocks ? (int64_t)a.b.n_tokens * ((a.G + 15) / 16) : a.b.n_seqs * std::min<int64_t>(((int64_t)a.b.max_new * a.G + 15) / 16, kKvFewRows / 16);
    const int64_t many = blocks ? 0 : rows / 128 + a.b.n_seqs;
    if (few * H > kKvMaxGroups || many * H > kKvMaxGroups / 2) return PK_ERR_UNSUPPORTED;
    a.part = reinterpret_cast<float *>(kv->ws);
    a.part_floats = kKvPartFloats;
    a.part_ml = a.part + kKvPartFloats;
    a.part_q = a.part_ml + kKvPartFloats / kv->dp * 2;
    a.arrivals = reinterpret_cast<uint32_t *>(a.part_q + kKvPartFloats / kv->dp);
    return launch_kv_attend(a, kv->cfg.storage, kv->dp, q->dtype, s) == hipSuccess ? PK_OK : PK_ERR_HIP;
}

} // namespace

extern "C" {

size_t pk_kv_arena_bytes(const pk_kv_config *cfg)
{
    KvDev c;
    return valid(cfg) ? lay_out(*cfg, nullptr, &c) : 0;
}

int pk_kv_create(const pk_kv_config *cfg, void *arena, size_t arena_bytes, pk_kv **out)
{
    if (!out) return PK_ERR_INVALID_ARG;
    *out = nullptr;
    if (!valid(cfg) || !arena || (reinterpret_cast<uintptr_t>(arena) & 255)) return PK_ERR_INVALID_ARG;
    if (arena_bytes < pk_kv_arena_bytes(cfg)) return PK_ERR_NOMEM;
    pk_kv *kv = new (std::nothrow) pk_kv();
    if (!kv) return PK_ERR_NOMEM;
    kv->cfg = *cfg;
    kv->dp = padded(cfg->head_dim);
    lay_out(*cfg, static_cast<char *>(arena), &kv->dev);
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess || hipDeviceGetAttribute(&kv->num_cu, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) {
        (void)hipGetLastError();
        delete kv;
        return PK_ERR_HIP;
    }
    void *p = nullptr;
    const size_t parts = (size_t)(kKvPartFloats + kKvPartFloats / kv->dp * 3) * sizeof(float);
    if (hipMalloc(&p, parts + kKvArrivals * sizeof(uint32_t)) != hipSuccess) {
        (void)hipGetLastError();
        delete kv;
        return PK_ERR_NOMEM;
    }
    kv->ws = static_cast<char *>(p);
    // (a blocking clear, done before any stream's work can reach it)
    if (hipMemset(kv->ws + parts, 0, kKvArrivals * sizeof(uint32_t)) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
        (void)hipGetLastError();
        (void)hipFree(p);
        delete kv;
        return PK_ERR_HIP;
    }
    kv->magic = kKvMagic;
    *out = kv;
    return PK_OK;
}

int pk_kv_free(pk_kv *kv)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    kv->magic = 0;
    const bool ok = hipFree(kv->ws) == hipSuccess;
    delete kv;
    return ok ? PK_OK : PK_ERR_HIP;
}

int pk_kv_append(pk_kv *kv, const pk_kv_batch *batch, const pk_rows *k, const pk_rows *v, void *stream)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    KvBatch b;
    bool none;
    int rc = kv_take_batch(kv, batch, &b, &none);
    if (rc != PK_OK || none) return rc;
    KvRows kr, vr;
    rc = take_rows(k, &kr);
    if (rc == PK_OK) rc = take_rows(v, &vr);
    if (rc != PK_OK) return rc;
    if (k->dtype != v->dtype) return PK_ERR_INVALID_ARG;
    if (kv_touched(kv->dev, b) > kKvMaxTouched) return PK_ERR_UNSUPPORTED;
    return launch_kv_append(kv->dev, kv->cfg.storage, kv->dp, b, kr, vr, k->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_HIP;
}

int pk_kv_read(pk_kv *kv, const pk_kv_batch *batch, void *k_out, void *v_out, int32_t dtype, void *stream)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    KvBatch b;
    bool none;
    const int rc = kv_take_batch(kv, batch, &b, &none);
    if (rc != PK_OK || none) return rc;
    if (!k_out || !v_out || !row_type(dtype) || ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 15)) return PK_ERR_INVALID_ARG;
    if (kv_touched(kv->dev, b) > kKvMaxTouched) return PK_ERR_UNSUPPORTED;
    return launch_kv_read(kv->dev, kv->cfg.storage, kv->dp, b, k_out, v_out, dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_HIP;
}

int pk_kv_bounds(pk_kv *kv, const int32_t *pages, int64_t n, float *hi, float *lo, void *stream)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    if (n < 0 || n > 0x7fffffff) return PK_ERR_INVALID_ARG;
    if (n == 0) return PK_OK;
    if (!pages || !hi || !lo || ((reinterpret_cast<uintptr_t>(hi) | reinterpret_cast<uintptr_t>(lo)) & 15)) return PK_ERR_INVALID_ARG;
    return launch_kv_bounds(kv->dev, kv->dp, pages, n, hi, lo, static_cast<hipStream_t>(stream)) == hipSuccess ? PK_OK : PK_ERR_HIP;
}

int pk_kv_attend(pk_kv *kv, const pk_kv_batch *batch, const pk_rows *q, int32_t n_q_heads, float scale, int32_t window, void *out, float *lse,
                 void *stream)
{
    return attend(kv, batch, q, n_q_heads, scale, window, nullptr, 0, nullptr, out, lse, static_cast<hipStream_t>(stream));
}

int pk_kv_attend_scored(pk_kv *kv, const pk_kv_batch *batch, const pk_rows *q, int32_t n_q_heads, float scale, int32_t window,
                        const pk_kv_scores *scores, void *out, float *lse, void *stream)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    if (!scores) return PK_ERR_INVALID_ARG;
    return attend(kv, batch, q, n_q_heads, scale, window, nullptr, 0, scores, out, lse, static_cast<hipStream_t>(stream));
}

int pk_kv_attend_blocks(pk_kv *kv, const pk_kv_batch *batch, const pk_rows *q, int32_t n_q_heads, float scale, const int32_t *blocks,
                        int32_t n_blocks, void *out, float *lse, void *stream)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    if (n_blocks < 1 || n_blocks > kKvMaxSelect) return PK_ERR_INVALID_ARG;
    if (!blocks && batch && batch->n_tokens > 0) return PK_ERR_INVALID_ARG;
    static const int32_t nothing = 0;
    return attend(kv, batch, q, n_q_heads, scale, 0, blocks ? blocks : &nothing, n_blocks, nullptr, out, lse, static_cast<hipStream_t>(stream));
}

int pk_kv_select(pk_kv *kv, const pk_kv_batch *batch, const pk_rows *q, int32_t n_q_heads, int32_t n_blocks, int32_t sink, int32_t local,
                 int32_t *out_blocks, void *stream)
{
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    KvBatch b;
    bool none;
    int rc = kv_take_batch(kv, batch, &b, &none);
    if (rc != PK_OK) return rc;
    if (n_blocks < 1 || sink < 0 || local < 1 || (int64_t)sink + local > n_blocks) return PK_ERR_INVALID_ARG;
    if (n_blocks > kKvMaxSelect || (!none && (std::min<int64_t>(b.max_len, (int64_t)b.cols * kv->cfg.page_tokens) + kv->cfg.page_tokens - 1) / kv->cfg.page_tokens > kKvMaxSelect))
        return PK_ERR_UNSUPPORTED;
    if (none) return PK_OK;
    KvRows qr;
    int G;
    rc = take_queries(kv, q, n_q_heads, &qr, &G);
    if (rc != PK_OK) return rc;
    if (!out_blocks) return PK_ERR_INVALID_ARG;
    if (kv_select_workgroups(kv->dev, b, G) > kKvMaxGroups) return PK_ERR_UNSUPPORTED;
    return launch_kv_select(kv->dev, kv->dp, b, qr, q->dtype, G, n_blocks, sink, local, kv->num_cu, out_blocks, static_cast<hipStream_t>(stream)) == hipSuccess
               ? PK_OK
               : PK_ERR_HIP;
}

} // extern "C"
