// Paged key/value cache: what its kernels and its host side share (gfx950 only).
#pragma once

#include <algorithm>

#include "pk_internal.h"

namespace pk {

// ------------------------------------------------------------------ layout
// Regions of the arena, each [pages][heads] of one page's
//   k, v [P / 16]    runs of 16 tokens, DP channels each (zero padded from D), in the order in which a wave's lanes take them as a
//                    product's operands, 16 bytes a lane.  Neighbouring lanes have to have neighbouring bytes: a load whose lanes
//                    lie 16 bytes each in rows of their own is 64 accesses of the first cache, not 16, and bound by them (sparse
//                    attention of 1024 tokens to 32 blocks each of int8: 1.0 of 1.1 million cycles).
//                    Keys: groups of four tokens, their rows' 16-byte pieces side by side [4][DP * bytes / 16][4 tokens][16 bytes].
//                    Values: 16 bytes of one channel, 16 or 8 tokens, the channels side by side [1 or 2][DP][16 bytes].
//                    4 bits: a key's piece is 32 channels, the even one of two in the lower half of a byte; values: 16 tokens of channel
//                    32 q + c, then the same of 32 q + 16 + c, [DP / 32 q][16 c][2][8 bytes], the even token in the lower half.
//   ks, vs [P]       scales of keys and values (coded storages)
//   ke  [P / 16]     4 bits: 127 - e of every token and 32 channels of its key, whose codes stand for 2^-e of what they else would:
//                    [DP / 32][4 t][4 i] for token 4 i + t of the 16, so that a lane has its four tokens' side by side
//   bc  [2][DP]      bounds of the keys (largest, smallest value of each channel) in int8, zero padded
//   bs  [1]          their scale
struct KvDev {
    char *k, *v;
    float *ks, *vs;
    uint8_t *ke;
    int8_t *bc;
    float *bs;
    uint32_t n_pages;
    int32_t H, D, P, logP;
};

template <int S> constexpr bool kv_coded = S == PK_I8 || S == PK_F8 || S == PK_F4;
template <int S> constexpr float kv_largest = S == PK_F8 ? 448.f : S == PK_F4 ? 6.f : 127.f;
template <int S> constexpr int kv_bits = S == PK_F4 ? 4 : S == PK_I8 || S == PK_F8 ? 8 : 16;

// Where byte `at` of a token's key lies in its page and head, of RB bytes a row.
template <int RB>
__device__ __forceinline__ int k_place(int tok, int at)
{
    return (tok >> 2) * (RB * 4) + (at >> 4) * 64 + (tok & 3) * 16 + (at & 15);
}
// Where the power of two of a token's key lies, for channels 32 group and on.
template <int DP>
__device__ __forceinline__ int e_place(int tok, int group)
{
    return ((tok >> 4) * (DP / 32) + group) * 16 + (tok & 3) * 4 + (tok >> 2 & 3);
}

// One call's batch, as the kernels get it.
struct KvBatch {
    const int32_t *tables, *offsets, *lens;
    int32_t n_seqs, n_tokens, max_new, max_len, cols;
    int64_t table_stride;
};

struct KvRows {
    const char *data;
    int64_t token_stride, head_stride; // in elements
};

// Rows of one sequence in a batch.  Whatever the arrays hold, what comes out lies in the bounds that the host was told.
struct KvSeq {
    int32_t first; // its first new token among the batch's
    int32_t m;     // new tokens
    int32_t len;   // tokens in the cache, the new ones included
};
__device__ __forceinline__ KvSeq kv_seq(const KvBatch &b, int s, int P)
{
    KvSeq q;
    const int o0 = min(max(b.offsets[s], 0), b.n_tokens), o1 = min(max(b.offsets[s + 1], o0), b.n_tokens);
    q.first = o0;
    q.m = min(o1 - o0, b.max_new);
    const long long most = min((long long)b.max_len, (long long)b.cols * P);
    q.len = (int32_t)min((long long)max(b.lens[s], 0), most);
    return q;
}

// The sequence that token t of a batch belongs to (the last one whose offset is not beyond t).
__device__ __forceinline__ int kv_seq_of(const KvBatch &b, int t)
{
    int lo = 0, hi = b.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (b.offsets[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Physical page of a position; n_pages and more: the table has none there.
__device__ __forceinline__ uint32_t kv_page(const KvDev &c, const int32_t *table, int32_t pos)
{
    return (uint32_t)table[pos >> c.logP];
}

// ------------------------------------------------------------------ elements
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Rows of the caller's may begin at any element.
struct __attribute__((packed, aligned(2))) AnyEight16 {
    u32x4 v;
};
struct __attribute__((packed, aligned(2))) AnyFour16 {
    u32x2 v;
};
struct __attribute__((packed, aligned(4))) AnyFour32 {
    f32x4 v;
};

// Eight consecutive elements of a row of type T as floats.
template <int T>
__device__ __forceinline__ void load_eight(float (&x)[8], const char *row, int at)
{
    if constexpr (T == PK_F32) {
        const f32x4 a = reinterpret_cast<const AnyFour32 *>(row + (size_t)at * 4)->v;
        const f32x4 b = reinterpret_cast<const AnyFour32 *>(row + (size_t)at * 4 + 16)->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[i + 4] = b[i];
        }
    } else {
        const u32x4 w = reinterpret_cast<const AnyEight16 *>(row + (size_t)at * 2)->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (T == PK_BF16) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                const half2v h = __builtin_bit_cast(half2v, (uint32_t)w[i]);
                x[2 * i] = (float)h[0];
                x[2 * i + 1] = (float)h[1];
            }
        }
    }
}

// Four of them.
template <int T>
__device__ __forceinline__ void load_four(float (&x)[4], const char *row, int at)
{
    if constexpr (T == PK_F32) {
        const f32x4 a = reinterpret_cast<const AnyFour32 *>(row + (size_t)at * 4)->v;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i];
    } else {
        const u32x2 w = reinterpret_cast<const AnyFour16 *>(row + (size_t)at * 2)->v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (T == PK_BF16) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                const half2v h = __builtin_bit_cast(half2v, (uint32_t)w[i]);
                x[2 * i] = (float)h[0];
                x[2 * i + 1] = (float)h[1];
            }
        }
    }
}

// Two floats as 16-bit elements of type T, rounded to nearest even.
template <int T>
__device__ __forceinline__ uint32_t pack16(float a, float b)
{
    if constexpr (T == PK_BF16) {
        const bf2 r = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, r);
    } else {
        const half2v r = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, r);
    }
}

// int8 codes are held so that little turns them into operands: the matrix cores take denormal numbers as what they are, and a byte u in
// the lower half of 16 bits is the number u times the type's smallest (2^-24, 2^-133).  Keys are held with 128 added, which a
// product's start value takes back (-128 times the sum of the query, whole numbers of that unit: nothing is lost but what 32 bits round);
// one byte permutation makes two operands.  Values are held as sign and magnitude, as an element that all heavy keys have as zero
// has to come out of the sum as what the others make of it; a permutation and a mask make two operands, the sign bit in its place.
// e4m3 codes have an instruction of their own.
template <int S, int T> constexpr float kv_smallest = S != PK_I8 ? 1.f : T == PK_F16 ? 0x1p-24f : 0x1p-133f;

// Four codes of keys, or of values, as four elements of type T, times the type's smallest number if S is PK_I8.
template <int S, int T, bool VALUES>
__device__ __forceinline__ void codes_to(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    if constexpr (S == PK_I8 && VALUES) {
        lo = __builtin_amdgcn_perm(w, w, 0x01010000u) & 0x807f807fu;
        hi = __builtin_amdgcn_perm(w, w, 0x03030202u) & 0x807f807fu;
    } else if constexpr (S == PK_I8) {
        lo = __builtin_amdgcn_perm(w, w, 0x0c010c00u);
        hi = __builtin_amdgcn_perm(w, w, 0x0c030c02u);
    } else if constexpr (T == PK_F16) {
        lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
        hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true));
    } else {
        lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
        hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
    }
}

// Eight e2m1 codes of 4 bits as elements of type T, times `scale`, a power of two: exact, as a code has two bits and both types have
// 2^-15 of the smallest.
template <int T>
__device__ __forceinline__ u32x4 eight_of_4(uint32_t w, float scale)
{
    if constexpr (T == PK_F16)
        return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3))};
    else
        return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}

// 2^-e of a byte 127 - e.
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// One code of a key, or of a value, as the number that it stands for (before its scale).
template <int S, bool VALUES>
__device__ __forceinline__ float code_value(uint8_t c)
{
    if constexpr (S == PK_F4) return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)c, 1.f, 0)[0];
    else if constexpr (S == PK_I8 && VALUES) return (float)(c & 0x80 ? -(int)(c & 0x7f) : (int)c);
    else if constexpr (S == PK_I8) return (float)((int)c - 128);
    else {
        const half2v h = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)c, 1.f, false));
        return (float)h[0];
    }
}

// What turns a row whose largest magnitude is `most` into codes; none of it for a row of zeros.  The division is rounded
// correctly, so that the codes are the same wherever they are computed.
__device__ __forceinline__ float code_factor(float most, float largest)
{
    return most > 0.f ? fminf(largest / most, 3.0e38f) : 0.f;
}

template <int S, bool VALUES>
__device__ __forceinline__ uint8_t to_code(float x, float up)
{
    const float y = fminf(fmaxf(x * up, -kv_largest<S>), kv_largest<S>);
    if constexpr (S == PK_I8) {
        const int code = (int)rintf(y);
        return (uint8_t)(!VALUES ? code + 128 : code < 0 ? 0x80 - code : code);
    }
    return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false);
}

// ------------------------------------------------------------------ launches
struct KvAttend {
    KvDev c;
    KvBatch b;
    KvRows q;
    int32_t G;            // query heads of one key/value head
    float scale;
    int32_t window;       // 0: none
    const int32_t *blocks; // sparse: [n_tokens][H][n_blocks], else null
    int32_t n_blocks;
    int32_t scored;       // the next four are looked at
    float cap;            // 0: none
    const float *slopes;  // [H * G] or null
    const int32_t *starts; // [n_tokens] or null
    const int32_t *prefix; // [n_seqs] or null
    char *out;            // [n_tokens][H * G][D]
    float *lse;           // [n_tokens][H * G] or null
    float *part, *part_ml, *part_q; // room for partial results: part_floats of O, two floats for each row of them (maximum and sum), one for
                                    // each row that has parts (the scores' scale)
    int64_t part_floats;
    uint32_t *arrivals;    // parts of a row tile that have ended, zeros between calls: kKvArrivals of them
    int32_t num_cu;
    // set by the launch
    int32_t few_rows;      // sequences with more rows of queries than this (kKvFewRows at most; 0 where it runs alone) are taken by the kernel for many
    int32_t row_tiles;     // of one sequence (sparse: of one token)
    int32_t part_row;      // floats of a row of partial results
    int32_t join_here;     // the kernel for few rows joins its parts itself
    int32_t n_split, split_tiles; // parts that the keys are cut into, and tiles of 64 keys of each
};

hipError_t launch_kv_append(const KvDev &c, int storage, int dp, const KvBatch &b, const KvRows &k, const KvRows &v, int dtype, hipStream_t s);
hipError_t launch_kv_read(const KvDev &c, int storage, int dp, const KvBatch &b, void *k, void *v, int dtype, hipStream_t s);
hipError_t launch_kv_bounds(const KvDev &c, int dp, const int32_t *pages, int64_t n, float *hi, float *lo, hipStream_t s);
hipError_t launch_kv_select(const KvDev &c, int dp, const KvBatch &b, const KvRows &q, int dtype, int G, int n_blocks, int sink, int local,
                            int num_cu, int32_t *out, hipStream_t s);
int64_t kv_select_workgroups(const KvDev &c, const KvBatch &b, int G); // of that launch, of 256 threads at least
hipError_t launch_kv_attend(const KvAttend &a, int storage, int dp, int dtype, hipStream_t s);

// ------------------------------------------------------------------ host side
constexpr uint64_t kKvMagic = 0x70616e63616b7631ull;
constexpr int64_t kKvMaxGroups = (1 << 24) - 1; // workgroups of 256 threads of a launch (of 512: half as many): a grid has 32 bits for its threads
constexpr int kKvMaxTouched = 1 << 23;    // pages of one sequence that a call writes or reads: the same
constexpr int64_t kKvMaxTokens = 1 << 30; // of a sequence: positions and what is added to them fit 32 bits

constexpr int kKvTile = 64;          // keys of one step of the attention kernels
constexpr int kKvFewRows = 128;      // rows of queries of a sequence and head that the kernel for few takes at most
constexpr int64_t kKvPartFloats = 16 << 20; // partial results that a cache's workspace has room for: 512 workgroups' of 256 rows of 128 channels
constexpr int kKvArrivals = 4096;
constexpr int kKvMaxPage = 128;
constexpr int kKvMaxSelect = 32768;  // blocks that one query chooses from: their keys lie in LDS

// bytes of a token's key (or value) of one head, dp channels
inline size_t kv_row_bytes(int storage, int dp) { return (size_t)dp * (storage == PK_F4 ? 4 : storage == PK_I8 || storage == PK_F8 ? 8 : 16) / 8; }
inline bool kv_is_coded(int storage) { return storage == PK_I8 || storage == PK_F8 || storage == PK_F4; }

// pages that one sequence's new tokens can touch
inline int kv_touched(const KvDev &c, const KvBatch &b)
{
    const int64_t pages = ((int64_t)b.max_new + c.P - 2) / c.P + 1;
    return (int)(pages < b.cols ? pages : b.cols);
}

} // namespace pk

struct pk_kv {
    uint64_t magic;
    pk_kv_config cfg;
    int dp;
    pk::KvDev dev;
    int num_cu;
    char *ws; // partial results of split attention
};

namespace pk {

inline bool kv_live(const pk_kv *kv) { return kv && kv->magic == kKvMagic; }

// The batch as the kernels get it.  *none: there is nothing to do.
inline int kv_take_batch(const pk_kv *kv, const pk_kv_batch *b, KvBatch *o, bool *none)
{
    if (!b || b->n_seqs < 0 || b->n_tokens < 0 || b->max_new < 0 || b->max_len < 0 || b->n_cols < 0) return PK_ERR_INVALID_ARG;
    if (b->max_new > b->n_tokens) return PK_ERR_INVALID_ARG;
    if (b->n_seqs > PK_KV_MAX_SEQS) return PK_ERR_UNSUPPORTED;
    *none = b->n_seqs == 0 || b->n_tokens == 0 || b->max_new == 0;
    if (*none) return b->n_tokens > 0 ? PK_ERR_INVALID_ARG : PK_OK; // tokens of no sequence
    if (!b->tables || !b->offsets || !b->lens || b->n_cols < 1 || b->table_stride < b->n_cols || b->max_len < 1) return PK_ERR_INVALID_ARG;
    if (std::min<int64_t>(b->max_len, (int64_t)b->n_cols * kv->cfg.page_tokens) > kKvMaxTokens) return PK_ERR_UNSUPPORTED;
    *o = KvBatch{b->tables, b->offsets, b->lens, b->n_seqs, b->n_tokens, b->max_new, b->max_len, b->n_cols, b->table_stride};
    return PK_OK;
}

} // namespace pk
