// Which blocks of a sequence a query attends to: the ones whose bounds promise the largest scores.
#include "pk_kv.h"

namespace pk {
namespace {

constexpr int kThreads = 256;

// The scores' order as whole numbers: larger is better; 0 is for blocks that cannot be chosen.
__device__ __forceinline__ uint32_t score_key(float v)
{
    const uint32_t b = __float_as_uint(v);
    return max(b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u), 1u);
}

// One workgroup: one token, one key/value head.
//   U[block, head] = sum_c max(q_c hi_c, q_c lo_c) = q+ hi + q- lo, whole numbers: int8 products of the rows [hi, lo] of the bounds with
//   [q+, q-] of the group's queries, 16 blocks by 16 heads at a time
//   score[block] = max over the group's heads of U scale_q, times the bounds' scale
// No sum of it is rounded, so the choice is the same whatever computes it.  The keys of the scores stay in LDS; the n-th largest is
// found by its four bytes, one histogram each, and what is chosen comes out in ascending order.
template <int T, int DP>
__global__ __launch_bounds__(kThreads) void kv_select_kernel(KvDev c, KvBatch b, KvRows qin, int G, int n, int sink, int local, int32_t *out)
{
    extern __shared__ uint32_t keys[];
    __shared__ uint32_t hist[256];
    __shared__ uint32_t found[3], waves[4];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g = lane >> 4;
    const int t = blockIdx.x, h = blockIdx.y;
    const int seq = kv_seq_of(b, t);
    const KvSeq sq = kv_seq(b, seq, c.P);
    const int i = t - sq.first, pos = sq.len - sq.m + i;
    int32_t *o = out + ((size_t)t * c.H + h) * n;
    const bool none = i < 0 || i >= sq.m || pos < 0;
    const int mine = none ? -1 : pos >> c.logP, nb = mine + 1;
    const int32_t *table = b.tables + (size_t)seq * b.table_stride;
    for (int i0 = tid; i0 < nb; i0 += kThreads) keys[i0] = 0;
    __syncthreads();

    constexpr int KS = DP / 64; // products over a half of a row of bounds
    for (int gt = 0; gt < G; gt += 16) {
        // the queries' codes: lane (head, g) has channels 64 k + 16 g .. + 15
        float x[KS][16], most = 0.f;
        const bool there = gt + col < G;
        const char *qrow = qin.data + ((size_t)t * qin.token_stride + (size_t)(h * G + min(gt + col, G - 1)) * qin.head_stride) * 2;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = 0.f;
                const int at = k * 64 + g * 16 + e;
                if (there && at < c.D) load_eight<T>(y, qrow, at);
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
        for (int b0 = wave * 16; b0 < nb; b0 += 64) {
            const int blk = min(b0 + col, nb - 1);
            const uint32_t page = (uint32_t)table[blk];
            const size_t ph = (size_t)(page < c.n_pages ? page : 0) * c.H + h;
            const int8_t *row = c.bc + ph * 2 * DP + g * 16;
            i32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(row + k * 64), qp[k], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(row + DP + k * 64), qm[k], acc, 0, 0, 0);
            }
            const float bs = c.bs[ph];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v = there ? (float)acc[j] * qscale : -INFINITY;
#pragma unroll
                for (int d = 1; d < 16; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
                const int at = b0 + g * 4 + j; // its scale and page are with the lane of that column
                const float scale = __shfl(bs, g * 4 + j);
                const uint32_t pg = (uint32_t)__shfl((int)page, g * 4 + j);
                if (col == 0 && at < nb && pg < c.n_pages) {
                    const uint32_t key = at < sink || at > mine - local ? 0xffffffffu : score_key(v * scale + 0.f); // (no zero of a sign)
                    keys[at] = max(keys[at], key);
                }
            }
        }
    }
    __syncthreads();

    // the n-th largest key, byte by byte; `need` of the keys equal to it are chosen, the lowest blocks first
    uint32_t prefix = 0, mask = 0, need = (uint32_t)n;
    bool all = false;
    for (int shift = 24; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int i0 = tid; i0 < nb; i0 += kThreads)
            if (keys[i0] && (keys[i0] & mask) == prefix) atomicAdd(&hist[(keys[i0] >> shift) & 255u], 1u);
        __syncthreads();
        // how many lie in bins above this thread's
        uint32_t own = hist[tid], above = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t v = (uint32_t)__shfl_down((int)above, d);
            if (lane + d < 64) above += v;
        }
        if (lane == 0) waves[wave] = above;
        if (tid == 0) found[0] = 0xffffffffu;
        __syncthreads();
        for (int w = wave + 1; w < 4; ++w) above += waves[w];
        above -= own;
        if (above < need && above + own >= need) {
            found[0] = (uint32_t)tid;
            found[1] = need - above;
        }
        __syncthreads();
        if (found[0] == 0xffffffffu) { // fewer than n in all (only in the first round)
            all = true;
            break;
        }
        prefix |= found[0] << shift;
        mask |= 255u << shift;
        need = found[1];
        __syncthreads();
    }
    uint32_t done = 0, equal = 0;
    for (int i0 = 0; i0 < nb; i0 += kThreads) {
        const uint32_t key = i0 + tid < nb ? keys[i0 + tid] : 0;
        const bool is = key && !all && key == prefix, over = key && (all || key > prefix);
        // ranks among the equal ones, then among the chosen ones
        const unsigned long long eq = __ballot(is);
        if (lane == 0) waves[wave] = (uint32_t)__popcll(eq);
        __syncthreads();
        uint32_t rank = equal + (uint32_t)__popcll(eq & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) rank += waves[w];
        equal += waves[0] + waves[1] + waves[2] + waves[3];
        const bool take = over || (is && rank < need);
        const unsigned long long tk = __ballot(take);
        __syncthreads();
        if (lane == 0) waves[wave] = (uint32_t)__popcll(tk);
        __syncthreads();
        uint32_t place = done + (uint32_t)__popcll(tk & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) place += waves[w];
        done += waves[0] + waves[1] + waves[2] + waves[3];
        if (take && place < (uint32_t)n) o[place] = i0 + tid;
        __syncthreads();
    }
    for (int i0 = (int)done + tid; i0 < n; i0 += kThreads) o[i0] = -1;
}

template <int T, int DP>
hipError_t run(const KvDev &c, const KvBatch &b, const KvRows &q, int G, int n, int sink, int local, int32_t *out, hipStream_t s)
{
    const int64_t keys = ((int64_t)b.max_len + c.P - 1) / c.P;
    const size_t lds = (size_t)(keys < b.cols ? keys : b.cols) * sizeof(uint32_t);
    if (lds > (48u << 10)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_select_kernel<T, DP>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kv_select_kernel<T, DP><<<dim3((unsigned)b.n_tokens, c.H), kThreads, lds, s>>>(c, b, q, G, n, sink, local, out);
    return hipGetLastError();
}

} // namespace

hipError_t launch_kv_select(const KvDev &c, int dp, const KvBatch &b, const KvRows &q, int dtype, int G, int n_blocks, int sink, int local,
                            int32_t *out, hipStream_t s)
{
    if (dtype == PK_F16) return dp == 64 ? run<PK_F16, 64>(c, b, q, G, n_blocks, sink, local, out, s) : dp == 128 ? run<PK_F16, 128>(c, b, q, G, n_blocks, sink, local, out, s) : run<PK_F16, 256>(c, b, q, G, n_blocks, sink, local, out, s);
    return dp == 64 ? run<PK_BF16, 64>(c, b, q, G, n_blocks, sink, local, out, s) : dp == 128 ? run<PK_BF16, 128>(c, b, q, G, n_blocks, sink, local, out, s) : run<PK_BF16, 256>(c, b, q, G, n_blocks, sink, local, out, s);
}

} // namespace pk
