// Pages of a key/value cache: who has them, which are free, giving them to sequences, sharing, copying and moving them.
// See include/pancake.h for the contract.  Integer work on tables and counts; pages themselves move at the rate of a copy.
// Every result is a function of the inputs alone: counts are sums, pages are handed out by rank (the lowest free ones in the order
// of sequences and positions), and no order of atomics decides anything.
#include <algorithm>
#include <new>

#include "pk_kv.h"

namespace pk {
namespace {

constexpr int kThreads = 256;
constexpr int kGrantThreads = 1024; // of the one workgroup that hands out pages
constexpr int64_t kMaxPageGroups = 1 << 20; // workgroups that copy pages of a list or a cache, in turns where there are more pages

struct KvPool {
    uint32_t n_pages, n_words;
    int32_t *refs;          // [n_pages] table entries that hold the page
    int32_t *users, *last;  // [n_pages] of a call: sequences that write into a shared page, and the last one plus 1; zeros between calls
    int32_t *list;          // [n_pages] free pages that a call hands out
    uint32_t *bits;         // [n_words] free pages, 32 a word (beyond n_pages: 0)
    int32_t *rank;          // [n_words] of a call: pages in use before a word's
    int32_t *base, *copy_to, *copy_from; // [PK_KV_MAX_SEQS] of a call: entries of the sequences before; the page copied for a sequence, or -1
};

// The regions of an arena, bytes of a page each.
constexpr int kRegions = 7;
struct KvMove {
    char *to[kRegions];
    const char *from[kRegions];
    uint32_t bytes[kRegions];
    uint32_t to_pages, from_pages;
};

// One page of every region, by `pieces` workgroups.  Reads are asked for four at a time.
__device__ __forceinline__ void copy_page(const KvMove &m, uint32_t dst, uint32_t src, int piece, int pieces)
{
#pragma unroll 1
    for (int r = 0; r < kRegions; ++r) {
        const uint32_t bytes = m.bytes[r];
        char *to = m.to[r] + (size_t)dst * bytes;
        const char *from = m.from[r] + (size_t)src * bytes;
        if (bytes % 16 == 0) {
            const uint32_t n = bytes / 16, step = pieces * kThreads;
            for (uint32_t i = piece * kThreads + threadIdx.x; i < n; i += 4 * step) {
                u32x4 w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i + k * step < n) w[k] = *reinterpret_cast<const u32x4 *>(from + (size_t)(i + k * step) * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i + k * step < n) *reinterpret_cast<u32x4 *>(to + (size_t)(i + k * step) * 16) = w[k];
            }
        } else {
            for (uint32_t i = piece * kThreads + threadIdx.x; i < bytes / 4; i += pieces * kThreads)
                *reinterpret_cast<uint32_t *>(to + (size_t)i * 4) = *reinterpret_cast<const uint32_t *>(from + (size_t)i * 4);
        }
    }
}

__global__ __launch_bounds__(kThreads) void kv_copy_kernel(KvMove m, const int32_t *dst, const int32_t *src, int64_t n)
{
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const uint32_t d = (uint32_t)dst[i], s = (uint32_t)src[i];
        if (d < m.to_pages && s < m.from_pages) copy_page(m, d, s, blockIdx.y, gridDim.y);
    }
}

// One more owner of a page (whose count may have been zero).
__device__ __forceinline__ void take_page(const KvPool &p, uint32_t page)
{
    if (atomicAdd(&p.refs[page], 1) == 0) atomicAnd(&p.bits[page >> 5], ~(1u << (page & 31)));
}
// One owner less; a page that nobody had stays so.
__device__ __forceinline__ void drop_page(const KvPool &p, uint32_t page)
{
    const int was = atomicSub(&p.refs[page], 1);
    if (was == 1) atomicOr(&p.bits[page >> 5], 1u << (page & 31));
    else if (was <= 0) atomicAdd(&p.refs[page], 1);
}

__global__ __launch_bounds__(kThreads) void kv_clear_kernel(KvPool p)
{
    const size_t step = (size_t)gridDim.x * kThreads;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < p.n_pages; i += step) {
        p.refs[i] = p.users[i] = p.last[i] = 0;
        if (i < p.n_words) p.bits[i] = (i + 1) * 32 <= p.n_pages ? ~0u : (1u << (p.n_pages & 31)) - 1;
    }
}

__global__ __launch_bounds__(kThreads) void kv_adopt_kernel(KvPool p, pk_kv_tables t)
{
    for (int64_t row = blockIdx.x; row < t.n_rows; row += gridDim.x)
        for (int j = threadIdx.x; j < t.n_cols; j += kThreads) {
            const uint32_t page = (uint32_t)t.data[row * t.stride + j];
            if (page < p.n_pages) take_page(p, page);
        }
}

__global__ __launch_bounds__(kThreads) void kv_fork_kernel(KvPool p, pk_kv_tables t, const int32_t *lens, const int32_t *from, const int32_t *to, int logP, int P)
{
    const int f = from[blockIdx.x], d = to[blockIdx.x];
    if ((uint32_t)f >= (uint32_t)t.n_rows || (uint32_t)d >= (uint32_t)t.n_rows) return;
    const int pages = (int)(((int64_t)max(lens[f], 0) + P - 1) >> logP);
    for (int j = threadIdx.x; j < t.n_cols; j += kThreads) {
        const uint32_t page = j < pages ? (uint32_t)t.data[f * t.stride + j] : ~0u;
        if (page < p.n_pages) take_page(p, page);
        t.data[d * t.stride + j] = page < p.n_pages ? (int32_t)page : -1;
    }
}

__global__ __launch_bounds__(kThreads) void kv_release_kernel(KvPool p, pk_kv_tables t, const int32_t *rows, const int32_t *keep, int logP, int P)
{
    const int row = rows[blockIdx.x];
    if ((uint32_t)row >= (uint32_t)t.n_rows) return;
    const int64_t kept = keep ? ((int64_t)max(keep[blockIdx.x], 0) + P - 1) >> logP : 0;
    for (int64_t j = kept + threadIdx.x; j < t.n_cols; j += kThreads) {
        // (exchanged: an entry of a row that is listed twice is given up once)
        const uint32_t page = (uint32_t)atomicExch(&t.data[row * t.stride + j], -1);
        if (page < p.n_pages) drop_page(p, page);
    }
}

__global__ __launch_bounds__(kThreads) void kv_counts_kernel(KvPool p, int32_t *out)
{
    const size_t step = (size_t)gridDim.x * kThreads;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < p.n_pages; i += step) out[i] = p.refs[i];
}

// Sum over the threads before this one, and over all; sums: one for each wave.
__device__ __forceinline__ int scan(int v, int *sums, int &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
    }
    __syncthreads(); // (sums may still be read from before)
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    return before + upto - v;
}

// All of the workgroup's writes and atomics are done, for all of its waves: the barrier does not wait for them, each wave waits for its own.  (All are of one
// CU, whose cache they share: no fence, which would write back an L2.)
__device__ __forceinline__ void all_done()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Entries of a sequence's table that a call's tokens go into.
struct KvEntries {
    int begin, first, count; // the first new position; the first entry, and how many
};
__device__ __forceinline__ KvEntries kv_entries(const KvBatch &b, int s, int P, int logP)
{
    const KvSeq q = kv_seq(b, s, P);
    const int begin = max(q.len - q.m, 0), first = begin >> logP;
    return KvEntries{begin, first, q.m > 0 && q.len > 0 ? ((q.len - 1) >> logP) - first + 1 : 0};
}

// The lowest free pages, `need` of them, into list[0 ..), and out of the free ones; how many there are (more than needed may be counted).  1024 words a step, each thread
// one, so that the pages of neighbouring words are listed by as many threads; four steps' words are asked for at once.
struct KvFree {
    uint32_t word[4];
    __device__ __forceinline__ void ask(const KvPool &p, uint32_t w0)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w = w0 + k * kGrantThreads + threadIdx.x;
            word[k] = w < p.n_words ? p.bits[w] : 0;
        }
    }
};
__device__ __forceinline__ int take_free(const KvPool &p, KvFree &f, int need, int32_t *list, int *sums) // (f: asked for from word 0 on)
{
    int have = 0;
    for (uint32_t w0 = 0;;) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (have >= need) return have;
            uint32_t w = f.word[k];
            const uint32_t mine = w0 + k * kGrantThreads + threadIdx.x;
            int total, at = have + scan(__popc(w), sums, total);
            while (w && at < need) {
                list[at++] = (int32_t)(mine * 32 + __ffs(w) - 1);
                w &= w - 1;
            }
            if (w != f.word[k]) p.bits[mine] = w;
            have += total;
        }
        w0 += kGrantThreads * 4;
        if (w0 >= p.n_words) return have;
        f.ask(p, w0);
    }
}

// Pages for a batch's new tokens, by one workgroup, 1024 entries at a time, in the order of sequences and positions:
//   1  entries that hold a page of several owners are counted, and the last sequence with each is noted
//   2  what an entry needs is decided and written in its place (-1: a page; -2 - page: a page instead of that one)
//   3  the lowest free pages, as many as are needed
//   4  entries get theirs by rank; counts, and the list of pages to be copied, which the next launch does
// Everything fits the caches: the time is that of the chains of dependent loads, to which an entry's sequence, found among those before it, adds.
// Measured (with the launch behind it): a prompt of 4096 tokens among 255 decoding sequences 15.1 us, 64 prompts of 8192 69, one of 131072 41.  By sequences, some lanes
// each, with free pages listed by who has their words and fences between the phases: 78, 139, 100.
__global__ __launch_bounds__(kGrantThreads) void kv_grant_kernel(KvPool p, KvBatch b, int P, int logP, int32_t *missing)
{
    __shared__ int sums[kGrantThreads / 64];
    __shared__ int lost; // pages that are not there and would have to hold older tokens
    const int tid = threadIdx.x;
    if (tid == 0) lost = 0;
    int entries = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += kGrantThreads) {
        const int s = s0 + tid, n = s < b.n_seqs ? kv_entries(b, s, P, logP).count : 0;
        int total;
        const int before = scan(n, sums, total);
        if (s < b.n_seqs) {
            p.base[s] = entries + before;
            p.copy_to[s] = -1;
        }
        entries += total;
    }
    all_done();

    struct Entry {
        int s;
        int32_t *at;
        bool older; // its page has tokens from before the call
    };
    auto entry_of = [&](int e) __attribute__((always_inline)) {
        int lo = 0, hi = b.n_seqs - 1; // the last sequence whose entries do not begin beyond e: one that has some
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.base[mid] <= e) lo = mid;
            else hi = mid - 1;
        }
        const KvEntries k = kv_entries(b, lo, P, logP);
        const int j = k.first + (e - p.base[lo]);
        return Entry{lo, const_cast<int32_t *>(b.tables) + (size_t)lo * b.table_stride + j, k.begin > (int64_t)j << logP};
    };

    for (int e = tid; e < entries; e += kGrantThreads) {
        const Entry x = entry_of(e);
        const uint32_t page = (uint32_t)*x.at;
        if (page < p.n_pages && p.refs[page] > 1) {
            atomicAdd(&p.users[page], 1);
            atomicMax(&p.last[page], x.s + 1);
        }
    }
    all_done();

    int need = 0;
    for (int e0 = 0; e0 < entries; e0 += kGrantThreads) {
        bool wants = false;
        if (e0 + tid < entries) {
            const Entry x = entry_of(e0 + tid);
            const uint32_t page = (uint32_t)*x.at;
            if (page < p.n_pages) {
                // (written by other waves: read where their atomics wrote)
                const int refs = p.refs[page], users = __hip_atomic_load(&p.users[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                          last = __hip_atomic_load(&p.last[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                wants = refs > 1 && (users < refs || last != x.s + 1);
                if (wants) *x.at = -2 - (int32_t)page;
            } else {
                wants = !x.older;
                if (!wants) atomicAdd(&lost, 1);
                *x.at = -1;
            }
        }
        int total;
        scan(wants ? 1 : 0, sums, total);
        need += total;
    }

    KvFree free;
    free.ask(p, 0);
    const int have = take_free(p, free, need, p.list, sums);
    all_done();

    int given = 0;
    for (int e0 = 0; e0 < entries; e0 += kGrantThreads) {
        const bool inside = e0 + tid < entries;
        Entry x{};
        int32_t entry = 0;
        if (inside) {
            x = entry_of(e0 + tid);
            entry = *x.at; // (as this thread left it)
        }
        const bool wants = inside && (entry < -1 || (entry == -1 && !x.older));
        int total;
        const int rank = given + scan(wants ? 1 : 0, sums, total);
        given += total;
        if (!inside) continue;
        const int32_t old = entry < -1 ? -2 - entry : entry;
        if (old >= 0) p.users[old] = p.last[old] = 0;
        if (!wants) continue;
        const int32_t page = rank < have ? p.list[rank] : -1;
        *x.at = page;
        if (entry < -1) atomicSub(&p.refs[old], 1); // (it keeps one owner at least)
        if (page < 0) continue;
        p.refs[page] = 1;
        if (entry < -1 && x.older) { // (a sequence's first entry alone)
            p.copy_from[x.s] = old;
            p.copy_to[x.s] = page;
        }
    }
    if (tid == 0 && missing) *missing = max(need - have, 0) + lost;
}

// The same where every entry has a thread of its own (a decoding step): entries, owners and what is decided stay in registers, the first free pages
// (of 131072) are asked for at the start, and their list lies in LDS.  Measured: 256 branches, four of each shared page, 7.1 us; four of one sequence 5.7 (13.4).
__global__ __launch_bounds__(kGrantThreads) void kv_grant_once_kernel(KvPool p, KvBatch b, int P, int logP, int W, int32_t *missing)
{
    __shared__ int sums[kGrantThreads / 64];
    __shared__ int32_t list[kGrantThreads];
    __shared__ int lost;
    const int tid = threadIdx.x, in = tid & (W - 1), s = tid / W;
    KvFree free;
    free.ask(p, 0);
    if (tid == 0) lost = 0;
    int32_t *entry = nullptr;
    uint32_t page = 0;
    bool inside = false, older = false;
    int refs = 0;
    if (s < b.n_seqs) {
        const KvEntries k = kv_entries(b, s, P, logP);
        const int j = k.first + in;
        inside = in < k.count;
        older = k.begin > (int64_t)j << logP; // the page has tokens from before the call
        if (inside) {
            entry = const_cast<int32_t *>(b.tables) + (size_t)s * b.table_stride + j;
            page = (uint32_t)*entry;
            if (page < p.n_pages) {
                refs = p.refs[page];
                if (refs > 1) {
                    atomicAdd(&p.users[page], 1);
                    atomicMax(&p.last[page], s + 1);
                }
            }
        }
    }
    const bool there = inside && page < p.n_pages, shared = there && refs > 1;
    bool wants = inside && !there && !older;
    all_done();
    if (inside && !there && older) atomicAdd(&lost, 1);
    if (shared) {
        // (where the other waves' atomics wrote, not in this CU's cache)
        const int users = __hip_atomic_load(&p.users[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), last = __hip_atomic_load(&p.last[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wants = users < refs || last != s + 1;
    }
    int need;
    const int rank = scan(wants ? 1 : 0, sums, need);
    if (shared) p.users[page] = p.last[page] = 0; // (all have read them: the scan is past)

    const int have = take_free(p, free, need, list, sums);
    __syncthreads();
    if (wants || (inside && !there)) {
        const int32_t mine = wants && rank < have ? list[rank] : -1;
        *entry = mine;
        if (shared) atomicSub(&p.refs[page], 1); // (it keeps one owner at least)
        if (mine >= 0) p.refs[mine] = 1;
        if (shared && older && mine >= 0) p.copy_from[s] = (int32_t)page;
        if (in == 0) p.copy_to[s] = shared && older ? mine : -1; // (older tokens lie in a sequence's first entry alone)
    } else if (in == 0 && s < b.n_seqs) p.copy_to[s] = -1;
    if (tid == 0 && missing) *missing = max(need - have, 0) + lost;
}

__global__ __launch_bounds__(kThreads) void kv_granted_copy_kernel(KvPool p, KvMove m)
{
    const int32_t to = p.copy_to[blockIdx.x];
    if (to >= 0) copy_page(m, (uint32_t)to, (uint32_t)p.copy_from[blockIdx.x], blockIdx.y, gridDim.y);
}

__device__ __forceinline__ uint32_t in_use(const KvPool &p, uint32_t word)
{
    const uint32_t there = (word + 1) * 32ull <= p.n_pages ? ~0u : (1u << (p.n_pages & 31)) - 1;
    return ~p.bits[word] & there;
}

// Pages in use before each word's, by one workgroup, 131072 pages a step: 13000 pages 4.7 us (32 words a thread, fewer steps for many pages: 10.3).
__global__ __launch_bounds__(kGrantThreads) void kv_rank_kernel(KvPool from, KvPool to, int32_t *missing)
{
    __shared__ int sums[kGrantThreads / 64];
    constexpr int EACH = 4;
    int upto = 0;
    for (uint32_t w0 = 0; w0 < from.n_words; w0 += kGrantThreads * EACH) {
        const uint32_t first = w0 + threadIdx.x * EACH;
        int n[EACH], all = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            n[k] = first + k < from.n_words ? __popc(in_use(from, first + k)) : 0;
            all += n[k];
        }
        int total, at = upto + scan(all, sums, total);
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            if (first + k < from.n_words) from.rank[first + k] = at;
            at += n[k];
        }
        upto += total;
    }
    if (threadIdx.x == 0) {
        from.base[0] = upto;
        if (missing) *missing = max(upto - (int)min(to.n_pages, 0x7fffffffu), 0);
    }
}

// The number among the pages in use; -1 for a page that is not.
__device__ __forceinline__ int32_t rank_of(const KvPool &p, uint32_t page)
{
    if (page >= p.n_pages) return -1;
    const uint32_t w = in_use(p, page >> 5), bit = 1u << (page & 31);
    return w & bit ? p.rank[page >> 5] + __popc(w & (bit - 1)) : -1;
}

__global__ __launch_bounds__(kThreads) void kv_rename_kernel(KvPool from, KvPool to, pk_kv_tables in, pk_kv_tables out)
{
    const size_t step = (size_t)gridDim.x * kThreads, me = (size_t)blockIdx.x * kThreads + threadIdx.x;
    for (size_t i = me; i < (size_t)in.n_rows * in.n_cols; i += step) {
        const size_t row = i / in.n_cols, col = i % in.n_cols;
        const int32_t name = rank_of(from, (uint32_t)in.data[row * in.stride + col]);
        out.data[row * out.stride + col] = (uint32_t)name < to.n_pages ? name : -1;
    }
    const uint32_t used = min((uint32_t)from.base[0], to.n_pages);
    for (size_t i = me; i < to.n_pages; i += step) {
        if (i >= used) to.refs[i] = 0;
        to.users[i] = to.last[i] = 0;
        if (i < to.n_words) {
            const uint32_t there = (i + 1) * 32 <= to.n_pages ? ~0u : (1u << (to.n_pages & 31)) - 1;
            to.bits[i] = there & (i * 32 >= used ? ~0u : used - i * 32 >= 32 ? 0u : ~((1u << (used & 31)) - 1));
        }
    }
}

__global__ __launch_bounds__(kThreads) void kv_move_kernel(KvPool from, KvPool to, KvMove m)
{
    for (uint32_t page = blockIdx.x; page < from.n_pages; page += gridDim.x) {
        const int32_t name = rank_of(from, page);
        if ((uint32_t)name >= to.n_pages) continue;
        copy_page(m, (uint32_t)name, page, blockIdx.y, gridDim.y);
        if (threadIdx.x == 0 && blockIdx.y == 0) to.refs[name] = from.refs[page];
    }
}

} // namespace
} // namespace pk

// ------------------------------------------------------------------ host side

using namespace pk;

struct pk_kv_pool {
    uint64_t magic;
    pk_kv kv; // (the cache's numbers as they are; its handle may go first)
    KvPool dev;
};

namespace {

constexpr uint64_t kPoolMagic = 0x70616e63706f6f6cull;

bool live(const pk_kv_pool *p) { return p && p->magic == kPoolMagic; }

// Regions of the pool's memory; base may be null (sizes only).
size_t lay_out(int64_t n_pages, char *base, KvPool *p)
{
    const size_t n = (size_t)n_pages, words = (n + 31) / 32;
    size_t off = 0;
    auto take = [&](size_t count) {
        char *at = base ? base + off : nullptr;
        off += (count * 4 + 255) / 256 * 256;
        return reinterpret_cast<int32_t *>(at);
    };
    p->n_pages = (uint32_t)n;
    p->n_words = (uint32_t)words;
    p->refs = take(n);
    p->users = take(n);
    p->last = take(n);
    p->list = take(n);
    p->bits = reinterpret_cast<uint32_t *>(take(words));
    p->rank = take(words);
    p->base = take(PK_KV_MAX_SEQS);
    p->copy_to = take(PK_KV_MAX_SEQS);
    p->copy_from = take(PK_KV_MAX_SEQS);
    return off;
}

KvMove move_between(const pk_kv &to, const pk_kv &from)
{
    const size_t H = from.cfg.n_heads, P = from.cfg.page_tokens, dp = from.dp, row = kv_row_bytes(from.cfg.storage, from.dp);
    const size_t scales = kv_is_coded(from.cfg.storage) ? H * P * sizeof(float) : 0, powers = from.cfg.storage == PK_F4 ? H * P * (dp / 32) : 0;
    const size_t bytes[kRegions] = {H * P * row, H * P * row, scales, scales, powers, H * 2 * dp, H * sizeof(float)};
    auto regions = [](const KvDev &c, char *(&r)[kRegions]) {
        char *all[kRegions] = {c.k, c.v, reinterpret_cast<char *>(c.ks), reinterpret_cast<char *>(c.vs), reinterpret_cast<char *>(c.ke), reinterpret_cast<char *>(c.bc), reinterpret_cast<char *>(c.bs)};
        std::copy(all, all + kRegions, r);
    };
    KvMove m{};
    char *source[kRegions];
    regions(to.dev, m.to);
    regions(from.dev, source);
    for (int i = 0; i < kRegions; ++i) m.from[i] = source[i], m.bytes[i] = (uint32_t)bytes[i];
    m.to_pages = to.dev.n_pages;
    m.from_pages = from.dev.n_pages;
    return m;
}

// Caches whose pages are alike.
bool alike(const pk_kv_config &a, const pk_kv_config &b)
{
    return a.n_heads == b.n_heads && a.head_dim == b.head_dim && a.page_tokens == b.page_tokens && a.storage == b.storage;
}

// Workgroups that share a page, so that a few pages have the chip: of about 16 KB of it each where there are many pages.
int pieces_of(const KvMove &m, int64_t pages, int num_cu)
{
    size_t bytes = 0;
    for (uint32_t x : m.bytes) bytes += x;
    const int64_t most = std::max<int64_t>((int64_t)(bytes / (8 << 10)), 1), wanted = std::max<int64_t>(8 * (int64_t)num_cu / std::max<int64_t>(pages, 1), 1);
    return (int)std::min(most, wanted);
}

bool valid(const pk_kv_tables *t, bool *none)
{
    if (!t || t->n_rows < 0 || t->n_cols < 0) return false;
    *none = t->n_rows == 0 || t->n_cols == 0;
    return *none || (t->data && t->stride >= t->n_cols);
}

int done() { return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_HIP; }

unsigned threads_for(size_t n, int num_cu) { return (unsigned)std::max<size_t>(std::min<size_t>((n + kThreads - 1) / kThreads, (size_t)num_cu * 8), 1); }

void clear(const pk_kv_pool *pool, hipStream_t s)
{
    kv_clear_kernel<<<threads_for(pool->dev.n_pages, pool->kv.num_cu), kThreads, 0, s>>>(pool->dev);
}

} // namespace

extern "C" {

size_t pk_kv_pool_bytes(const pk_kv_config *cfg)
{
    KvPool p;
    return pk_kv_arena_bytes(cfg) ? lay_out(cfg->n_pages, nullptr, &p) : 0;
}

int pk_kv_pool_create(pk_kv *kv, void *memory, size_t bytes, pk_kv_pool **out)
{
    if (!out) return PK_ERR_INVALID_ARG;
    *out = nullptr;
    if (!kv_live(kv)) return PK_ERR_BAD_HANDLE;
    if (!memory || (reinterpret_cast<uintptr_t>(memory) & 255)) return PK_ERR_INVALID_ARG;
    if (bytes < pk_kv_pool_bytes(&kv->cfg)) return PK_ERR_NOMEM;
    pk_kv_pool *pool = new (std::nothrow) pk_kv_pool();
    if (!pool) return PK_ERR_NOMEM;
    pool->kv = *kv;
    lay_out(kv->cfg.n_pages, static_cast<char *>(memory), &pool->dev);
    clear(pool, nullptr);
    if (done() != PK_OK || hipDeviceSynchronize() != hipSuccess) {
        (void)hipGetLastError();
        delete pool;
        return PK_ERR_HIP;
    }
    pool->magic = kPoolMagic;
    *out = pool;
    return PK_OK;
}

int pk_kv_pool_free(pk_kv_pool *pool)
{
    if (!live(pool)) return PK_ERR_BAD_HANDLE;
    pool->magic = 0;
    delete pool;
    return PK_OK;
}

int pk_kv_pool_clear(pk_kv_pool *pool, void *stream)
{
    if (!live(pool)) return PK_ERR_BAD_HANDLE;
    clear(pool, static_cast<hipStream_t>(stream));
    return done();
}

int pk_kv_pool_adopt(pk_kv_pool *pool, const pk_kv_tables *tables, void *stream)
{
    if (!live(pool)) return PK_ERR_BAD_HANDLE;
    bool none;
    if (!valid(tables, &none)) return PK_ERR_INVALID_ARG;
    if (none) return PK_OK;
    kv_adopt_kernel<<<(unsigned)std::min<int64_t>(tables->n_rows, kMaxPageGroups), kThreads, 0, static_cast<hipStream_t>(stream)>>>(pool->dev, *tables);
    return done();
}

int pk_kv_pool_grant(pk_kv_pool *pool, const pk_kv_batch *batch, int32_t *missing, void *stream)
{
    if (!live(pool)) return PK_ERR_BAD_HANDLE;
    KvBatch b{};
    bool none;
    const int rc = kv_take_batch(&pool->kv, batch, &b, &none);
    if (rc != PK_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (none) b.n_seqs = 0; // (the number of missing pages is written all the same)
    const int entries = none ? 1 : kv_touched(pool->kv.dev, b); // of a sequence at most
    int W = 1;
    while (W < 64 && W < entries) W *= 2;
    if (entries <= W && (int64_t)b.n_seqs * W <= kGrantThreads) kv_grant_once_kernel<<<1, kGrantThreads, 0, s>>>(pool->dev, b, pool->kv.dev.P, pool->kv.dev.logP, W, missing);
    else kv_grant_kernel<<<1, kGrantThreads, 0, s>>>(pool->dev, b, pool->kv.dev.P, pool->kv.dev.logP, missing);
    if (!none) {
        const KvMove m = move_between(pool->kv, pool->kv);
        kv_granted_copy_kernel<<<dim3(b.n_seqs, pieces_of(m, b.n_seqs, pool->kv.num_cu)), kThreads, 0, s>>>(pool->dev, m);
    }
    return done();
}

int pk_kv_pool_fork(pk_kv_pool *pool, const pk_kv_tables *tables, const int32_t *lens, const int32_t *from, const int32_t *to, int32_t n, void *stream)
{
    if (!live(pool)) return PK_ERR_BAD_HANDLE;
    bool none;
    if (!valid(tables, &none) || n < 0 || (n > 0 && (!lens || !from || !to))) return PK_ERR_INVALID_ARG;
    if (n > kKvMaxGroups) return PK_ERR_UNSUPPORTED;
    if (none || n == 0) return PK_OK;
    kv_fork_kernel<<<n, kThreads, 0, static_cast<hipStream_t>(stream)>>>(pool->dev, *tables, lens, from, to, pool->kv.dev.logP, pool->kv.dev.P);
    return done();
}

int pk_kv_pool_release(pk_kv_pool *pool, const pk_kv_tables *tables, const int32_t *rows, const int32_t *keep, int32_t n, void *stream)
{
    if (!live(pool)) return PK_ERR_BAD_HANDLE;
    bool none;
    if (!valid(tables, &none) || n < 0 || (n > 0 && !rows)) return PK_ERR_INVALID_ARG;
    if (n > kKvMaxGroups) return PK_ERR_UNSUPPORTED;
    if (none || n == 0) return PK_OK;
    kv_release_kernel<<<n, kThreads, 0, static_cast<hipStream_t>(stream)>>>(pool->dev, *tables, rows, keep, pool->kv.dev.logP, pool->kv.dev.P);
    return done();
}

int pk_kv_pool_compact(pk_kv_pool *from, pk_kv_pool *to, const pk_kv_tables *tables, const pk_kv_tables *out, int32_t *missing, void *stream)
{
    if (!live(from) || !live(to)) return PK_ERR_BAD_HANDLE;
    bool none, out_none;
    if (from == to || !valid(tables, &none) || !valid(out, &out_none)) return PK_ERR_INVALID_ARG;
    if (tables->n_rows != out->n_rows || tables->n_cols != out->n_cols || from->kv.dev.k == to->kv.dev.k) return PK_ERR_INVALID_ARG;
    if (!alike(from->kv.cfg, to->kv.cfg)) return PK_ERR_DIM_MISMATCH;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int cu = from->kv.num_cu;
    kv_rank_kernel<<<1, kGrantThreads, 0, s>>>(from->dev, to->dev, missing);
    const size_t entries = (size_t)tables->n_rows * tables->n_cols;
    kv_rename_kernel<<<threads_for(std::max<size_t>(entries, to->dev.n_pages), cu), kThreads, 0, s>>>(from->dev, to->dev, *tables, *out);
    const KvMove m = move_between(to->kv, from->kv);
    const int64_t pages = from->dev.n_pages;
    kv_move_kernel<<<dim3((unsigned)std::min(pages, kMaxPageGroups), pieces_of(m, pages, cu)), kThreads, 0, s>>>(from->dev, to->dev, m);
    return done();
}

int pk_kv_pool_counts(pk_kv_pool *pool, int32_t *counts, void *stream)
{
    if (!live(pool)) return PK_ERR_BAD_HANDLE;
    if (!counts) return PK_ERR_INVALID_ARG;
    kv_counts_kernel<<<threads_for(pool->dev.n_pages, pool->kv.num_cu), kThreads, 0, static_cast<hipStream_t>(stream)>>>(pool->dev, counts);
    return done();
}

int pk_kv_copy(pk_kv *to, pk_kv *from, const int32_t *to_pages, const int32_t *from_pages, int64_t n, void *stream)
{
    if (!kv_live(to) || !kv_live(from)) return PK_ERR_BAD_HANDLE;
    if (n < 0 || n > 0x7fffffff || (n > 0 && (!to_pages || !from_pages))) return PK_ERR_INVALID_ARG;
    if (!alike(to->cfg, from->cfg)) return PK_ERR_DIM_MISMATCH;
    if (n == 0) return PK_OK;
    const KvMove m = move_between(*to, *from);
    kv_copy_kernel<<<dim3((unsigned)std::min(n, kMaxPageGroups), pieces_of(m, n, from->num_cu)), kThreads, 0, static_cast<hipStream_t>(stream)>>>(m, to_pages, from_pages, n);
    return done();
}

} // extern "C"
