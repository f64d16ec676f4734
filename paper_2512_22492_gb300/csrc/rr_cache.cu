// The rollout's key-value cache in pages (fork, extend, append, truncate, compact) and the
// verification of drafted tokens, for GB300 (sm_103a); include/rr.h has the definitions.
#include <algorithm>
#include <climits>

#include "rr_cache.cuh"

namespace {

// ---------------------------------------------------------------------------
// Bookkeeping
// ---------------------------------------------------------------------------
//
// Each of these calls reads short lists and tables and writes some entries: a chain of a
// few dependent loads, whose latency is the cost, so that few launches and few barriers
// are what counts (3 to 6 us a call among others).  One cluster of 1 or 8 blocks does a call; its
// barriers are the hardware's.  Every block checks the whole of the call's lists by itself, and nothing
// is written before all of them have (a call that fails leaves the cache as it was).

constexpr int kBookThreads = 512;
constexpr int kBookWarps = kBookThreads / 32;
constexpr int kBookRanks = 8;

__device__ __forceinline__ int cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return int(r);
}
__device__ __forceinline__ int cluster_size() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return int(r);
}
// Everything that the cluster's threads wrote before is seen by all of them after.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() {
    cluster_arrive();
    cluster_wait();
}

struct Ranks {
    int rank, size;
    __device__ __forceinline__ Ranks() : rank(cluster_rank()), size(cluster_size()) {}
    // This block's part of n things, in order.
    __device__ __forceinline__ int64_t first(int64_t n) const { return n * rank / size; }
    __device__ __forceinline__ int64_t end(int64_t n) const { return n * (rank + 1) / size; }
    // This thread's or warp's number among the cluster's, and how many there are.
    __device__ __forceinline__ int thread() const { return rank * kBookThreads + int(threadIdx.x); }
    __device__ __forceinline__ int threads() const { return size * kBookThreads; }
    __device__ __forceinline__ int warp() const { return rank * kBookWarps + int(threadIdx.x >> 5); }
    __device__ __forceinline__ int warps() const { return size * kBookWarps; }
};

// One bit for each sequence of the cache, in shared memory.
struct Listed {
    uint32_t* bits;
    __device__ __forceinline__ Listed(uint32_t* shared, int max_seqs) : bits(shared) {
        for (int i = threadIdx.x; i < (max_seqs + 31) / 32; i += kBookThreads) bits[i] = 0;
        __syncthreads();
    }
    __device__ __forceinline__ bool add(int s) { return atomicOr(&bits[s >> 5], 1u << (s & 31)) >> (s & 31) & 1; }
    __device__ __forceinline__ bool has(int s) const { return bits[s >> 5] >> (s & 31) & 1; }
};

// The block's OR of bad, the same in all of its threads.
__device__ __forceinline__ int agree(int bad) {
    __shared__ int all;
    if (threadIdx.x == 0) all = 0;
    __syncthreads();
    bad = __reduce_or_sync(~0u, bad);
    if (bad && (threadIdx.x & 31) == 0) atomicOr(&all, bad);
    __syncthreads();
    const int r = all;
    __syncthreads();
    return r;
}

// Exclusive sum of v over the block's threads; *total: of all of them.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* total) {
    __shared__ int64_t part[kBookWarps];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int64_t s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(~0u, s, d);
        if (lane >= d) s += o;
    }
    if (lane == 31) part[w] = s;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kBookWarps; ++i) {
        if (i < w) before += part[i];
        all += part[i];
    }
    __syncthreads();
    *total = all;
    return before + s - v;
}

// Sums over the cluster's blocks of what each has counted, and put into b.sums[k * kBookRanks +
// rank] before a barrier (a block alone need not): of the ranks before this one, and of all.
__device__ __forceinline__ int64_t rank_sum(const Book& b, const Ranks& r, int k, int64_t mine, int64_t* total) {
    if (r.size == 1) {
        *total = mine;
        return 0;
    }
    int64_t before = 0, all = 0;
    for (int i = 0; i < r.size; ++i) {
        const int64_t v = __ldcg(&b.sums[k * kBookRanks + i]);
        if (i < r.rank) before += v;
        all += v;
    }
    *total = all;
    return before;
}

// Four pages' holders from page p on (a multiple of 4); pages from `end` on count as held.
__device__ __forceinline__ int4 four(const int32_t* refs, int64_t p, int64_t end) {
    int4 v = make_int4(1, 1, 1, 1);
    if (p + 3 < end) return __ldcg(reinterpret_cast<const int4*>(refs + p));
    if (p < end) v.x = __ldcg(refs + p);
    if (p + 1 < end) v.y = __ldcg(refs + p + 1);
    if (p + 2 < end) v.z = __ldcg(refs + p + 2);
    return v;
}
__device__ __forceinline__ int zeros(const int4& v) { return (v.x == 0) + (v.y == 0) + (v.z == 0) + (v.w == 0); }

// A rank's pages: whole fours, so that vectors stay aligned.
struct Pages {
    int64_t first, end;
    __device__ __forceinline__ Pages(const Ranks& r, int n_pages) {
        const int64_t fours = (int64_t(n_pages) + 3) / 4;
        first = r.first(fours) * 4;
        end = min(r.end(fours) * 4, int64_t(n_pages));
    }
    // Free pages among them.
    __device__ __forceinline__ int64_t free(const int32_t* refs) const {
        int n = 0;
#pragma unroll 4
        for (int64_t p = first + 4 * int64_t(threadIdx.x); p < end; p += 4 * kBookThreads) n += zeros(four(refs, p, end));
        int64_t all;
        block_scan(n, &all);
        return all;
    }
};

__device__ __forceinline__ int32_t pages_of(int32_t tokens, int shift) {
    return int32_t((int64_t(tokens) + (1 << shift) - 1) >> shift);
}

// Ends a call that cannot be done; all of its blocks come here.
__device__ __forceinline__ void fail(const Book& b, const Ranks& r, int bad) {
    if (r.rank == 0 && threadIdx.x == 0) atomicOr(&b.control[kState], bad);
}

extern __shared__ uint32_t shared_bits[];

__global__ void __launch_bounds__(kBookThreads) rr_cache_fork_kernel(const __grid_constant__ CacheShape c, const Book b,
                                                                     const int32_t* parents, const int32_t* children, int n) {
    after_previous();
    const Ranks r;
    Listed listed(shared_bits, c.max_seqs);
    int bad = __ldcg(&b.control[kState]) | __ldcg(&b.control[kLate]);
    for (int i = threadIdx.x; i < n; i += kBookThreads) {
        const int p = parents[i], s = children[i];
        if (!c.has_seq(p) || !c.has_seq(s)) {
            bad |= kBadRange;
            continue;
        }
        if (listed.add(s)) bad |= kBadTwice;
        if (__ldcg(&b.lengths[s]) != 0) bad |= kBadChild;
        if (!c.has_length(__ldcg(&b.lengths[p]))) bad |= kBadRange;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kBookThreads)
        if (c.has_seq(parents[i]) && listed.has(parents[i])) bad |= kBadTwice;
    bad = agree(bad);
    // A warp takes 128 entries of one parent's row.  All of them are looked at before any is
    // written (0.3 us; of a parent listed several times in a row once); those of a warp's first task
    // (there are others only in long calls) stay in its registers.
    constexpr int kEach = 128;
    const int lane = threadIdx.x & 31;
    const int chunks = (c.max_pages + kEach - 1) / kEach;
    struct Task {
        int s, length, first, end;
        int32_t id[kEach / 32];
    };
    const auto task_of = [&](int64_t task) {
        Task t;
        const int i = int(task / chunks), p = parents[i];
        t.first = int(task % chunks) * kEach;
        t.s = children[i];
        t.length = __ldcg(&b.lengths[p]);
        t.end = min(pages_of(t.length, c.shift), t.first + kEach);
#pragma unroll
        for (int k = 0; k < kEach / 32; ++k) {
            const int j = t.first + lane + 32 * k;
            t.id[k] = j < t.end ? __ldcg(&b.table[int64_t(p) * c.max_pages + j]) : -1;
        }
        return t;
    };
    const int64_t tasks = bad ? 0 : int64_t(n) * chunks;
    Task kept = {};
    bool found = false;
    for (int64_t task = r.warp(); task < tasks; task += r.warps()) {
        const int i = int(task / chunks);
        if (task != r.warp() && i && parents[i] == parents[i - 1]) continue;
        const Task t = task_of(task);
        if (task == r.warp()) kept = t;
#pragma unroll
        for (int k = 0; k < kEach / 32; ++k) found |= t.first + lane + 32 * k < t.end && !c.has_page(t.id[k]);
    }
    if (found) atomicOr(&b.control[kState], kBadTable);
    cluster_barrier();
    if (bad || __ldcg(&b.control[kState])) return fail(b, r, bad);
    for (int64_t task = r.warp(); task < tasks; task += r.warps()) {
        const Task t = task == r.warp() ? kept : task_of(task);
        if (t.first == 0 && lane == 0) b.lengths[t.s] = t.length;
#pragma unroll
        for (int k = 0; k < kEach / 32; ++k) {
            const int j = t.first + lane + 32 * k;
            if (j >= t.end) continue;
            b.table[int64_t(t.s) * c.max_pages + j] = t.id[k];
            atomicAdd(&b.refs[t.id[k]], 1);
        }
    }
}

__device__ __forceinline__ int64_t new_tokens(const int32_t* starts, int i) { return starts ? int64_t(starts[i + 1]) - starts[i] : 1; }

// A listed sequence's next tokens: where they begin, and the page that is partly filled.
struct Growth {
    int s = 0, length = 0, count = 0, filled = 0;
    int32_t page = -1;   // partly filled (-1: none, or no tokens come)
    int32_t holders = 0; // of that page
    int64_t entry = 0;   // its place in the table
    __device__ __forceinline__ Growth() {}
    __device__ __forceinline__ Growth(const CacheShape& c, const Book& b, const int32_t* seqs, const int32_t* starts, int i) {
        s = seqs[i];
        count = int(new_tokens(starts, i));
        length = __ldcg(&b.lengths[s]);
        filled = length & (c.page - 1);
        entry = int64_t(s) * c.max_pages + (length >> c.shift);
        page = filled && count ? __ldcg(&b.table[entry]) : -1;
        if (!c.has_page(page)) page = -1;
        if (page >= 0) holders = __ldcg(&b.refs[page]);
    }
    __device__ __forceinline__ int grown(const CacheShape& c) const {
        return pages_of(length + count, c.shift) - pages_of(length, c.shift);
    }
};

__global__ void __launch_bounds__(kBookThreads) rr_cache_extend_kernel(const __grid_constant__ CacheShape c, const Book b,
                                                                       const int32_t* seqs, const int32_t* starts, int n) {
    after_previous();
    const Ranks r;
    Listed listed(shared_bits, c.max_seqs);
    int bad = __ldcg(&b.control[kState]) | __ldcg(&b.control[kLate]);
    for (int i = threadIdx.x; i < n; i += kBookThreads) {
        const int s = seqs[i];
        const int64_t count = new_tokens(starts, i);
        if (!c.has_seq(s)) {
            bad |= kBadRange;
            continue;
        }
        if (listed.add(s)) bad |= kBadTwice;
        const int length = __ldcg(&b.lengths[s]);
        if (!c.has_length(length) || count < 0) bad |= kBadRange;
        else if (length + count > c.max_length()) bad |= kBadPool;
        else if (count && (length & (c.page - 1)) && !c.has_page(__ldcg(&b.table[int64_t(s) * c.max_pages + (length >> c.shift)])))
            bad |= kBadTable;
    }
    bad = agree(bad);
    if (r.rank == 0 && threadIdx.x == 0) b.control[kMoves] = 0;
    const int lo = int(r.first(n)), hi = int(r.end(n));
    // A thread's first sequence stays in its registers; there are others only in long lists.
    const auto growth_of = [&](int base, const Growth& kept) {
        const int i = base + int(threadIdx.x);
        return base == lo || i >= hi ? kept : Growth(c, b, seqs, starts, i);
    };
    Growth kept;
    if (!bad && lo + int(threadIdx.x) < hi) kept = Growth(c, b, seqs, starts, lo + int(threadIdx.x));
    // Who holds each shared page that is partly filled, among the listed ones.
    for (int base = lo; !bad && base < hi; base += kBookThreads) {
        const int i = base + int(threadIdx.x);
        const Growth g = growth_of(base, kept);
        if (i < hi && g.page >= 0 && g.holders > 1) {
            atomicAdd(&b.held[g.page], 1);
            atomicMax(&b.last[g.page], i + 1);
        }
    }
    const Pages mine(r, c.n_pages);
    const int64_t free = bad ? 0 : mine.free(b.refs);
    cluster_barrier();
    if (bad) return fail(b, r, bad);
    // A copy for each holder, but for the last where all of them are listed; then whole
    // pages.  b.plan: the sequence's place among the pages to be taken, and whether a copy is.
    int64_t needed = 0;
    for (int base = lo; base < hi; base += kBookThreads) {
        const int i = base + int(threadIdx.x);
        const Growth g = growth_of(base, kept);
        int need = 0, copy = 0;
        if (i < hi) {
            if (g.page >= 0 && g.holders > 1) copy = !(__ldcg(&b.held[g.page]) == g.holders && __ldcg(&b.last[g.page]) == i + 1);
            need = copy + g.grown(c);
        }
        int64_t total;
        const int64_t at = needed + block_scan(need, &total);
        // (A place past the pool's end only in a call that fails.)
        if (i < hi) b.plan[i] = int32_t(min(at, int64_t(INT_MAX / 2))) * 2 + copy;
        needed += total;
    }
    if (threadIdx.x == 0) {
        b.sums[r.rank] = needed;
        b.sums[kBookRanks + r.rank] = free;
    }
    cluster_barrier();
    int64_t all_needed, all_free;
    const int64_t needed_before = rank_sum(b, r, 0, needed, &all_needed);
    int64_t k = rank_sum(b, r, 1, free, &all_free);
    if (all_needed > all_free) bad = kBadPool;
    // The lowest free pages, in order.
    if (!bad) {
        for (int64_t base = mine.first; base < mine.end && k < all_needed; base += 4 * kBookThreads) {
            const int64_t p = base + 4 * int64_t(threadIdx.x);
            const int4 v = four(b.refs, p, mine.end);
            int64_t total, at = k + block_scan(zeros(v), &total);
            if (v.x == 0 && at < all_needed) b.free[at++] = int32_t(p);
            if (v.y == 0 && at < all_needed) b.free[at++] = int32_t(p + 1);
            if (v.z == 0 && at < all_needed) b.free[at++] = int32_t(p + 2);
            if (v.w == 0 && at < all_needed) b.free[at++] = int32_t(p + 3);
            k += total;
        }
    }
    cluster_barrier();
    const int lane = threadIdx.x & 31;
    for (int base = lo; base < hi; base += kBookThreads) {
        const int i = base + int(threadIdx.x);
        Growth g = growth_of(base, kept);
        if (i >= hi) g.page = -1, g.count = 0;
        if (g.page >= 0 && g.holders > 1) b.held[g.page] = b.last[g.page] = 0;
        if (bad) continue;
        const int plan = i < hi ? b.plan[i] : 0, copy = plan & 1;
        int64_t at = needed_before + (plan >> 1);
        if (copy) {
            const int to = __ldcg(&b.free[at]);
            b.table[g.entry] = to;
            b.refs[to] = 1;
            atomicSub(&b.refs[g.page], 1);
            b.moves[atomicAdd(&b.control[kMoves], 1)] = make_int4(g.page, to, g.filled, 0);
        }
        at += copy;
        if (i < hi) b.lengths[g.s] = g.length + g.count;
        // New pages: of a sequence that takes many, by its warp.
        const int grown = i < hi ? g.grown(c) : 0;
        int64_t entry = i < hi ? int64_t(g.s) * c.max_pages + pages_of(g.length, c.shift) : 0;
        for (int j = 0; j < min(grown, 2); ++j) {
            const int to = __ldcg(&b.free[at + j]);
            b.table[entry + j] = to;
            b.refs[to] = 1;
        }
        for (uint32_t many = __ballot_sync(~0u, grown > 2); many; many &= many - 1) {
            const int x = __ffs(many) - 1, n = __shfl_sync(~0u, grown, x);
            const int64_t from = __shfl_sync(~0u, at, x), into = __shfl_sync(~0u, entry, x);
            for (int j = 2 + lane; j < n; j += 32) {
                const int to = __ldcg(&b.free[from + j]);
                b.table[into + j] = to;
                b.refs[to] = 1;
            }
        }
    }
    if (bad) fail(b, r, bad);
}

// The filled tokens of the pages that rr_cache_extend_kernel took copies of.  A run is
// a layer's keys or values of one head, `filled` rows of `pitch`; a block takes 16 runs of a
// page, two a warp.  (42 copies of 1.2 MB, from and to L2: 15 us, 6.6 TB/s.)
constexpr int kRuns = 16;
__global__ void __launch_bounds__(256) rr_cache_copy_rows_kernel(const __grid_constant__ CacheShape c, const Book b, char* pages) {
    after_previous();
    if (__ldcg(&b.control[kState])) return;
    const int moves = __ldcg(&b.control[kMoves]);
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int vecs_row = c.pitch / 8;
    const unsigned parts = unsigned(c.runs + kRuns - 1) / kRuns;
    for (uint64_t task = blockIdx.x; task < uint64_t(moves) * parts; task += gridDim.x) {
        const unsigned move = task >> 32 ? unsigned(task / parts) : unsigned(task) / parts;
        const int run = int(task - uint64_t(move) * parts) * kRuns + 2 * w;
        if (run >= c.runs) continue;
        const bool second = run + 1 < c.runs;
        const int4 m = __ldcg(&b.moves[move]);
        const int64_t step = c.run_bytes / 16;
        const uint4* from = reinterpret_cast<const uint4*>(pages + m.x * c.page_bytes + run * c.run_bytes);
        uint4* to = reinterpret_cast<uint4*>(pages + m.y * c.page_bytes + run * c.run_bytes);
        const int vecs = m.z * vecs_row;
        for (int i = lane; i < vecs; i += 128) {
            uint4 u[4], v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + 32 * k < vecs) {
                    u[k] = from[i + 32 * k];
                    if (second) v[k] = from[step + i + 32 * k];
                }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + 32 * k < vecs) {
                    to[i + 32 * k] = u[k];
                    if (second) to[step + i + 32 * k] = v[k];
                }
        }
    }
}

__global__ void __launch_bounds__(kBookThreads) rr_cache_truncate_kernel(const __grid_constant__ CacheShape c, const Book b,
                                                                         const int32_t* seqs, const int32_t* drop, int n) {
    after_previous();
    const Ranks r;
    Listed listed(shared_bits, c.max_seqs);
    int bad = __ldcg(&b.control[kState]) | __ldcg(&b.control[kLate]);
    for (int i = threadIdx.x; i < n; i += kBookThreads) {
        const int s = seqs[i];
        if (!c.has_seq(s)) {
            bad |= kBadRange;
            continue;
        }
        if (listed.add(s)) bad |= kBadTwice;
        const int length = __ldcg(&b.lengths[s]);
        if (!c.has_length(length) || (drop && (drop[i] < 0 || drop[i] > length))) bad |= kBadRange;
    }
    bad = agree(bad);
    const int lane = threadIdx.x & 31;
    // The pages are looked at before any is given up (0.6 us).
    bool found = false;
    for (int i = r.warp(); !bad && i < n; i += r.warps()) {
        const int s = seqs[i], length = __ldcg(&b.lengths[s]), left = drop ? length - drop[i] : 0;
        const int32_t* const row = b.table + int64_t(s) * c.max_pages;
#pragma unroll 4
        for (int j = pages_of(left, c.shift) + lane; j < pages_of(length, c.shift); j += 32) found |= !c.has_page(__ldcg(&row[j]));
    }
    if (found) atomicOr(&b.control[kState], kBadTable);
    cluster_barrier();
    if (bad || __ldcg(&b.control[kState])) return fail(b, r, bad);
    for (int i = r.warp(); i < n; i += r.warps()) {
        const int s = seqs[i], length = __ldcg(&b.lengths[s]), left = drop ? length - drop[i] : 0;
        __syncwarp();
        int32_t* const row = b.table + int64_t(s) * c.max_pages;
#pragma unroll 4
        for (int j = pages_of(left, c.shift) + lane; j < pages_of(length, c.shift); j += 32) {
            const int id = row[j];
            row[j] = -1;
            atomicSub(&b.refs[id], 1);
        }
        if (lane == 0) b.lengths[s] = left;
    }
}

// With U(p) the pages in use before page p and U pages in use in all: hole number
// p - U(p) is page p < U that is free, and of the pages p >= U in use, U - 1 - U(p) are
// behind p.  The k-th hole gets the k-th of these pages.
__global__ void __launch_bounds__(kBookThreads) rr_cache_compact_kernel(const __grid_constant__ CacheShape c, const Book b) {
    after_previous();
    const Ranks r;
    const int bad = __ldcg(&b.control[kState]) | __ldcg(&b.control[kLate]);
    const Pages mine(r, c.n_pages);
    const int64_t free = mine.free(b.refs);
    if (threadIdx.x == 0) b.sums[r.rank] = mine.end - mine.first - free;
    cluster_barrier();
    if (bad) {
        // (fail() stops the launch that moves pages, too.)
        if (r.rank == 0 && threadIdx.x == 0) b.control[kMoves] = 0;
        return fail(b, r, bad);
    }
    int64_t used;
    int64_t before = rank_sum(b, r, 0, mine.end - mine.first - free, &used);
    int64_t holes = 0;
    for (int64_t base = mine.first; base < mine.end; base += 4 * kBookThreads) {
        const int64_t p = base + 4 * int64_t(threadIdx.x);
        const int4 v = four(b.refs, p, mine.end);
        const int refs[4] = {v.x, v.y, v.z, v.w};
        const int n = int(max(min(mine.end - p, int64_t(4)), int64_t(0)));
        int64_t total, u = before + block_scan(n - zeros(v), &total);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= n) continue;
            if (refs[k]) {
                if (p + k >= used) b.moves[used - 1 - u].w = int32_t(p + k);
                ++u;
            } else if (p + k < used) {
                b.moves[p + k - u].y = int32_t(p + k);
                ++holes;
            }
        }
        before += total;
    }
    block_scan(holes, &holes);
    if (threadIdx.x == 0) b.sums[kBookRanks + r.rank] = holes;
    cluster_barrier();
    int64_t moves;
    rank_sum(b, r, 1, holes, &moves);
    if (r.rank == 0 && threadIdx.x == 0) {
        b.control[kMoves] = int32_t(moves);
        b.control[kUsed] = int32_t(used);
    }
    for (int64_t k = r.thread(); k < moves; k += r.threads()) {
        const int from = __ldcg(&b.moves[moves - 1 - k].w), to = __ldcg(&b.moves[k].y);
        b.moves[k].x = from;
        b.free[from] = to;
        b.refs[to] = __ldcg(&b.refs[from]);
        b.refs[from] = 0;
    }
}

// The moved pages' contents and their places in the table.  One thread of a block (one an SM)
// has 32 KiB at a time copied through shared memory by bulk copies, four of them on their
// way in while two are on theirs out; its other warps see to the table.  (Loads and
// stores by all threads, 64 bytes of each in flight: 304 MB in 58 us, 5.2 TB/s; so 44 to 45, 6.8.)
constexpr int kMoveChunk = 32768, kMoveStages = 6, kMoveAhead = 4;
__global__ void __launch_bounds__(256) rr_cache_move_kernel(const __grid_constant__ CacheShape c, const Book b, char* pages) {
    extern __shared__ __align__(128) char stages[];
    __shared__ uint64_t full[kMoveStages];
    after_previous();
    if (__ldcg(&b.control[kState])) return;
    const int moves = __ldcg(&b.control[kMoves]), used = __ldcg(&b.control[kUsed]);
    if (!moves) return;
    if (threadIdx.x == 0) {
        const auto smem = [](const void* p) { return uint32_t(__cvta_generic_to_shared(p)); };
        for (int i = 0; i < kMoveStages; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem(&full[i])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        const int64_t chunks = (c.page_bytes + kMoveChunk - 1) / kMoveChunk, all = moves * chunks;
        const int n = int(all > blockIdx.x ? (all - blockIdx.x + gridDim.x - 1) / gridDim.x : 0);
        int4 move = make_int4(0, 0, 0, 0);
        int64_t out[kMoveStages];
        int bytes[kMoveStages];
        // (Unrolled by stage, so that out and bytes are registers.)
        bool ok = true;
        int asked = 0, landed = 0;
        for (int base = 0; ok && base < n + kMoveAhead; base += kMoveStages) {
#pragma unroll
            for (int s = 0; s < kMoveStages; ++s) {
                const int i = base + s;
                if (ok && i < n) {
                    // The stage's last copy out has been read.
                    if (i >= kMoveStages) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kMoveStages - kMoveAhead - 1) : "memory");
                    const int64_t task = blockIdx.x + int64_t(i) * gridDim.x, m = task / chunks, at = (task - m * chunks) * kMoveChunk;
                    move = __ldcg(&b.moves[m]);
                    bytes[s] = int(min(c.page_bytes - at, int64_t(kMoveChunk)));
                    out[s] = move.y * c.page_bytes + at;
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem(&full[s])), "r"(bytes[s]) : "memory");
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                                     smem(stages + s * kMoveChunk)),
                                 "l"(pages + move.x * c.page_bytes + at), "r"(bytes[s]), "r"(smem(&full[s]))
                                 : "memory");
                    asked = i + 1;
                }
                constexpr int kBack = kMoveStages - kMoveAhead;
                const int j = i - kMoveAhead, from = (s + kBack) % kMoveStages;
                if (ok && j >= 0 && j < n) {
                    uint32_t done = 0;
                    const long long t0 = clock64();
                    while (!done) {
                        asm volatile(
                            "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                            : "=r"(done)
                            : "r"(smem(&full[from])), "r"(j / kMoveStages & 1)
                            : "memory");
                        if (!done && clock64() - t0 > 4000000000ll) break;       // two seconds or so
                    }
                    if (!done) {
                        atomicOr(&b.control[kLate], kBadWait);
                        ok = false;
                    } else {
                        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(pages + out[from]),
                                     "r"(smem(stages + from * kMoveChunk)), "r"(bytes[from])
                                     : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        landed = j + 1;
                    }
                }
            }
        }
        // (Of a call that gave up: what is on its way has to land before the block ends; a tenth of a second
        // or so is waited for it at most.)
        const long long t0 = clock64();
        for (int i = landed; !ok && i < asked; ++i) {
            uint32_t done = 0;
            while (!done && clock64() - t0 < 200000000ll)
                asm volatile(
                    "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                    : "=r"(done)
                    : "r"(smem(&full[i % kMoveStages])), "r"(i / kMoveStages & 1)
                    : "memory");
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (threadIdx.x < 32) return;
    const int lane = threadIdx.x & 31;
    for (int s = int(blockIdx.x * 7 + (threadIdx.x >> 5)) - 1; s < c.max_seqs; s += int(gridDim.x) * 7) {
        const int length = __ldcg(&b.lengths[s]);
        if (!c.has_length(length)) continue;
        int32_t* const row = b.table + int64_t(s) * c.max_pages;
        const int n = pages_of(length, c.shift);
#pragma unroll 4
        for (int j = lane; j < n; j += 32) {
            const int id = row[j];
            if (id >= used && id < c.n_pages) row[j] = __ldcg(&b.free[id]);
        }
    }
}

// ---------------------------------------------------------------------------
// New tokens' keys and values
// ---------------------------------------------------------------------------

// A warp takes one token's row: 2 n_kv vectors of `dim` elements, `pitch` in the page.
// VEC: rows can be read 16 bytes at a time.
template <bool VEC>
__device__ __forceinline__ void append_row(const CacheShape& c, const Book& b, char* pages, int layer, const uint16_t* k, int64_t ldk,
                                           const uint16_t* v, int64_t ldv, const int32_t* seqs, const int32_t* starts, int n, int rows,
                                           int row) {
    const int lane = threadIdx.x & 31;
    int i = row, j = 0, count = 1;
    if (starts) {
        // The first sequence that ends behind the row; 32 places looked at at a time.
        int lo = 0, left = n;
        while (left > 0) {
            const int step = (left + 31) / 32, at = lo + min((lane + 1) * step, left);
            const int before = __popc(__ballot_sync(~0u, starts[at] <= row && (lane + 1) * step <= left));
            // (Sequences lo .. lo + before * step - 1 end at or before it.)
            lo += before * step;
            left = min(step - 1, left - before * step);
        }
        i = lo;
        if (i >= n) return;
        const int first = starts[i], end = starts[i + 1];
        // (A sequence whose rows are not all there is left out, below.)
        if (first < 0 || row < first || row >= end || end > rows) return;
        j = row - first;
        count = end - first;
    }
    const int s = seqs[i];
    int length = 0, id = -1, bad = 0;
    if (!c.has_seq(s)) bad = kBadRange;
    else length = __ldcg(&b.lengths[s]);
    const int64_t pos = int64_t(length) - count + j;
    if (!bad && (!c.has_length(length) || pos < 0)) bad = kBadRange;
    if (!bad) id = __ldcg(&b.table[int64_t(s) * c.max_pages + (pos >> c.shift)]);
    if (!bad && !c.has_page(id)) bad = kBadTable;
    if (bad) {
        if (lane == 0) atomicOr(&b.control[kLate], bad);
        return;
    }
    char* const to = pages + id * c.page_bytes + layer * c.layer_bytes + (pos & (c.page - 1)) * (2 * c.pitch);
    const int each = c.pitch / 8, half = c.n_kv * each;
    for (int x = lane; x < 2 * half; x += 32) {
        const int head = x / each, d = (x - head * each) * 8;      // heads of the keys, then of the values
        const bool val = head >= c.n_kv;
        const uint16_t* from = (val ? v + row * ldv + int64_t(head - c.n_kv) * c.dim : k + row * ldk + int64_t(head) * c.dim) + d;
        uint4 u;
        if (VEC) {
            u = *reinterpret_cast<const uint4*>(from);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = d + e < c.dim ? from[e] : 0u;
            u = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
        *reinterpret_cast<uint4*>(to + head * c.run_bytes + 2 * d) = u;
    }
}

template <bool VEC>
__global__ void __launch_bounds__(256) rr_cache_append_kernel(const __grid_constant__ CacheShape c, const Book b, char* pages, int layer,
                                                              const uint16_t* k, int64_t ldk, const uint16_t* v, int64_t ldv,
                                                              const int32_t* seqs, const int32_t* starts, int n, int rows) {
    after_previous();
    if (__ldcg(&b.control[kState])) return;
    const int lane = threadIdx.x & 31, row = int(blockIdx.x * 8 + (threadIdx.x >> 5));
    if (row >= rows) return;
    // What of the lists does not fit is seen by no row, or not by all: the warps look through them
    // together, and have what they look at on its way while the row is written.
    const int64_t from = int64_t(row) * 32 + lane;
    int s = 0, first = 0, end = 0;
    if (starts && from < n) s = seqs[from], first = starts[from], end = starts[from + 1];
    append_row<VEC>(c, b, pages, layer, k, ldk, v, ldv, seqs, starts, n, rows, row);
    const auto check = [&] {
        if (!c.has_seq(s) || first < 0 || end < first || end > rows) atomicOr(&b.control[kLate], kBadRange);
    };
    check();
    for (int64_t i = from + int64_t(rows) * 32; starts && i < n; i += int64_t(rows) * 32) {
        s = seqs[i], first = starts[i], end = starts[i + 1];
        check();
    }
}

// ---------------------------------------------------------------------------
// Drafted tokens
// ---------------------------------------------------------------------------

constexpr int kAcceptRanks = 8;
constexpr int kAcceptThreads = 1024;      // at most
constexpr int kMaxVocab = 1 << 20;

// A probability x in whole numbers of 2^-42, ties to even; NaN counts as 0.  In two parts, in
// float32: h = floor(x 2^22), by adding 2^23 and cutting off, and the rest x 2^42 - h 2^20, which is exact
// and is rounded to a whole number by adding 2^23.  Both stand in the low bits of a float from
// kMagic on.  (Conversions to 64-bit integers run at a fraction of the rate: 64 sequences of 151936
// entries took 52 us with them; mantissas shifted as integers 24 us; so 18 us.)
constexpr uint32_t kMagic = 0x4B000000u;      // 2^23
struct Units {
    uint32_t high, low;       // kMagic + h, kMagic + the rest
    __device__ __forceinline__ Units(float x) {
        x = __saturatef(x);
        const float h = __fadd_rz(x * 4194304.0f, 8388608.0f);
        const float rest = fmaf(h - 8388608.0f, -1048576.0f, x * 4398046511104.0f);
        high = __float_as_uint(h);
        low = __float_as_uint(rest + 8388608.0f);
    }
    __device__ __forceinline__ uint64_t value() const { return (uint64_t(high - kMagic) << 20) + (low - kMagic); }
};

struct AcceptArgs {
    const float *p, *q;
    int64_t ldp, ldq;
    const int32_t *drafts, *starts;
    const float *u, *v;
    int32_t *accepted, *tokens, *rejected;
    int32_t rows, vocab;
};

// What a token is drawn from: the rest (p, less q or without the refused draft), or p.
struct Draw {
    const float *p, *q;       // q NULL: no draft was refused, or it came without probabilities
    int without;              // the refused draft's token, or -1
    bool vec;                 // rows can be read 16 bytes at a time
    // Entries [k, k + 128), up to `end`, four a lane: one after another (ORDER, or vec), or 32 apart.
    template <bool ORDER>
    __device__ __forceinline__ int index(int k, int lane, int e) const { return ORDER || vec ? k + 4 * lane + e : k + lane + 32 * e; }
    template <bool ORDER>
    __device__ __forceinline__ void load(const float* x, int k, int lane, int end, float* to) const {
        const int i = k + 4 * lane;
        if (vec && i + 3 < end) {
            const float4 r = __ldcg(reinterpret_cast<const float4*>(x + i));
            to[0] = r.x, to[1] = r.y, to[2] = r.z, to[3] = r.w;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = index<ORDER>(k, lane, e) < end ? __ldcg(x + index<ORDER>(k, lane, e)) : 0.0f;
    }
    // Of N times 128 entries from k on, the lane's.
    template <bool ORDER, int N>
    __device__ __forceinline__ void values(int k, int lane, int end, float (*x)[4]) const {
        float b[N][4];
#pragma unroll
        for (int h = 0; h < N; ++h) load<ORDER>(p, k + 128 * h, lane, end, x[h]);
        if (q) {
#pragma unroll
            for (int h = 0; h < N; ++h) load<ORDER>(q, k + 128 * h, lane, end, b[h]);
#pragma unroll
            for (int h = 0; h < N; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[h][e] -= b[h][e];
        }
    }
};

// One cluster of 8 blocks takes a sequence.  Its blocks find the accepted drafts each for
// itself; every warp adds up its run of the vocabulary, all sums go to all blocks, and the
// warp whose run holds the drawn number looks through it again.  Sums of whole
// numbers: their order changes nothing.  Reads one row of p, and of q where a draft was
// refused; a chain of starts, drafts, their probabilities, sums and search comes on top (64 sequences
// of 151936 entries: 56 MB, 16.5 us on the GPU, of which HBM takes 8.6; one: 7.8).
__global__ void __launch_bounds__(kAcceptThreads, 1) rr_accept_kernel(const __grid_constant__ AcceptArgs a) {
    __shared__ uint64_t sums[2][kAcceptRanks * kAcceptThreads / 32];
    __shared__ int first_refused;
    // Another block's shared memory may be written once that block runs: waited for before
    // the first sums go there, behind the loads.
    cluster_arrive();
    after_previous();
    const int i = blockIdx.x / kAcceptRanks, rank = cluster_rank();
    const int lane = threadIdx.x & 31, per_block = blockDim.x / 32, w = rank * per_block + int(threadIdx.x >> 5);
    const int all = kAcceptRanks * per_block;
    const int start = a.starts ? a.starts[i] : i, end = a.starts ? a.starts[i + 1] : i + 1;
    const bool fits = start >= 0 && end <= a.rows && end > start;
    const int n = fits ? end - start - 1 : 0;
    if (threadIdx.x == 0) first_refused = n;
    __syncthreads();
    for (int j = threadIdx.x; j < n; j += blockDim.x) {
        const int x = a.drafts[start + j];
        bool ok = x >= 0 && x < a.vocab;
        if (ok) {
            const double own = a.q ? double(a.q[(start + j) * a.ldq + x]) : 1.0;
            ok = double(a.u[start + j]) * own < double(a.p[(start + j) * a.ldp + x]);
        }
        if (!ok) atomicMin(&first_refused, j);
    }
    __syncthreads();
    const int got = first_refused;
    const bool refused = got < n;
    const int64_t row = fits ? start + got : 0;
    Draw d;
    d.p = a.p + row * a.ldp;
    d.q = refused && a.q ? a.q + row * a.ldq : nullptr;
    d.without = refused && !a.q ? a.drafts[row] : -1;
    d.vec = reinterpret_cast<uintptr_t>(d.p) % 16 == 0 && reinterpret_cast<uintptr_t>(d.q) % 16 == 0;
    const int each = (a.vocab + 4 * all - 1) / (4 * all) * 4;
    const int lo = min(w * each, a.vocab), hi = fits ? min(lo + each, a.vocab) : lo;
    // The sums before this warp's run, and of all; twice where all that is left is 0.
    uint64_t before, total, own;
    for (int pass = 0;; ++pass) {
        uint64_t mine = 0;
#pragma unroll 1
        for (int k = lo; k < hi; k += 512) {
            float x[4][4];
            d.values<false, 4>(k, lane, hi, x);
            // (16 of them stay within 32 bits.)
            uint32_t high = 0, low = 0;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Units u(x[h][e]);
                    high += u.high;
                    low += u.low;
                }
            }
            mine += (uint64_t(high - 16 * kMagic) << 20) + (low - 16 * kMagic);
        }
        if (lane == 0 && d.without >= lo && d.without < hi) mine -= Units(d.p[d.without]).value();
#pragma unroll
        for (int m = 16; m; m >>= 1) mine += __shfl_xor_sync(~0u, mine, m);
        if (pass == 0) cluster_wait();
        if (lane < kAcceptRanks) {
            uint32_t at = uint32_t(__cvta_generic_to_shared(&sums[pass][w])), to;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(lane));
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(mine) : "memory");
        }
        cluster_barrier();
        before = total = 0;
        for (int k = lane; k < all; k += 32) {
            total += sums[pass][k];
            if (k < w) before += sums[pass][k];
        }
#pragma unroll
        for (int m = 16; m; m >>= 1) {
            total += __shfl_xor_sync(~0u, total, m);
            before += __shfl_xor_sync(~0u, before, m);
        }
        own = mine;
        // (The same in all of the cluster's threads.)
        if (total || pass || !refused) break;
        d.q = nullptr;
        d.without = -1;
    }
    if (!fits) {
        if (rank == 0 && threadIdx.x == 0) {
            a.accepted[i] = -1;
            if (a.rejected) a.rejected[i] = 0;
        }
        return;
    }
    // The number drawn: floor(total v), v in whole numbers of 2^-31.
    const uint64_t v31 = min(uint64_t(fminf(fmaxf(a.v[i], 0.0f), 1.0f) * 2147483648.0f), uint64_t((1u << 31) - 1));
    const uint64_t t = (total >> 31) * v31 + ((total & ((1u << 31) - 1)) * v31 >> 31);
    if (rank == 0) {
        for (int j = threadIdx.x; j <= n; j += blockDim.x) {
            if (j < got) a.tokens[start + j] = a.drafts[start + j];
            else if (j > got || total == 0) a.tokens[start + j] = -1;
        }
        if (threadIdx.x == 0) {
            a.accepted[i] = got;
            if (a.rejected) a.rejected[i] = n - got;
        }
    }
    if (total == 0 || t < before || t - before >= own) return;
    uint64_t left = t - before;
    bool found = false;
    for (int base = lo; base < hi && !found; base += 512) {
        float y[4][4];
        d.values<true, 4>(base, lane, hi, y);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int k = base + 128 * h + 4 * lane;
            uint64_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = k + e == d.without ? 0 : Units(y[h][e]).value();
            const uint64_t mine = x[0] + x[1] + x[2] + x[3];
            uint64_t up = mine;
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) {
                const uint64_t o = __shfl_up_sync(~0u, up, m);
                if (lane >= m) up += o;
            }
            if (!found && up > left && up - mine <= left) {
                uint64_t rest = left - (up - mine);
                int e = 0;
#pragma unroll
                for (int z = 0; z < 3; ++z)
                    if (e == z && rest >= x[z]) rest -= x[z], ++e;
                a.tokens[row] = k + e;
            }
            const uint64_t last = __shfl_sync(~0u, up, 31);
            found |= last > left;
            left -= last;
        }
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// A launch as one or several clusters, behind the launch before it.
template <class... Params, class... Args>
cudaError_t launch_clusters(void (*kernel)(Params...), int cluster, unsigned grid, int threads, size_t smem, cudaStream_t stream,
                            Args... args) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

size_t bits_bytes(const rr_cache* C) { return size_t(C->max_seqs + 31) / 32 * 4; }

// Blocks that share a call's bookkeeping: one where it has a warp for each part of the work and
// goes through the pool's pages at once.
int book_ranks(int64_t warps, int64_t pages) { return warps <= kBookWarps && pages <= 4 * kBookThreads ? 1 : kBookRanks; }

rr_status check_list(int n, const rr_cache* C) {
    if (n < 0 || n > C->max_seqs) return rr_fail(RR_EINVAL, "%d sequences: 0..%d", n, C->max_seqs);
    return RR_OK;
}

rr_status copy_grid(int dev, unsigned* grid) {
    static std::atomic<int> sms[kMaxDevices] = {};
    int n = sms[dev].load(std::memory_order_relaxed);
    if (!n) {
        RR_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        sms[dev].store(n, std::memory_order_relaxed);
    }
    *grid = unsigned(n) * 8;
    return RR_OK;
}

}  // namespace

extern "C" rr_status rr_cache_bytes(const rr_cache* C, int64_t* page_bytes, int64_t* pitch, int64_t* book_bytes) {
    rr_clear_error();
    RR_TRY(check_cache(C));
    const CacheShape c = shape_of(C);
    if (page_bytes) *page_bytes = c.page_bytes;
    if (pitch) *pitch = c.pitch;
    if (book_bytes) *book_bytes = book_of(C, nullptr, nullptr);
    return RR_OK;
}

extern "C" rr_status rr_cache_clear(const rr_cache* C, void* book, cudaStream_t stream) {
    RR_TRACE("rr_cache_clear");
    rr_clear_error();
    RR_TRY(check_cache(C));
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, book, 16, "book"));
    Book b;
    const int64_t bytes = book_of(C, book, &b);
    RR_CUDA(cudaMemsetAsync(book, 0, size_t(bytes), stream));
    RR_CUDA(cudaMemsetAsync(b.table, 0xFF, size_t(C->max_seqs) * C->max_pages * 4, stream));
    return RR_OK;
}

extern "C" rr_status rr_cache_fork(const rr_cache* C, void* book, const int32_t* parents, const int32_t* children, int32_t n,
                                   cudaStream_t stream) {
    RR_TRACE("rr_cache_fork");
    rr_clear_error();
    RR_TRY(check_cache(C));
    RR_TRY(check_list(n, C));
    if (n == 0) return RR_OK;
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, book, 16, "book"));
    RR_TRY(check_device(dev, parents, 4, "parents"));
    RR_TRY(check_device(dev, children, 4, "children"));
    Book b;
    book_of(C, book, &b);
    const int ranks = book_ranks(int64_t(n) * ((C->max_pages + 127) / 128), 0);
    RR_CUDA(launch_clusters(rr_cache_fork_kernel, ranks, unsigned(ranks), kBookThreads, bits_bytes(C), stream, shape_of(C), b, parents,
                            children, n));
    return RR_OK;
}

extern "C" rr_status rr_cache_extend(const rr_cache* C, void* pages, void* book, const int32_t* seqs, const int32_t* starts, int32_t n,
                                     cudaStream_t stream) {
    RR_TRACE("rr_cache_extend");
    rr_clear_error();
    RR_TRY(check_cache(C));
    RR_TRY(check_list(n, C));
    if (n == 0) return RR_OK;
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, pages, 16, "pages"));
    RR_TRY(check_device(dev, book, 16, "book"));
    RR_TRY(check_device(dev, seqs, 4, "seqs"));
    if (starts) RR_TRY(check_device(dev, starts, 4, "starts"));
    Book b;
    book_of(C, book, &b);
    const CacheShape c = shape_of(C);
    unsigned most;
    RR_TRY(copy_grid(dev, &most));
    const int ranks = book_ranks(n / 32, C->n_pages);
    RR_CUDA(launch_clusters(rr_cache_extend_kernel, ranks, unsigned(ranks), kBookThreads, bits_bytes(C), stream, c, b, seqs, starts, n));
    const unsigned grid = unsigned(std::min<int64_t>(most, int64_t(n) * ((c.runs + kRuns - 1) / kRuns)));
    RR_CUDA(launch_after(rr_cache_copy_rows_kernel, grid, 256, stream, c, b, static_cast<char*>(pages)));
    return RR_OK;
}

extern "C" rr_status rr_cache_append(const rr_cache* C, void* pages, void* book, int32_t layer, const void* k, int64_t ldk, const void* v,
                                     int64_t ldv, int32_t rows, const int32_t* seqs, const int32_t* starts, int32_t n,
                                     cudaStream_t stream) {
    RR_TRACE("rr_cache_append");
    rr_clear_error();
    RR_TRY(check_cache(C));
    RR_TRY(check_list(n, C));
    if (layer < 0 || layer >= C->layers) return rr_fail(RR_EINVAL, "layer %d of %d", layer, C->layers);
    if (rows < 0 || (!starts && rows != n)) return rr_fail(RR_EINVAL, "%d rows of %d sequences", rows, n);
    const int64_t cols = int64_t(C->n_kv) * C->dim;
    if (ldk < cols || ldv < cols)
        return rr_fail(RR_EINVAL, "row strides %lld and %lld of rows of %lld", (long long)ldk, (long long)ldv, (long long)cols);
    if (n == 0 || rows == 0) return RR_OK;
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, pages, 16, "pages"));
    RR_TRY(check_device(dev, book, 16, "book"));
    RR_TRY(check_device(dev, k, 2, "k"));
    RR_TRY(check_device(dev, v, 2, "v"));
    RR_TRY(check_device(dev, seqs, 4, "seqs"));
    if (starts) RR_TRY(check_device(dev, starts, 4, "starts"));
    Book b;
    book_of(C, book, &b);
    const bool vec = (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0 && ldk % 8 == 0 && ldv % 8 == 0 && C->dim % 8 == 0;
    RR_CUDA(launch_after(vec ? rr_cache_append_kernel<true> : rr_cache_append_kernel<false>, unsigned((int64_t(rows) + 7) / 8), 256, stream,
                         shape_of(C), b, static_cast<char*>(pages), layer, static_cast<const uint16_t*>(k), ldk,
                         static_cast<const uint16_t*>(v), ldv, seqs, starts, n, rows));
    return RR_OK;
}

extern "C" rr_status rr_cache_truncate(const rr_cache* C, void* book, const int32_t* seqs, const int32_t* drop, int32_t n,
                                       cudaStream_t stream) {
    RR_TRACE("rr_cache_truncate");
    rr_clear_error();
    RR_TRY(check_cache(C));
    RR_TRY(check_list(n, C));
    if (n == 0) return RR_OK;
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, book, 16, "book"));
    RR_TRY(check_device(dev, seqs, 4, "seqs"));
    if (drop) RR_TRY(check_device(dev, drop, 4, "drop"));
    Book b;
    book_of(C, book, &b);
    const int ranks = book_ranks(n, 0);
    RR_CUDA(launch_clusters(rr_cache_truncate_kernel, ranks, unsigned(ranks), kBookThreads, bits_bytes(C), stream, shape_of(C), b, seqs,
                            drop, n));
    return RR_OK;
}

extern "C" rr_status rr_cache_compact(const rr_cache* C, void* pages, void* book, cudaStream_t stream) {
    RR_TRACE("rr_cache_compact");
    rr_clear_error();
    RR_TRY(check_cache(C));
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, pages, 16, "pages"));
    RR_TRY(check_device(dev, book, 16, "book"));
    Book b;
    book_of(C, book, &b);
    const CacheShape c = shape_of(C);
    unsigned most;
    RR_TRY(copy_grid(dev, &most));
    const int ranks = book_ranks(0, C->n_pages);
    RR_CUDA(launch_clusters(rr_cache_compact_kernel, ranks, unsigned(ranks), kBookThreads, 0, stream, c, b));
    constexpr int kSmem = kMoveStages * kMoveChunk;
    static std::atomic<uint32_t> ready{0};
    RR_CUDA(allow_smem(rr_cache_move_kernel, kSmem, dev, &ready));
    const int64_t chunks = (c.page_bytes + kMoveChunk - 1) / kMoveChunk * (C->n_pages / 2);
    const unsigned grid = unsigned(std::max<int64_t>(1, std::min<int64_t>(most / 8, std::max<int64_t>(chunks, (C->max_seqs + 6) / 7))));
    RR_CUDA(launch_clusters(rr_cache_move_kernel, 1, grid, 256, kSmem, stream, c, b, static_cast<char*>(pages)));
    return RR_OK;
}

extern "C" rr_status rr_cache_check(const rr_cache* C, void* book, cudaStream_t stream) {
    rr_clear_error();
    RR_TRY(check_cache(C));
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, book, 16, "book"));
    int32_t words[2] = {0, 0};       // kState, kLate
    RR_CUDA(cudaMemcpyAsync(words, book, 8, cudaMemcpyDeviceToHost, stream));
    RR_CUDA(cudaStreamSynchronize(stream));
    const int state = words[0] | words[1];
    if (!state) return RR_OK;
    RR_CUDA(cudaMemsetAsync(book, 0, 8, stream));
    RR_CUDA(cudaStreamSynchronize(stream));
    if (state & kBadWait) return rr_fail(RR_ECUDA, "a wait of a call on the cache ran out");
    // (A call that is not done takes over what one before it left, so that both are reported.)
    const char* const what = !words[0] ? "a call on the cache left something out" : !words[1] ? "a call on the cache was not done"
                                       : "a call on the cache left something out, and a later one was not done";
    return rr_fail(RR_EINVAL, "%s:%s%s%s%s%s", what, state & kBadRange ? " a sequence, length or count is out of range;" : "",
                   state & kBadTwice ? " a sequence is listed twice;" : "", state & kBadPool ? " no room for the new tokens;" : "",
                   state & kBadChild ? " a child holds tokens;" : "", state & kBadTable ? " the table has a page out of range;" : "");
}

extern "C" rr_status rr_accept(const float* p, int64_t ldp, const float* q, int64_t ldq, const int32_t* drafts, const int32_t* starts,
                               const float* u, const float* v, int32_t rows, int32_t n, int32_t vocab, int32_t* accepted, int32_t* tokens,
                               int32_t* rejected, cudaStream_t stream) {
    RR_TRACE("rr_accept");
    rr_clear_error();
    if (vocab < 1 || vocab > kMaxVocab) return rr_fail(RR_ELAYOUT, "%d tokens in the vocabulary: 1..%d", vocab, kMaxVocab);
    if (n < 0 || n > INT_MAX / kAcceptRanks || rows < 0 || (!starts && rows != n))
        return rr_fail(RR_EINVAL, "%d rows of %d sequences", rows, n);
    if (ldp < vocab || (q && ldq < vocab))
        return rr_fail(RR_EINVAL, "row strides %lld and %lld of rows of %d", (long long)ldp, (long long)ldq, vocab);
    if (n == 0) return RR_OK;
    if (rows == 0) return rr_fail(RR_EINVAL, "0 rows of %d sequences", n);
    int dev;
    RR_TRY(current_device(&dev));
    RR_TRY(check_device(dev, p, 4, "p"));
    if (q) RR_TRY(check_device(dev, q, 4, "q"));
    if (starts) {
        RR_TRY(check_device(dev, starts, 4, "starts"));
        RR_TRY(check_device(dev, drafts, 4, "drafts"));
        RR_TRY(check_device(dev, u, 4, "u"));
    }
    RR_TRY(check_device(dev, v, 4, "v"));
    RR_TRY(check_device(dev, accepted, 4, "accepted"));
    RR_TRY(check_device(dev, tokens, 4, "tokens"));
    if (rejected) RR_TRY(check_device(dev, rejected, 4, "rejected"));
    const AcceptArgs a = {p, q, ldp, ldq, drafts, starts, u, v, accepted, tokens, rejected, rows, vocab};
    // One block of 1024 threads fits an SM, and 15 clusters of 8 the GPU: up to there they read a row
    // soonest, beyond it blocks of 256, four an SM, need not wait for one another.  (us on the GPU, 256 /
    // 1024 threads, 151936 entries without drafts: n 1 8.5 / 7.2, 12 11.5 / 8.5, 16 12.4 / 12.7, 24 12.7 /
    // 14.2, 64 14.6 / 31.3; with refused drafts 1 10.4 / 9.0, 12 14.2 / 10.5, 16 14.9 / 16.8, 64 17.9 / 38.7.
    // 512 entries: 4.3 / 6.0 at 1, less than the host's time of a call either way, 4.9 / 10.6 at 16.)
    const int threads = n > 15 ? 256 : kAcceptThreads;
    RR_CUDA(launch_clusters(rr_accept_kernel, kAcceptRanks, unsigned(n) * kAcceptRanks, threads, 0, stream, a));
    return RR_OK;
}
