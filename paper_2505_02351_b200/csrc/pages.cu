// Pages of the cache: copying them, and the block tables, lengths and reference counts that say whose they are -- sequences
// forked, resized (their pages dropped and given), the pages in use moved together.
//
// A page is free where its count is 0, and free pages are handed out lowest number first in the order of the requests: ranks
// (prefix sums) of the free pages and of what is asked, whose results do not depend on the order of any atomic.  That part is one
// cluster of kClusterCtas CTAs, which exchanges its sums through distributed shared memory and takes a few barriers (a grid
// would need a launch per step), or one CTA where the pool and the requests are few.  What scales with the batch's tables and the
// pools -- dropping and sharing a table's pages, moving data -- runs on the whole GPU before and behind it.
//
// Data moves by bulk copies through shared memory, a ring of slots per warp that its first lane fills and empties: 64 pages of 64
// pools (264 MB read and written) 46 us, 5.7 TB/s, where loads and stores through registers took 51 to 52; the part-full page of a
// 16383-token prompt for 128 samples (504 MB, the reads from L2) 62 to 64 us against 79 to 85; 129 of 512 pages compacted (528 MB) 96 to 98.
// Rings of 8 or 16 KB slots and one or two CTAs per SM are within 3 % of that.  Few pages: 8 to 12 us for a call's two or three launches,
// a chain of dependent loads of tables and counts (about 0.7 us each) and barriers between.
//
#include <cooperative_groups.h>

#include "common.cuh"

namespace optgqa {

namespace cg = cooperative_groups;

namespace {

constexpr int kClusterCtas = 8;
constexpr int kClusterThreads = 1024;
constexpr int kCopyThreads = 128;
constexpr int kCopyWarps = kCopyThreads / 32;
constexpr int kCopyCtasPerSm = 3;
constexpr int kSlots = 4;                   // of a warp's ring
constexpr int kSlotBytes = 4096;
constexpr unsigned kFull = 0xffffffffu;

// Read of what other multiprocessors wrote in this launch: past L1.
__device__ __forceinline__ int ld_cg(const int* p) { return __ldcg(p); }

__device__ __forceinline__ bool in_pool(int page, int num_blocks) { return (unsigned)page < (unsigned)num_blocks; }

// ----------------------------------------------------------------------------- moving data
// Where share i of W begins in a list of `total`.
__device__ __forceinline__ long long share_of(long long total, long long i, long long W) {
    return total < (1ll << 40) ? total * i / W : total / W * i + total % W * i / W;
}

struct CopyRing {
    alignas(128) char data[kCopyWarps][kSlots][kSlotBytes];
    uint64_t full[kCopyWarps][kSlots];
};

__device__ __forceinline__ void bulk_s2g(void* dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
}

// Page src[i] to page dst[i] in every pool for i < n; kRows: the first rows[i] rows of every head alone.  A piece is up to
// kSlotBytes of a page, or of one head's rows.  Whole pages: the warps take the pieces in turn (in runs of their own, 47 us against
// 45 for the 64 pages).  Part-full ones: each warp takes a run of pieces, so that it looks a pair up once and not for every
// 4 KB (63 us against 70).
template <bool kRows>
__device__ __forceinline__ void copy_pages(CopyRing& ring, const PoolSet& pools, const PageShape& sh, const int* src, const int* dst,
                                           const int* rows, int n, int* status, int block, int blocks) {
    if (threadIdx.x & 31) return;
    const int w = threadIdx.x >> 5;
    uint64_t* full = ring.full[w];
    const unsigned run = kRows ? sh.head_bytes : sh.page_bytes, per_run = (run + kSlotBytes - 1) / kSlotBytes, runs = sh.page_bytes / run;
    const unsigned per_pool = per_run * runs, per_pair = per_pool * (unsigned)sh.num_pools;
    const long long total = (long long)n * per_pair;
    const long long warp = (long long)block * kCopyWarps + w, warps = (long long)blocks * kCopyWarps;
    const long long step = kRows ? 1 : warps, stop = kRows ? share_of(total, warp + 1, warps) : total;
    long long next = kRows ? share_of(total, warp, warps) : warp;
    if (next >= stop) return;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) mbar_init(&full[i], 1);
    fence_barrier_init();
    char* to[kSlots];
    unsigned bytes[kSlots];
    int pair = -1, from_page = 0, to_page = 0;
    unsigned limit = 0;
    // the next piece there is, into slot k; false at the end
    auto fill = [&](int k) -> bool {
        for (; next < stop; next += step) {
            const int i = total <= 0xffffffffll ? (int)((unsigned)next / per_pair) : (int)(next / per_pair);
            if (i != pair) {
                pair = i;
                from_page = ld_cg(src + i), to_page = ld_cg(dst + i);
                limit = kRows ? (unsigned)ld_cg(rows + i) * sh.row_bytes : run;
                if (!in_pool(from_page, sh.num_blocks) || !in_pool(to_page, sh.num_blocks)) limit = 0;
            }
            const unsigned rest = (unsigned)(next - (long long)i * per_pair), pool = rest / per_pool, in = rest - pool * per_pool;
            const unsigned r = in / per_run, off = (in - r * per_run) * kSlotBytes;
            if (off >= limit) {
                if (kRows && limit == 0) next = (long long)(i + 1) * per_pair - 1;      // nothing of this pair
                continue;
            }
            const size_t at = (size_t)r * run + off;
            const char* base = pools.p[pool];
            char* out = pools.p[pool] + (size_t)to_page * sh.page_bytes + at;
            const unsigned size = min(limit - off, (unsigned)kSlotBytes);
#pragma unroll
            for (int u = 0; u < kSlots; ++u)
                if (u == k) to[u] = out, bytes[u] = size;
            mbar_expect_tx(&full[k], size);
            bulk_g2s(ring.data[w][k], base + (size_t)from_page * sh.page_bytes + at, size, &full[k]);
            next += step;
            return true;
        }
        return false;
    };
    int filled = 0;
    while (filled < kSlots - 1 && fill(filled)) ++filled;
    for (int done = 0; done < filled; ++done) {
        const int k = done % kSlots;
        if (!mbar_wait(&full[k], (done / kSlots) & 1, status)) {
            for (int i = 0; i < 200; ++i) __nanosleep(1000);        // let what is in flight land
            break;
        }
        char* out = to[0];
        unsigned size = bytes[0];
#pragma unroll
        for (int u = 1; u < kSlots; ++u)
            if (u == k) out = to[u], size = bytes[u];
        bulk_s2g(out, ring.data[w][k], size);
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");      // the slot before this one has been read: it is next
        if (fill(filled % kSlots)) ++filled;
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

template <bool kRows>
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const __grid_constant__ PoolSet pools, const PageShape sh, const int* src,
                                                                  const int* dst, const int* rows, int n, int* status) {
    extern __shared__ __align__(128) char smem[];
    grid_dependency_wait();
    if (!kRows) grid_dependency_launch();   // (not before the wait, nor at all behind a table's kernel of the same call: see below)
    copy_pages<kRows>(*reinterpret_cast<CopyRing*>(smem), pools, sh, src, dst, rows, n, status, blockIdx.x, gridDim.x);
}

// ----------------------------------------------------------------------------- tables
// The attention kernels read tables and lengths before they wait, so a call that writes those lets no other call's kernel start
// before its own last kernel has ended.  A kernel behind which another one of the same call follows, which waits first, signals early.
// The last ones never do: behind a grid that does not signal, a dependent one starts when it has ended and its memory can be seen.
// A kernel that writes no table (copy_pages_kernel<false>) signals once it has waited, and so behind the tables' writer.

__device__ __forceinline__ int pages_of(int tokens, const PageTables& t) {
    return min((max(tokens, 0) + t.bs - 1) / t.bs, t.width);
}

// Entries [from, to) of a table's row let go, four loads in flight per thread.
__device__ __forceinline__ void drop_pages(const PageTables& t, int row, int from, int to, int first, int step) {
    int* entry = t.tables + (size_t)row * t.width;
    for (long long i = from + first; i < to; i += 4ll * step) {
        int page[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) page[u] = i + (long long)u * step < to ? entry[i + (long long)u * step] : -1;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (in_pool(page[u], t.num_blocks)) atomicSub(t.refs + page[u], 1);
            if (i + (long long)u * step < to) entry[i + (long long)u * step] = -1;
        }
    }
}

// What is asked of request i: the sequence's row, or -1 where the request is void.
__device__ __forceinline__ int fork_row(const PageTables& t, const PageRequests& r, int i) {
    const int parent = r.a[i], child = r.b[i];
    return (unsigned)parent < (unsigned)t.rows && (unsigned)child < (unsigned)t.rows ? child : -1;
}
// What the children held is dropped (the whole grid: a warp per 128 entries of a table's row).
__global__ void __launch_bounds__(256) fork_drop_kernel(const PageTables t, const PageRequests r) {
    grid_dependency_launch();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, row = fork_row(t, r, blockIdx.y);
    if (row < 0) return;
    const int pages = pages_of(t.lens[row], t);
    const int step = gridDim.x * 8 * 128;
    for (int from = (blockIdx.x * 8 + (threadIdx.x >> 5)) * 128; from < pages; from += step)
        drop_pages(t, row, from, min(from + 128, pages), lane, 32);
}

// The CTAs of a cluster, or the one there is.
template <int kCtas>
__device__ __forceinline__ void sync_all() {
    if constexpr (kCtas > 1) {
        cg::this_cluster().sync();
    } else {
        __threadfence();            // counts are changed and read past L1
        __syncthreads();
    }
}
template <int kCtas>
__device__ __forceinline__ int cta_rank() {
    if constexpr (kCtas > 1) return (int)cg::this_cluster().block_rank();
    else return 0;
}
// Every CTA of the cluster has begun, and may be written to, where all arrived and one has waited.  (Whole warps.)
template <int kCtas>
__device__ __forceinline__ void arrive_begun() {
    if constexpr (kCtas > 1) cluster_arrive_relaxed();
}
template <int kCtas>
__device__ __forceinline__ void wait_begun() {
    if constexpr (kCtas > 1) cluster_wait();
}
// `v` to place `rank` of every CTA's `all`.
template <int kCtas>
__device__ __forceinline__ void tell_all(long long* all, int rank, long long v) {
    if constexpr (kCtas > 1) {
        if (threadIdx.x < kCtas) *cg::this_cluster().map_shared_rank(all + rank, threadIdx.x) = v;
    } else if (threadIdx.x == 0) {
        all[0] = v;
    }
}

// Sum over the CTA's threads of `v`, of the threads before this one (exclusive) and in all (total); scratch [33].
__device__ __forceinline__ long long block_scan(long long v, long long* scratch, long long& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(kFull, incl, o);
        if (lane >= o) incl += u;
    }
    __syncthreads();                        // the scratch of the scan before
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        const long long w = scratch[lane];
        long long s = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(kFull, s, o);
            if (lane >= o) s += u;
        }
        scratch[lane] = s - w;
        if (lane == 31) scratch[32] = s;
    }
    __syncthreads();
    total = scratch[32];
    return scratch[warp] + incl - v;
}

// Four counts of pages from `at` on (a multiple of 4); past the end as if in use.
__device__ __forceinline__ int4 four_counts(const int* refs, int at, int num_blocks) {
    if (at + 4 <= num_blocks) return __ldcg(reinterpret_cast<const int4*>(refs + at));
    int4 v = make_int4(1, 1, 1, 1);
    if (at < num_blocks) v.x = ld_cg(refs + at);
    if (at + 1 < num_blocks) v.y = ld_cg(refs + at + 1);
    if (at + 2 < num_blocks) v.z = ld_cg(refs + at + 2);
    return v;
}

// A CTA's share of the pool: whole fours of pages.
struct Slice {
    int begin, end;
};
template <int kCtas>
__device__ __forceinline__ Slice slice_of(int num_blocks, int rank) {
    const int fours = num_blocks / 4 + (num_blocks % 4 != 0), per = (fours + kCtas - 1) / kCtas;
    const long long b = 4ll * per * rank, e = b + 4ll * per;
    return {(int)min(b, (long long)num_blocks), (int)min(e, (long long)num_blocks)};
}

// The cluster: what the requests let go is dropped, what they ask for and what is free is counted, the free pages that are handed
// out are listed, and every request that can be served is: where its own pages and those asked before it are there.  Each CTA has a
// share of the requests, in the order of the list, and a slice of the pool.  A round trip to L2 is 0.7 us, so what does not depend on
// one another is loaded together, and what a request needs later stays in shared memory (of up to kTold requests per CTA).
constexpr int kTold = kClusterThreads;
constexpr int kListed = 1024;               // free pages listed in shared memory, by one CTA

// What is known of the requests of a CTA's share.
struct Told {
    int need[kTold];        // pages asked, -1: void
    int first[kTold];       // the table entry they begin at
    int rows[kTold];        // rows of a part-full page to copy
    int src[kTold];         // from which page
    int from[kTold];        // table entries to let go: from .. to - 1
    int to[kTold];
    long long before[kTold];        // pages asked before it in the share
};

template <bool kFork, int kCtas>
__global__ void __launch_bounds__(kClusterThreads)
give_pages_kernel(const PageTables t, const PageRequests r, const PageWork w, bool drops) {
    extern __shared__ __align__(128) char smem[];
    __shared__ long long scratch[33];
    __shared__ long long all_need[kCtas], all_free[kCtas];
    __shared__ int listed[kListed];
    const int rank = cta_rank<kCtas>(), tid = threadIdx.x;
    arrive_begun<kCtas>();
    grid_dependency_launch();
    grid_dependency_wait();
    const int share = (r.n + kCtas - 1) / kCtas, mine = min(share * rank, r.n), count = min(share, r.n - mine);
    // in shared memory, or in the workspace where there are more
    Told& told = *reinterpret_cast<Told*>(smem);
    const bool few = share <= kTold;
    int* const need_of = few ? told.need : w.need + mine;
    int* const first_of = few ? told.first : w.first + mine;
    int* const rows_of = few ? told.rows : w.rows + mine;
    int* const src_of = few ? told.src : w.src + mine;
    int* const from_of = few ? told.from : w.from + mine;
    int* const to_of = few ? told.to : w.to + mine;
    long long* const before_of = few ? told.before : w.before + mine;
    // 2^k threads of the CTA for one request
    int lanes = 1;
    while (lanes < kClusterThreads && (long long)share * (lanes * 2) <= kClusterThreads) lanes *= 2;
    const int group = tid / lanes, sub = tid % lanes, groups = kClusterThreads / lanes;

    for (int i = tid; i < count; i += kClusterThreads) {
        const int a = r.a[mine + i], b = r.b[mine + i];
        const bool real = (unsigned)a < (unsigned)t.rows && (kFork ? (unsigned)b < (unsigned)t.rows : b >= 0 && b <= (long long)t.width * t.bs);
        int need = -1, first = 0, rows = 0, from = 0, to = 0;
        if (real) {
            const int tokens = t.lens[a], have = pages_of(tokens, t);
            if (kFork) {
                const int n = min(max(tokens, 0), t.width * t.bs);
                first = n / t.bs;
                rows = n % t.bs;
                need = rows != 0;
                to = pages_of(t.lens[b], t);
            } else {
                const int want = pages_of(b, t);
                first = have;
                need = max(want - have, 0);
                from = want;
                to = have;
                if (b > tokens && tokens > 0 && have > 0) rows = tokens % t.bs;     // (whether they are copied is seen below)
            }
        }
        need_of[i] = need;
        first_of[i] = first;
        rows_of[i] = rows;
        from_of[i] = from;
        to_of[i] = drops ? to : from;
    }
    __syncthreads();
    wait_begun<kCtas>();
    // the pages that may be copied from (parents and sequences that grow drop nothing), requested beside what is dropped
    for (int i = tid; i < count; i += kClusterThreads) {
        int last = -1;
        if (rows_of[i] > 0) last = t.tables[(size_t)r.a[mine + i] * t.width + (kFork ? first_of[i] : first_of[i] - 1)];
        src_of[i] = last;
    }
    for (int i = group; i < count; i += groups)
        if (from_of[i] < to_of[i]) drop_pages(t, kFork ? r.b[mine + i] : r.a[mine + i], from_of[i], to_of[i], sub, lanes);
    if (drops) sync_all<kCtas>();
    else __syncthreads();

    // what is free: of the slice's first pages, which is mostly all of it, the counts are kept
    const Slice s = slice_of<kCtas>(t.num_blocks, rank);
    const bool one_tile = s.end - s.begin <= 4 * kClusterThreads;
    int4 v = make_int4(1, 1, 1, 1);
    if (s.begin + 4 * tid < s.end) v = four_counts(t.refs, s.begin + 4 * tid, t.num_blocks);
    // what is asked, request by request
    long long asked = 0;
    for (int base = 0; base < count; base += kClusterThreads) {
        const int i = base + tid;
        int need = 0;
        if (i < count) {
            need = need_of[i];
            // a part-full last page that another sequence holds too is replaced before this one writes into it
            if (!kFork && rows_of[i] > 0) {
                const int last = src_of[i];
                if (in_pool(last, t.num_blocks) && ld_cg(t.refs + last) > 1) {
                    need_of[i] = ++need;
                    --first_of[i];
                } else {
                    rows_of[i] = 0;
                }
            }
        }
        long long total;
        const long long before = block_scan(max(need, 0), scratch, total);
        if (i < count) before_of[i] = asked + before;
        asked += total;
    }
    long long zeros = (v.x == 0) + (v.y == 0) + (v.z == 0) + (v.w == 0), here;
    for (int at = s.begin + 4 * (tid + kClusterThreads); at < s.end; at += 4 * kClusterThreads) {
        const int4 u = four_counts(t.refs, at, t.num_blocks);
        zeros += (u.x == 0) + (u.y == 0) + (u.z == 0) + (u.w == 0);
    }
    const long long zeros_before = block_scan(zeros, scratch, here);        // (in the order of the pages where there is one tile)
    tell_all<kCtas>(all_need, rank, asked);
    tell_all<kCtas>(all_free, rank, here);
    sync_all<kCtas>();
    long long total_need = 0, total_free = 0, rank_need = 0, rank_free = 0;
    for (int c = 0; c < kCtas; ++c) {
        if (c == rank) rank_need = total_need, rank_free = total_free;
        total_need += all_need[c];
        total_free += all_free[c];
    }
    // the list of the pages to hand out
    const bool near = kCtas == 1 && total_need <= kListed;
    int* const list = near ? listed : w.free_list;
    for (int base = s.begin; base < s.end && rank_free < total_need; base += 4 * kClusterThreads) {
        const int at = base + 4 * tid;
        long long k = zeros_before, total = here;
        if (!one_tile) {
            v = make_int4(1, 1, 1, 1);
            if (at < s.end) v = four_counts(t.refs, at, t.num_blocks);
            k = block_scan((v.x == 0) + (v.y == 0) + (v.z == 0) + (v.w == 0), scratch, total);
        }
        k += rank_free;
        if (v.x == 0 && k++ < total_need) list[k - 1] = at;
        if (v.y == 0 && k++ < total_need) list[k - 1] = at + 1;
        if (v.z == 0 && k++ < total_need) list[k - 1] = at + 2;
        if (v.w == 0 && k++ < total_need) list[k - 1] = at + 3;
        rank_free += total;
    }
    if constexpr (kCtas > 1) sync_all<kCtas>();
    else __syncthreads();               // (one CTA reads its own list)

    for (int i = group; i < count; i += groups) {
        const int need = need_of[i], rows = rows_of[i], a = r.a[mine + i], b = r.b[mine + i];
        const long long from = rank_need + before_of[i];
        const bool served = need >= 0 && (need == 0 || from + need <= total_free);
        auto page_at = [&](long long k) { return near || kCtas == 1 ? list[from + k] : ld_cg(w.free_list + from + k); };
        if (served && need > 0) {
            const int first = first_of[i];
            int* entry = t.tables + (size_t)(kFork ? b : a) * t.width;
            for (long long k = sub; k < need; k += 4ll * lanes) {
                int page[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) page[u] = k + (long long)u * lanes < need ? page_at(k + (long long)u * lanes) : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (page[u] < 0) break;
                    if (first + k + (long long)u * lanes < t.width) entry[first + k + (long long)u * lanes] = page[u];
                    t.refs[page[u]] = 1;
                }
            }
        }
        if (sub == 0) {
            const int src = src_of[i];
            const bool copies = served && rows > 0;
            if (!kFork && copies) atomicSub(t.refs + src, 1);
            w.rows[mine + i] = copies ? rows : 0;
            w.src[mine + i] = src;
            w.dst[mine + i] = copies ? page_at(0) : -1;
            r.done[mine + i] = served;
            if (kFork) {
                if (need >= 0) t.lens[b] = served ? t.lens[a] : 0;
            } else if (served) {
                t.lens[a] = b;
            }
        }
    }
}

// The parents' whole pages shared with their children, and the part-full ones copied: by CTAs of their own, the first `sharing` and the
// others, or one behind the other (sharing 0).  Neighbouring requests of one parent are a run: the first of them adds for all.
__global__ void __launch_bounds__(kCopyThreads) fork_share_kernel(const __grid_constant__ PoolSet pools, const PageShape sh, const PageTables t,
                                                                  const PageRequests r, const PageWork w, int chunks, int sharing, int* status) {
    extern __shared__ __align__(128) char smem[];
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, block = blockIdx.x, warps = (sharing ? sharing : gridDim.x) * kCopyWarps;
    if (sharing && block >= sharing) {
        copy_pages<true>(*reinterpret_cast<CopyRing*>(smem), pools, sh, w.src, w.dst, w.rows, r.n, status, block - sharing, gridDim.x - sharing);
        return;
    }
    for (long long c = (long long)block * kCopyWarps + (threadIdx.x >> 5); c < (long long)r.n * chunks; c += warps) {
        const int i = (int)(c / chunks), from = (int)(c - (long long)i * chunks) * 128;
        const int parent = r.a[i];
        if ((unsigned)parent >= (unsigned)t.rows) continue;
        const int whole = min(max(t.lens[parent], 0) / t.bs, t.width);
        if (from >= whole) continue;
        const bool done = r.done[i] != 0;       // (and so the child is a row)
        int times = 0;
        if (i == 0 || r.a[i - 1] != parent) {
            for (int j = i;; j += 32) {
                const bool same = j + lane < r.n && r.a[j + lane] == parent;
                const unsigned run = __ballot_sync(kFull, same), ok = __ballot_sync(kFull, same && r.done[j + lane] != 0);
                const unsigned upto = run == kFull ? kFull : (1u << (__ffs(~run) - 1)) - 1u;
                times += __popc(ok & upto);
                if (run != kFull) break;
            }
        }
        const int* of = t.tables + (size_t)parent * t.width;
        int* entry = t.tables + (size_t)(done ? r.b[i] : 0) * t.width;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = from + u * 32 + lane;
            if (k >= whole) break;
            const int page = of[k];
            if (done) entry[k] = page;
            if (times && in_pool(page, t.num_blocks)) atomicAdd(t.refs + page, times);
        }
    }
    if (sharing) return;
    __syncwarp();
    copy_pages<true>(*reinterpret_cast<CopyRing*>(smem), pools, sh, w.src, w.dst, w.rows, r.n, status, block, gridDim.x);
}

// ----------------------------------------------------------------------------- compaction
// U pages are in use.  The k-th page in use at or past U goes to the k-th free one below U.
template <int kCtas>
__global__ void __launch_bounds__(kClusterThreads)
compact_plan_kernel(const int* refs, int* refs_out, int* page_map, int* used_out, const PageWork w, int num_blocks) {
    __shared__ long long scratch[33];
    __shared__ long long all_used[kCtas], all_low[kCtas];
    const int rank = cta_rank<kCtas>(), tid = threadIdx.x;
    arrive_begun<kCtas>();
    grid_dependency_launch();
    grid_dependency_wait();
    const Slice s = slice_of<kCtas>(num_blocks, rank);
    // of the slice's first pages, which is mostly all of it, the counts are kept
    int4 kept = make_int4(0, 0, 0, 0);
    if (s.begin + 4 * tid < s.end) kept = four_counts(refs, s.begin + 4 * tid, num_blocks);
    auto counts = [&](int at) { return at < s.begin + 4 * kClusterThreads ? kept : four_counts(refs, at, num_blocks); };
    long long count = 0, here;
    for (int at = s.begin + 4 * tid; at < s.end; at += 4 * kClusterThreads) {
        const int4 v = counts(at);
        const int live = min(4, num_blocks - at);       // past the end reads as in use
        count += (v.x > 0) + (v.y > 0) + (v.z > 0) + (v.w > 0) - (4 - live);
    }
    block_scan(count, scratch, here);
    wait_begun<kCtas>();
    tell_all<kCtas>(all_used, rank, here);
    sync_all<kCtas>();
    long long before = 0, U = 0;
    for (int c = 0; c < kCtas; ++c) {
        if (c == rank) before = U;
        U += all_used[c];
    }
    // pages in use below U: the holes and the movers are as many, U less those
    count = 0;
    for (int at = s.begin + 4 * tid; at < s.end && at < U; at += 4 * kClusterThreads) {
        const int4 v = counts(at);
        count += (at < U && v.x > 0) + (at + 1 < U && v.y > 0) + (at + 2 < U && v.z > 0) + (at + 3 < U && v.w > 0);
    }
    block_scan(count, scratch, here);
    tell_all<kCtas>(all_low, rank, here);
    sync_all<kCtas>();
    long long low = 0;
    for (int c = 0; c < kCtas; ++c) low += all_low[c];
    for (int base = s.begin; base < s.end; base += 4 * kClusterThreads) {
        const int at = base + 4 * tid;
        int ref[4] = {0, 0, 0, 0};
        if (at < s.end) {
            const int4 v = counts(at);
            ref[0] = v.x, ref[1] = v.y, ref[2] = v.z, ref[3] = v.w;
        }
        int live = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (at + u >= s.end) ref[u] = 0;
            live += ref[u] > 0;
        }
        long long total;
        long long k = before + block_scan(live, scratch, total);        // pages in use before this one
        before += total;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int page = at + u;
            if (page >= s.end) break;
            if (ref[u] > 0) {
                if (page < U) {
                    page_map[page] = page;
                    refs_out[page] = ref[u];
                } else {
                    w.src[k - low] = page;
                    w.rows[k - low] = ref[u];       // (its count)
                    refs_out[page] = 0;
                }
                ++k;
            } else {
                if (page < U) w.dst[page - k] = page;       // as many free ones before it as are not in use
                else refs_out[page] = 0;
                page_map[page] = -1;
            }
        }
    }
    sync_all<kCtas>();
    const long long moves = U - low;
    for (long long k = rank * kClusterThreads + tid; k < moves; k += kCtas * kClusterThreads) {
        const int from = ld_cg(w.src + k), to = ld_cg(w.dst + k);
        page_map[from] = to;
        refs_out[to] = ld_cg(w.rows + k);
    }
    if (rank == 0 && tid == 0) {
        used_out[0] = (int)U;
        w.first[0] = (int)moves;
    }
}

__global__ void __launch_bounds__(kCopyThreads) compact_move_kernel(const __grid_constant__ PoolSet pools, const PageShape sh, const int* tables,
                                                                    int* tables_out, const int* lens, const int* page_map, const PageWork w,
                                                                    int rows, int width, int bs, int* status) {
    extern __shared__ __align__(128) char smem[];
    grid_dependency_wait();
    const long long entries = (long long)rows * width;
    for (long long e = (long long)blockIdx.x * kCopyThreads + threadIdx.x; e < entries; e += (long long)gridDim.x * kCopyThreads) {
        const int row = (int)(e / width), k = (int)(e - (long long)row * width), page = tables[e];
        const bool held = (long long)k * bs < lens[row] && in_pool(page, sh.num_blocks);
        tables_out[e] = held ? page_map[page] : page;
    }
    __syncwarp();
    copy_pages<false>(*reinterpret_cast<CopyRing*>(smem), pools, sh, w.src, w.dst, nullptr, w.first[0], status, blockIdx.x, gridDim.x);
}

// One resident wave, or fewer where there are fewer pieces (and chunks of tables).
unsigned copy_ctas(const PageShape& sh, long long pairs, long long chunks = 0) {
    const long long per_page = (sh.page_bytes + kSlotBytes - 1) / kSlotBytes;
    const long long pieces = pairs * sh.num_pools * per_page, most = (long long)sm_count() * kCopyCtasPerSm;
    const long long ctas = ((pieces > chunks ? pieces : chunks) + kCopyWarps - 1) / kCopyWarps;
    return (unsigned)(ctas < 1 ? 1 : ctas < most ? ctas : most);
}

// A launch of the kernels with a ring.
template <typename... KArgs, typename... Args>
int launch_copying(void (*kernel)(KArgs...), unsigned ctas, std::atomic<bool>* configured, cudaStream_t stream, Args... args) {
    if (!ensure_smem_limit(kernel, sizeof(CopyRing), configured)) return OPT_GQA_ERR_CUDA;
    return launch_dependent(kernel, dim3(ctas), dim3(kCopyThreads), sizeof(CopyRing), stream, args...);
}

// One CTA instead of the cluster, whose barriers and sums through distributed shared memory cost 1 us, where its threads have one vector
// of counts each and there are no more than half as many requests.  (In a graph, us, one CTA against the cluster.  Steps that resize 32
// sequences in pools of 512, 4096, 8192 and 32768 pages: 8.3 8.2 9.3 10.6 against 9.4 9.7 9.6 9.2; of 256 and 1024 in 4096: 9.1 and 11.1
// against 9.7 and 10.9.)
constexpr int kOneCtaPages = 4 * kClusterThreads, kOneCtaRequests = kClusterThreads / 2;
bool one_cta(int num_blocks, int n) { return num_blocks <= kOneCtaPages && n <= kOneCtaRequests; }
// The compaction goes over the counts again and again and writes as much: 512, 2048, 4096 and 8192 pages 7.3 8.9 10.4 13.7 against 7.9 8.6
// 8.8 9.0.
constexpr int kOneCtaCompact = 1024;
// Entries of the children's tables up to which give_pages_kernel drops them itself, without a launch of the whole GPU before it.  (Forks
// of a parent whose pages fill the tables, us, itself against with that launch: one CTA, 256, 4096, 8192 and 16384 entries 9.8 11.6 14.4
// 15.4 against 10.3 11.4 12.0 11.9; the cluster, 2048, 16384, 32768 and 131072 entries 11.8 12.0 12.3 17.4 against 12.1 12.6 13.0 14.3.)
constexpr long long kOneCtaDrop = 4096, kClusterDrop = 32768;

}  // namespace

int launch_copy_pages(const PoolSet& pools, const PageShape& sh, const int* src, const int* dst, int n, int* status, cudaStream_t stream) {
    static std::atomic<bool> configured[kMaxDevices];
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    return launch_copying(copy_pages_kernel<false>, copy_ctas(sh, n), configured, stream, pools, sh, src, dst, nullptr, n, status);
}

// Sharing has CTAs of its own where they are few or fit beside the copying ones.  (In a graph, us, one behind the other against that: a
// prompt of 541 tokens to 4, 32 and 64 children in 8 pools 10.0 11.2 13.2 against 8.9 10.7 12.8; but 16383 tokens to 30 in 64 pools, where
// sharing would take 60 of 444 CTAs, 22.3 against 23.7.)
int launch_fork(const PoolSet& pools, const PageShape& sh, const PageTables& t, const PageRequests& r, const PageWork& w, int* status,
                cudaStream_t stream) {
    static std::atomic<bool> configured[kMaxDevices];
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    const long long entries = (long long)r.n * t.width;
    const bool one = one_cta(t.num_blocks, r.n), drops = entries <= (one ? kOneCtaDrop : kClusterDrop);
    int rc = OPT_GQA_OK;
    if (!drops) {
        const unsigned x = (unsigned)((t.width + 1023) / 1024);
        rc = launch_dependent(fork_drop_kernel, dim3(x < 64 ? x : 64, (unsigned)r.n), dim3(256), 0, stream, t, r);
        if (rc != OPT_GQA_OK) return rc;
    }
    rc = one ? launch_clusters(give_pages_kernel<true, 1>, dim3(1), dim3(kClusterThreads), 1, sizeof(Told), stream, t, r, w, drops)
             : launch_clusters(give_pages_kernel<true, kClusterCtas>, dim3(kClusterCtas), dim3(kClusterThreads), kClusterCtas, sizeof(Told), stream, t, r, w, drops);
    if (rc != OPT_GQA_OK) return rc;
    const int chunks = (t.width + 127) / 128;
    const long long wave = (long long)sm_count() * kCopyCtasPerSm, share = ((long long)r.n * chunks + kCopyWarps - 1) / kCopyWarps;
    const int sharing = 16 * share <= wave || share + copy_ctas(sh, r.n) <= wave ? (int)share : 0;
    const long long copy = copy_ctas(sh, r.n, sharing ? 0 : (long long)r.n * chunks);
    return launch_copying(fork_share_kernel, (unsigned)(sharing + (copy < wave - sharing ? copy : wave - sharing)), configured, stream, pools, sh,
                          t, r, w, chunks, sharing, status);
}

int launch_resize(const PoolSet& pools, const PageShape& sh, const PageTables& t, const PageRequests& r, const PageWork& w, int* status,
                  cudaStream_t stream) {
    static std::atomic<bool> configured[kMaxDevices];
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    const int rc = one_cta(t.num_blocks, r.n)
                       ? launch_clusters(give_pages_kernel<false, 1>, dim3(1), dim3(kClusterThreads), 1, sizeof(Told), stream, t, r, w, true)
                       : launch_clusters(give_pages_kernel<false, kClusterCtas>, dim3(kClusterCtas), dim3(kClusterThreads), kClusterCtas, sizeof(Told), stream, t, r, w, true);
    if (rc != OPT_GQA_OK) return rc;
    return launch_copying(copy_pages_kernel<true>, copy_ctas(sh, r.n), configured, stream, pools, sh, w.src, w.dst, w.rows, r.n, status);
}

int launch_compact(const PoolSet& pools, const PageShape& sh, const PageTables& t, int* tables_out, int* refs_out, int* page_map, int* used,
                   const PageWork& w, int* status, cudaStream_t stream) {
    static std::atomic<bool> configured[kMaxDevices];
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    const int rc = t.num_blocks <= kOneCtaCompact
                       ? launch_clusters(compact_plan_kernel<1>, dim3(1), dim3(kClusterThreads), 1, 0, stream, t.refs, refs_out, page_map, used, w, t.num_blocks)
                       : launch_clusters(compact_plan_kernel<kClusterCtas>, dim3(kClusterCtas), dim3(kClusterThreads), kClusterCtas, 0, stream, t.refs, refs_out, page_map, used, w, t.num_blocks);
    if (rc != OPT_GQA_OK) return rc;
    return launch_copying(compact_move_kernel, copy_ctas(sh, t.num_blocks / 2 + 1, (long long)t.rows * t.width / 32), configured, stream, pools,
                          sh, t.tables, tables_out, t.lens, page_map, w, t.rows, t.width, t.bs, status);
}

}  // namespace optgqa
