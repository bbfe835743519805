// Pages of the cache: copying them, and the block tables, lengths and reference counts that say whose they are -- sequences
// forked, resized (their pages dropped and given), the pages in use moved together.
//
// A page is free where its count is 0, and free pages are handed out lowest number first in the order of the requests: ranks
// (prefix sums) of the free pages and of what is asked, whose results do not depend on the order of any atomic.  That part is one
// cluster of kClusterCtas CTAs, which exchanges its sums through distributed shared memory and takes a few barriers: a grid
// would need a launch per step, one CTA an eighth of the loads in flight.  What scales with the batch's tables and the pools --
// dropping and sharing a table's pages, moving data -- runs on the whole GPU before and behind it.
//
// Data moves in pieces of 2 KB, one per warp and step, four independent 16-byte vectors per lane; a page's run of one head (bs
// rows) is always whole pieces, so the first rows of a page are the first vectors of each head's pieces.
#include <cooperative_groups.h>

#include "common.cuh"

namespace optgqa {

namespace cg = cooperative_groups;

namespace {

constexpr int kClusterCtas = 8;
constexpr int kClusterThreads = 1024;
constexpr int kAll = kClusterCtas * kClusterThreads;
constexpr int kPieceBytes = 2048;
constexpr int kCopyThreads = 256;
constexpr int kCopyCtasPerSm = 8;
constexpr unsigned kFull = 0xffffffffu;

// Read of what other multiprocessors wrote in this launch: past L1.
__device__ __forceinline__ int ld_cg(const int* p) { return __ldcg(p); }

__device__ __forceinline__ bool in_pool(int page, int num_blocks) { return (unsigned)page < (unsigned)num_blocks; }

// ----------------------------------------------------------------------------- moving data
// Every warp of the grid takes pieces in turn.  rows: how many of a page's rows are copied (null: all).
__device__ __forceinline__ void copy_pieces(const PoolSet& pools, const PageShape& sh, const int* src, const int* dst, const int* rows,
                                            int n) {
    const int lane = threadIdx.x & 31;
    const long long warp = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), warps = (long long)gridDim.x * (blockDim.x >> 5);
    const unsigned per_page = sh.page_bytes / kPieceBytes, per_pair = per_page * (unsigned)sh.num_pools;
    const long long total = (long long)n * per_pair;
    for (long long i = warp; i < total; i += warps) {
        const int pair = total <= 0xffffffffll ? (int)((unsigned)i / per_pair) : (int)(i / per_pair);
        const unsigned rest = (unsigned)(i - (long long)pair * per_pair), pool = rest / per_page, at = (rest - pool * per_page) * kPieceBytes;
        const int s = ld_cg(src + pair), d = ld_cg(dst + pair);
        if (!in_pool(s, sh.num_blocks) || !in_pool(d, sh.num_blocks)) continue;
        const unsigned in_head = at % sh.head_bytes + lane * 16;
        const unsigned limit = rows ? (unsigned)ld_cg(rows + pair) * sh.row_bytes : sh.head_bytes;
        const uint4* from = reinterpret_cast<const uint4*>(pools.p[pool] + (size_t)s * sh.page_bytes + at) + lane;
        uint4* to = reinterpret_cast<uint4*>(pools.p[pool] + (size_t)d * sh.page_bytes + at) + lane;
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (in_head + u * 512 < limit) v[u] = __ldcs(from + u * 32);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (in_head + u * 512 < limit) __stcs(to + u * 32, v[u]);
    }
}

__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const __grid_constant__ PoolSet pools, const PageShape sh, const int* src,
                                                                  const int* dst, const int* rows, int n, bool last) {
    if (last) grid_dependency_launch();     // (behind a table's kernel nothing may start early: see below)
    grid_dependency_wait();
    copy_pieces(pools, sh, src, dst, rows, n);
}

// ----------------------------------------------------------------------------- tables
// The kernels that write tables and lengths never let the next kernel of another call start early: the attention kernels read
// those before they wait.  Those behind which another kernel of the same call follows, which waits first, do.

__device__ __forceinline__ int pages_of(int tokens, const PageTables& t) {
    return min((max(tokens, 0) + t.bs - 1) / t.bs, t.width);
}

// Entries [from, to) of a table's row let go.
__device__ __forceinline__ void drop_pages(const PageTables& t, int row, int from, int to, int first, int step) {
    int* entry = t.tables + (size_t)row * t.width;
    for (int i = from + first; i < to; i += step) {
        const int page = entry[i];
        if (in_pool(page, t.num_blocks)) atomicSub(t.refs + page, 1);
        entry[i] = -1;
    }
}

// What is asked of request i: the sequence's row, or -1 where the request is void.
__device__ __forceinline__ int fork_row(const PageTables& t, const PageRequests& r, int i) {
    const int parent = r.a[i], child = r.b[i];
    return (unsigned)parent < (unsigned)t.rows && (unsigned)child < (unsigned)t.rows ? child : -1;
}
__device__ __forceinline__ int resize_row(const PageTables& t, const PageRequests& r, int i) {
    const int row = r.a[i], tokens = r.b[i];
    return (unsigned)row < (unsigned)t.rows && tokens >= 0 && tokens <= (long long)t.width * t.bs ? row : -1;
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
__device__ __forceinline__ Slice slice_of(int num_blocks, int rank) {
    const int fours = num_blocks / 4 + (num_blocks % 4 != 0), per = (fours + kClusterCtas - 1) / kClusterCtas;
    const long long b = 4ll * per * rank, e = b + 4ll * per;
    return {(int)min(b, (long long)num_blocks), (int)min(e, (long long)num_blocks)};
}

// The cluster: what is asked and what is free is counted, the free pages that are handed out are listed, and every request that
// can be served is.  Request i is served where its own pages and those asked before it are there.
template <bool kFork>
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kClusterThreads)
give_pages_kernel(const PageTables t, const PageRequests r, const PageWork w, bool drops) {
    __shared__ long long scratch[33];
    __shared__ long long all_need[kClusterCtas], all_free[kClusterCtas];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), tid = threadIdx.x;
    grid_dependency_launch();
    grid_dependency_wait();
    // 2^k threads for one request, of the whole cluster
    int lanes = 1;
    while (lanes < kAll && (long long)r.n * (lanes * 2) <= kAll) lanes *= 2;
    const int group = (rank * kClusterThreads + tid) / lanes, sub = (rank * kClusterThreads + tid) % lanes, groups = kAll / lanes;

    if (drops) {
        for (int i = group; i < r.n; i += groups) {
            const int row = kFork ? fork_row(t, r, i) : resize_row(t, r, i);
            if (row < 0) continue;
            drop_pages(t, row, kFork ? 0 : pages_of(r.b[i], t), pages_of(t.lens[row], t), sub, lanes);
        }
        cluster.sync();
    }

    // what is asked, request by request in the order of the list: a share of the list per CTA
    const int share = (r.n + kClusterCtas - 1) / kClusterCtas;
    const int mine = min(share * rank, r.n), mine_end = min(share * (rank + 1), r.n);
    long long asked = 0;
    for (int base = mine; base < mine_end; base += kClusterThreads) {
        const int i = base + tid;
        int need = 0, first = 0, rows = 0, last = -1;
        if (i < mine_end) {
            const int row = kFork ? fork_row(t, r, i) : resize_row(t, r, i);
            if (row < 0) {
                need = -1;
            } else if (kFork) {
                const int n = min(max(t.lens[r.a[i]], 0), t.width * t.bs);
                first = n / t.bs;
                rows = n % t.bs;
                need = rows != 0;
                if (rows) last = ld_cg(t.tables + (size_t)r.a[i] * t.width + first);
            } else {
                const int n = t.lens[row], want = pages_of(r.b[i], t);
                first = pages_of(n, t);
                if (r.b[i] > n) {
                    need = want - first;
                    // a part-full last page that another sequence holds too is replaced before this one writes into it
                    if (n > 0 && n % t.bs != 0 && first > 0) {
                        last = ld_cg(t.tables + (size_t)row * t.width + first - 1);
                        if (in_pool(last, t.num_blocks) && ld_cg(t.refs + last) > 1) {
                            rows = n % t.bs;
                            --first;
                            ++need;
                        }
                    }
                }
            }
        }
        long long total;
        const long long before = block_scan(max(need, 0), scratch, total);
        if (i < mine_end) {
            w.need[i] = need;
            w.first[i] = first;
            w.rows[i] = rows;
            w.src[i] = last;
            w.before[i] = asked + before;
        }
        asked += total;
    }
    // what is free
    const Slice s = slice_of(t.num_blocks, rank);
    long long zeros = 0;
    for (int at = s.begin + 4 * tid; at < s.end; at += 4 * kClusterThreads) {
        const int4 v = four_counts(t.refs, at, t.num_blocks);
        zeros += (v.x == 0) + (v.y == 0) + (v.z == 0) + (v.w == 0);
    }
    long long here;
    block_scan(zeros, scratch, here);
    if (tid < kClusterCtas) {
        *cluster.map_shared_rank(&all_need[rank], tid) = asked;
        *cluster.map_shared_rank(&all_free[rank], tid) = here;
    }
    cluster.sync();
    long long total_need = 0, total_free = 0, rank_free = 0;
    for (int c = 0; c < kClusterCtas; ++c) {
        if (c == rank) rank_free = total_free;
        total_need += all_need[c];
        total_free += all_free[c];
    }
    // the list of the pages to hand out
    for (int base = s.begin; base < s.end && rank_free < total_need; base += 4 * kClusterThreads) {
        const int at = base + 4 * tid;
        int4 v = make_int4(1, 1, 1, 1);
        if (at < s.end) v = four_counts(t.refs, at, t.num_blocks);
        long long total;
        long long k = rank_free + block_scan((v.x == 0) + (v.y == 0) + (v.z == 0) + (v.w == 0), scratch, total);
        if (v.x == 0 && k++ < total_need) w.free_list[k - 1] = at;
        if (v.y == 0 && k++ < total_need) w.free_list[k - 1] = at + 1;
        if (v.z == 0 && k++ < total_need) w.free_list[k - 1] = at + 2;
        if (v.w == 0 && k++ < total_need) w.free_list[k - 1] = at + 3;
        rank_free += total;
    }
    cluster.sync();

    for (int i = group; i < r.n; i += groups) {
        const int need = ld_cg(w.need + i), rows = ld_cg(w.rows + i);
        long long from = __ldcg(w.before + i);
        for (int c = 0; c < i / share; ++c) from += all_need[c];
        const bool served = need >= 0 && (need == 0 || from + need <= total_free);
        if (served && need > 0) {
            const int first = ld_cg(w.first + i);
            int* entry = t.tables + (size_t)(kFork ? r.b[i] : r.a[i]) * t.width;
            for (int k = sub; k < need; k += lanes) {
                const int page = ld_cg(w.free_list + from + k);
                if (first + k < t.width) entry[first + k] = page;
                t.refs[page] = 1;
            }
        }
        if (sub == 0) {
            if (!kFork && served && rows > 0) atomicSub(t.refs + ld_cg(w.src + i), 1);
            w.dst[i] = served && rows > 0 ? ld_cg(w.free_list + from) : -1;
            r.done[i] = served;
            if (kFork) {
                if (need >= 0) t.lens[r.b[i]] = served ? t.lens[r.a[i]] : 0;
            } else if (served) {
                t.lens[r.a[i]] = r.b[i];
            }
        }
    }
}

// The parents' whole pages shared with their children, then the part-full ones copied.  Neighbouring requests of one parent are
// a run: the first of them adds for all.
__global__ void __launch_bounds__(kCopyThreads) fork_share_kernel(const __grid_constant__ PoolSet pools, const PageShape sh, const PageTables t,
                                                                  const PageRequests r, const PageWork w, int chunks) {
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warps = gridDim.x * (kCopyThreads / 32);
    for (long long c = (long long)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); c < (long long)r.n * chunks; c += warps) {
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
    copy_pieces(pools, sh, w.src, w.dst, w.rows, r.n);
}

// ----------------------------------------------------------------------------- compaction
// U pages are in use.  The k-th page in use at or past U goes to the k-th free one below U.
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kClusterThreads)
compact_plan_kernel(const int* refs, int* refs_out, int* page_map, int* used_out, const PageWork w, int num_blocks) {
    __shared__ long long scratch[33];
    __shared__ long long all_used[kClusterCtas];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), tid = threadIdx.x;
    grid_dependency_launch();
    grid_dependency_wait();
    const Slice s = slice_of(num_blocks, rank);
    long long count = 0, here;
    for (int at = s.begin + 4 * tid; at < s.end; at += 4 * kClusterThreads) {
        const int4 v = four_counts(refs, at, num_blocks);
        const int live = min(4, num_blocks - at);       // past the end reads as in use
        count += (v.x > 0) + (v.y > 0) + (v.z > 0) + (v.w > 0) - (4 - live);
    }
    block_scan(count, scratch, here);
    if (tid < kClusterCtas) *cluster.map_shared_rank(&all_used[rank], tid) = here;
    cluster.sync();
    long long before = 0, U = 0;
    for (int c = 0; c < kClusterCtas; ++c) {
        if (c == rank) before = U;
        U += all_used[c];
    }
    // pages in use below U: the holes and the movers are as many, U less those
    __shared__ long long all_low[kClusterCtas];
    count = 0;
    for (int at = s.begin + 4 * tid; at < s.end && at < U; at += 4 * kClusterThreads) {
        const int4 v = four_counts(refs, at, num_blocks);
        count += (at < U && v.x > 0) + (at + 1 < U && v.y > 0) + (at + 2 < U && v.z > 0) + (at + 3 < U && v.w > 0);
    }
    block_scan(count, scratch, here);
    if (tid < kClusterCtas) *cluster.map_shared_rank(&all_low[rank], tid) = here;
    cluster.sync();
    long long low = 0;
    for (int c = 0; c < kClusterCtas; ++c) low += all_low[c];
    for (int base = s.begin; base < s.end; base += 4 * kClusterThreads) {
        const int at = base + 4 * tid;
        int ref[4] = {0, 0, 0, 0};
        if (at < s.end) {
            const int4 v = four_counts(refs, at, num_blocks);
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
    cluster.sync();
    const long long moves = U - low;
    for (long long k = rank * kClusterThreads + tid; k < moves; k += kAll) {
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
                                                                    int rows, int width, int bs) {
    grid_dependency_wait();
    const long long entries = (long long)rows * width;
    for (long long e = (long long)blockIdx.x * kCopyThreads + threadIdx.x; e < entries; e += (long long)gridDim.x * kCopyThreads) {
        const int row = (int)(e / width), k = (int)(e - (long long)row * width), page = tables[e];
        const bool held = (long long)k * bs < lens[row] && in_pool(page, sh.num_blocks);
        tables_out[e] = held ? page_map[page] : page;
    }
    copy_pieces(pools, sh, w.src, w.dst, nullptr, w.first[0]);
}

unsigned copy_ctas(const PageShape& sh, long long pairs) {
    const long long warps = pairs * sh.num_pools * (sh.page_bytes / kPieceBytes), most = (long long)sm_count() * kCopyCtasPerSm;
    const long long ctas = (warps + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
    return (unsigned)(ctas < 1 ? 1 : ctas < most ? ctas : most);
}

}  // namespace

int launch_copy_pages(const PoolSet& pools, const PageShape& sh, const int* src, const int* dst, int n, cudaStream_t stream) {
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    return launch_dependent(copy_pages_kernel, dim3(copy_ctas(sh, n)), dim3(kCopyThreads), 0, stream, pools, sh, src, dst, nullptr, n, true);
}

// Entries of the children's tables up to which the cluster drops them itself.
static constexpr long long kClusterDrop = 16384;

int launch_fork(const PoolSet& pools, const PageShape& sh, const PageTables& t, const PageRequests& r, const PageWork& w, cudaStream_t stream) {
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    const bool drops = (long long)r.n * t.width <= kClusterDrop;
    int rc = OPT_GQA_OK;
    if (!drops) {
        const unsigned x = (unsigned)((t.width + 1023) / 1024);
        rc = launch_dependent(fork_drop_kernel, dim3(x < 64 ? x : 64, (unsigned)r.n), dim3(256), 0, stream, t, r);
        if (rc != OPT_GQA_OK) return rc;
    }
    rc = launch_dependent(give_pages_kernel<true>, dim3(kClusterCtas), dim3(kClusterThreads), 0, stream, t, r, w, drops);
    if (rc != OPT_GQA_OK) return rc;
    return launch_dependent(fork_share_kernel, dim3(copy_ctas(sh, r.n)), dim3(kCopyThreads), 0, stream, pools, sh, t, r, w, (t.width + 127) / 128);
}

int launch_resize(const PoolSet& pools, const PageShape& sh, const PageTables& t, const PageRequests& r, const PageWork& w, cudaStream_t stream) {
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    const int rc = launch_dependent(give_pages_kernel<false>, dim3(kClusterCtas), dim3(kClusterThreads), 0, stream, t, r, w, true);
    if (rc != OPT_GQA_OK) return rc;
    return launch_dependent(copy_pages_kernel, dim3(copy_ctas(sh, r.n)), dim3(kCopyThreads), 0, stream, pools, sh, w.src, w.dst, w.rows, r.n, false);
}

int launch_compact(const PoolSet& pools, const PageShape& sh, const PageTables& t, int* tables_out, int* refs_out, int* page_map, int* used,
                   const PageWork& w, cudaStream_t stream) {
    if (sm_count() <= 0) return OPT_GQA_ERR_CUDA;
    const int rc = launch_dependent(compact_plan_kernel, dim3(kClusterCtas), dim3(kClusterThreads), 0, stream, t.refs, refs_out, page_map, used, w,
                                    t.num_blocks);
    if (rc != OPT_GQA_OK) return rc;
    return launch_dependent(compact_move_kernel, dim3(copy_ctas(sh, t.num_blocks / 2 + 1)), dim3(kCopyThreads), 0, stream, pools, sh, t.tables,
                            tables_out, t.lens, page_map, w, t.rows, t.width, t.bs);
}

}  // namespace optgqa
