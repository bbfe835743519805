// Attention of a chunk of new tokens per sequence over the paged cache, causal, with ALiBi and a local window where asked: one
// token (a decode row), a few (drafts to verify) or many (a prompt's chunk), in one batch.
//
//     out[t, h] = sum_j softmax_j(scale <q_t, k_j> - slope_h (pos_t - j)) v_j,   max(0, pos_t - window + 1) <= j <= pos_t
//
// An item is (sequence, KV head, block of up to 128 rows), a row being (new token, head of the group), over the 64-key tiles
// that some row of the block sees; S = Q K^T and O += P V run on tcgen05 with accumulators in tensor memory, softmax with a
// running maximum by one thread per row.  The items' tiles, laid end to end, are cut into one contiguous range per worker (a CTA,
// two per SM), so that one long context fills the GPU as well as a large ragged batch.  A range covers whole items, written
// out at once, and at its two ends parts of items: normalised partial rows and log-sum-exps in the workspace, two places a worker,
// merged by chunk_merge_kernel.  (The chunked prefill gives a block of rows to one CTA whatever the context: with few new tokens
// most of the GPU is idle.)  Few items are not cut (kCutCost).  Items of few tiles need no list but get a CTA each, and few items of
// longer contexts a cluster each, whose CTAs share the tiles and merge their rows through distributed shared memory (ctas_per_item).
//
// Products take 64 rows for blocks of up to 64, row 16 w + i in lane 32 w + i, so that a block of up to 16 or 32 rows lies in one
// or two row warps: items take the warps in turns, and one block's last product and its storing overlap the next one's first scores.
// (With 128 rows for those of more than 16, run without a pause, 8 drafts behind 16 to 32 k tokens took 74.6 us instead of 72.4, for
// the power; in a graph 66.3 instead of 67.0.)  Warps none of whose rows see a tile skip its softmax.
//
// 32/8 heads, 32 sequences of 3 to 6 new tokens behind 512 to 2048: 34.4 us (152 MB: 23.1 us of copy bandwidth); 32/4 heads, 8 of 8
// behind 16384 to 32768: 67 us (357 MB, 54.5); 64/8 heads, 60 decode rows and 4 chunks of 300 to 512: 97 us (409 MB, 62.3; 115
// without a pause, where the power limit takes the clock down); 32/8 heads, 511 behind 32768: 267 to 277 us (272 GFLOP, 165 at the
// burst rate, 196 at the sustained one; 315 without a pause).  What bounds them: between prologue and tail the cache is read at 6.9 to
// 7.3 TB/s where rows are few; besides that 2 us from the preceding kernel's end to the first scores, 4 to 5 us between the
// workers' mean end and the last one's, 2 us until the merge may read and 3 to 4 us of merge.  Blocks of 128 rows: 1.03 to 1.17 us a
// tile with two CTAs per SM, the tensor pipe 48 % active and, its instructions having a shortest time, 73 % occupied; as the prefill.
// With both kinds on an SM nothing is above 60 %: the chain from a tile's scores over its weights to the score buffer's next use.
//
// Built and not kept (the first two batches above, as the kernel then was): the last quarter of the list in small ranges that a worker
// asks for when it is done (clusterlaunchcontrol; 41 -> 53 us and 67 -> 79: the rings drain at each range); tiles prefetched into L2 (41
// -> 45 to 52, 67 -> 70 to 85: the TMA unit's instructions are what is short); blocks of up to 32 rows spread over all row warps, 16 keys
// each, with the maximum exchanged and the weights in shared memory (the same; the mixed batch 99 -> 123); four stages for heads of
// 64 (the same); fewer registers at launch and setmaxnreg (ptxas spilled 2.4 KB).
//
// Eight warps: 0-3 one thread per row (softmax), 4 the list of pieces and the TMA copies of Q and K, 6 those of V, 5 and 7
// issue S = Q K^T and O += P V.  Every wait is a bounded mbarrier wait.
#include "umma.cuh"

namespace optgqa {

namespace {

constexpr int kRows = kChunkRows;
constexpr int kTN = 64;                    // keys per tile
constexpr int kStages = 2;                 // of the K ring and of the V ring
constexpr int kCtasPerSm = 2;
constexpr int kThreads = 256;
// The cut counts in quarters of a tile's time, tiles at kTileCost and an item at what it costs besides (the next one's Q, the wait for
// its last P V, storing the rows): fitted to the times of 296 workers with different numbers of tiles and pieces, a tile 1.0 to 1.1
// us of any kind (two CTAs per SM), an item 1.2 to 1.6, one of more than 64 rows, which takes the row warps all together, 3.4.
constexpr int kTileCost = 4, kSmallItem = 5, kFullItem = 13;
constexpr int kMinShare = 8;               // a worker's share at least, in the same
constexpr int kNarrowRows = 64;            // up to which the products take 64 rows: row 16 w + i lies in lane 32 w + i
// The second half of the workers begins later, 1 us where the GPU is idle and 4 to 6 where a call follows another (an SM's second
// CTA finds its registers when the merge before is done): what a worker of it has less, and one of the first half more.
constexpr int kLateCost = 5;
// Where there are no more items than workers, nothing is cut -- one item each, and nothing to merge -- if the longest is not much
// above a worker's share: what cutting costs is kCutCost (with blocks of more than 64 rows kCutCostFull), and alone on its
// multiprocessor a worker is a fifth faster.  (In a graph, us, tables so wide that the host does not know, not cut against cut: 128
// items of 9 and 16 tiles 16.3 and 21.9 against 20.5 and 23.9, 256 of 9 and 24 19.6 and 37.0 against 25.7 and 42.1, 32 of 7 and 9
// 13.3 and 14.9 against 13.7 and 13.0, 72 of 128 rows and 9 and 11 tiles 17.2 and 19.0 against 21.2 and 21.6.)
constexpr int kCutCost = 28, kCutCostFull = 36;
constexpr int kDescs = 4;                  // pieces described ahead
constexpr int kDescBytes = 64;
constexpr int kOpens = 1, kContinues = 2, kCloses = 4;      // a worker's flags: see ChunkLayout
constexpr unsigned kFull = 0xffffffffu;
constexpr float kRescaleThreshold = 8.f;   // log2 units: O is rescaled only when a row's maximum grew by more

constexpr int kHalfBytes = kTN * 128;      // one 64-dim column half of a K tile
constexpr int kQHalfBytes = kRows * 128;   // one 64-dim column half of the Q tile
constexpr int kQuarterBytes = 32 * 128;    // a row warp's rows in it
// The ALiBi term inside a tile rides on the tensor core as one more k-step (see prefill_umma.cu): slope / |scale| as
// three bf16 values against the key's index in the tile.
constexpr int kExtRowGroupBytes = 256;
constexpr int kQxBytes = kRows / 8 * kExtRowGroupBytes;
constexpr int kKpBytes = kTN / 8 * kExtRowGroupBytes;
// barriers: q_full[4], q_empty[4], o_empty[4], k_full[], k_empty[], v_full[], v_empty[], s_full[2], p_full[2],
// desc_full[], desc_empty[]
constexpr int kNumBars = 12 + 4 * kStages + 4 + 2 * kDescs;
constexpr int kDescReaders = 7;            // warps that read a descriptor: all but the one that writes it

constexpr int kMaxSplit = 8;               // CTAs that share an item at most
constexpr size_t kSmemPerSm = 228 * 1024;
constexpr double kFarBytes = 126e6;         // what L2 holds
// Contexts, as the host can bound them, up to which more items than a wave may get a CTA each: see ctas_per_item.
constexpr int kOneTiles = 1024 / kTN + 1, kFarTiles = 1536 / kTN + 1;

template <int D>
struct ChLayout {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kQBytes = kHalves * kQHalfBytes;
    static constexpr int kOffQ = 0;
    static constexpr int kOffK = kQBytes;
    static constexpr int kOffV = kOffK + kStages * kTileBytes;
    static constexpr int kOffQx = kOffV + kStages * kTileBytes;
    static constexpr int kOffKp = kOffQx + kQxBytes;
    static constexpr int kOffBar = kOffKp + kKpBytes;
    static constexpr int kOffDesc = kOffBar + kNumBars * 8 + 16;
    static constexpr int kOffParts = kOffDesc + kDescs * kDescBytes;       // of a cluster's item: see merge_cluster
    static constexpr int kSmemBytes = kOffParts + 1024;
    static constexpr int kMostBytes = kSmemBytes + kRows * D * 4 + kMaxSplit * kRows * 4;
};

constexpr uint32_t kColS = 0;              // S buffers at 0 and kTN, P over the first half of its S
constexpr uint32_t kColO = 2 * kTN;
constexpr uint32_t kTmemCols = 256;

struct ChunkParams {
    __nv_bfloat16* out;
    const int32_t* q_start_loc;
    const int32_t* block_tables;
    const int32_t* context_lens;
    const float* slopes;
    int32_t* flags;             // see ChunkLayout, as the parts below
    int4* items;
    float* lse;
    float* part;
    int* status;
    float scale;
    int B, total_q, max_q, max_blocks, Hq, Hkv, bs, bs_log2, window, slot_rows, split, recv_rows;
};

// A sequence of the batch: its rows of q, context, position of its first new token, and its blocks first .. blocks - 1 that see a key.
struct Seq {
    int q0, q, n, pos0, first, blocks;
};

template <int TQ>
__device__ __forceinline__ Seq sequence(const ChunkParams& p, int s) {
    Seq x;
    // (inside the rows and the promised length, whatever the arrays hold)
    x.q0 = min(max(__ldg(p.q_start_loc + s), 0), p.total_q);
    const int q = max(min(__ldg(p.q_start_loc + s + 1), p.total_q) - x.q0, 0);
    x.q = min(q, p.max_q);
    x.n = max(__ldg(p.context_lens + s), 0);
    x.pos0 = x.n - q;
    x.blocks = x.pos0 + x.q > 0 ? (x.q + TQ - 1) / TQ : 0;      // (of more tokens than promised the first may all lie before position 0)
    x.first = x.pos0 < 0 ? min(-x.pos0 / TQ, x.blocks) : 0;
    return x;
}

__device__ __forceinline__ int linear_cta() { return blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z); }

// ----------------------------------------------------------------------------- an item shared by a cluster
// The CTAs of a cluster have a share of the item's tiles each and merge their rows through distributed shared memory: CTA c gets
// every part's columns c D / C and on, and writes them out.  What a CTA receives, behind its own buffers: four columns of a part by
// rows of 16 bytes, and the parts' log-sum-exps.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, int rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}

// 32 columns of a part's row to the CTAs that own them.
template <int D>
__device__ __forceinline__ void send_columns(uint32_t parts, int part, int C, int slot_rows, int row, int col, const float (&o)[32], float inv) {
    const int width = D / C;
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        const int own = (col + e) / width, four = (col + e) % width / 4;
        const uint32_t at = in_cta(parts + ((part * (width / 4) + four) * slot_rows + row) * 16, own);
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(o[e] * inv), "f"(o[e + 1] * inv), "f"(o[e + 2] * inv),
                     "f"(o[e + 3] * inv)
                     : "memory");
    }
}

// The parts' rows joined: this CTA's columns, a thread a row of eight.
template <int D, int G>
__device__ __forceinline__ void merge_cluster(const char* received, __nv_bfloat16* out, int rank, int C, int parts, int slot_rows, int rows,
                                              int q0, int pos0, int kvh, int Hq, int total_q) {
    const int width = D / C, padded = (rows + 15) / 16 * 16;
    const float4* x = reinterpret_cast<const float4*>(received);
    const float* lse = reinterpret_cast<const float*>(received + (size_t)slot_rows * D * 4);
    for (int i = threadIdx.x; i < padded * (width / 8); i += kThreads) {
        const int row = i % padded, eight = i / padded, t = q0 + row / G;
        if (row >= rows || pos0 + row / G < 0 || (unsigned)t >= (unsigned)total_q) continue;
        float top = -INFINITY, den = 0.f, num[8] = {};
        for (int u = 0; u < parts; ++u) top = fmaxf(top, lse[u * slot_rows + row]);
#pragma unroll 2
        for (int u = 0; u < parts; ++u) {
            const float l = lse[u * slot_rows + row];
            if (l == -INFINITY) continue;               // a part the row saw nothing of: its values mean nothing (a NaN is carried on)
            const float w = ex2((l - top) * kLog2e);
            const float4 a = x[(u * (width / 4) + 2 * eight) * slot_rows + row], b = x[(u * (width / 4) + 2 * eight + 1) * slot_rows + row];
            den += w;
            num[0] = fmaf(w, a.x, num[0]), num[1] = fmaf(w, a.y, num[1]), num[2] = fmaf(w, a.z, num[2]), num[3] = fmaf(w, a.w, num[3]);
            num[4] = fmaf(w, b.x, num[4]), num[5] = fmaf(w, b.y, num[5]), num[6] = fmaf(w, b.z, num[6]), num[7] = fmaf(w, b.w, num[7]);
        }
        const float inv = 1.f / den;
        *reinterpret_cast<uint4*>(out + ((size_t)t * Hq + kvh * G + row % G) * D + rank * width + eight * 8) =
            make_uint4(pack2(num[0] * inv, num[1] * inv), pack2(num[2] * inv, num[3] * inv), pack2(num[4] * inv, num[5] * inv),
                       pack2(num[6] * inv, num[7] * inv));
    }
}

// The tiles lo .. hi - 1 that the rows of block mt see.
template <int TQ>
__device__ __forceinline__ void block_tiles(const Seq& x, int mt, int window, int& lo, int& hi) {
    hi = (x.pos0 + min((mt + 1) * TQ, x.q) - 1) / kTN + 1;
    lo = window > 0 ? max(0, max(0, x.pos0 + mt * TQ) - window + 1) / kTN : 0;      // (from 0 on no window takes it past 32 bits)
}

// What the other warps need to know of a piece.
struct Piece {
    int q0, rows, kvh, s;           // row of q of the block's first token, rows, KV head, sequence
    int tile_hi, len, n, slot;      // last tile and how many, context, place in the workspace (-1: the whole item, rows to out)
    int pos0, warp0, once, pad;     // position of the block's first token; the row warp whose lanes are the first rows;
                                    // whether the tiles are read for this block alone
};

// Where a CTA's items come from.  kList: its share of the list; kOne: the grid, an item each; kShared: the same with an item's tiles
// shared by the CTAs of a cluster, p.split of them.  Kernels of their own: with the clusters' code in the list's, that took 3 to 9 %
// longer, with the single items' 1 to 2 %.
enum Route { kList, kOne, kShared };
template <int D, int G, Route kRoute>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
chunk_kernel(const __grid_constant__ CUtensorMap map_q32, const __grid_constant__ CUtensorMap map_q16,
             const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const ChunkParams p) {
    using L = ChLayout<D>;
    constexpr int kTileBytes = L::kTileBytes, kOffQ = L::kOffQ, kOffK = L::kOffK, kOffV = L::kOffV, kOffQx = L::kOffQx,
                  kOffKp = L::kOffKp;
    constexpr int TQ = kRows / G;          // tokens per block
    extern __shared__ char smem_raw[];
    char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
    uint64_t* q_full = bars;                    // [4], by the block's first row warp
    uint64_t* q_empty = bars + 4;
    uint64_t* o_empty = bars + 8;               // [4], one per row warp
    uint64_t* k_full = bars + 12;
    uint64_t* k_empty = k_full + kStages;
    uint64_t* v_full = k_empty + kStages;
    uint64_t* v_empty = v_full + kStages;
    uint64_t* s_full = v_empty + kStages;
    uint64_t* p_full = s_full + 2;
    uint64_t* desc_full = p_full + 2;
    uint64_t* desc_empty = desc_full + kDescs;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
    // units and blocks (of one head) of the sequences before each thread's chunk, from its warp's first on, and of each warp's
    // chunks, and the most units of a block; gone once the K ring is in use
    long long* c_units = reinterpret_cast<long long*>(smem + kOffK);
    long long* w_units = c_units + kThreads;
    long long* c_blocks = w_units + kThreads / 32;
    long long* w_blocks = c_blocks + kThreads;
    int* w_most = reinterpret_cast<int*>(w_blocks + kThreads / 32);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 192) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q32) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q16) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    auto item_cost = [&](const Seq& x) { return x.q * G > kNarrowRows ? kFullItem : kSmallItem; };
    auto seq_units = [&](const Seq& x, int& most) {
        long long sum = 0;
        for (int mt = x.first; mt < x.blocks; ++mt) {
            int lo, hi;
            block_tiles<TQ>(x, mt, p.window, lo, hi);
            sum += hi - lo;
            most = max(most, (hi - lo) * kTileCost + item_cost(x));
        }
        return sum * kTileCost + (x.blocks - x.first) * item_cost(x);
    };

    // ------------------------------------------------------------------ the items (the index arrays are read before the
    // wait for the preceding kernel: see the ordering contract in the header)
    const int chunk = (p.B + kThreads - 1) / kThreads;          // sequences per thread
    if constexpr (kRoute == kList) {
        long long units = 0, blocks = 0;
        int most = 0;
        for (int s = threadIdx.x * chunk; s < min((int)(threadIdx.x + 1) * chunk, p.B); ++s) {
            const Seq x = sequence<TQ>(p, s);
            units += seq_units(x, most);
            blocks += x.blocks - x.first;
        }
        long long upto = units, upto_b = blocks;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(kFull, upto, o), b = __shfl_up_sync(kFull, upto_b, o);
            if (lane >= o) upto += v, upto_b += b;
        }
        most = __reduce_max_sync(kFull, most);
        c_units[threadIdx.x] = upto - units;
        c_blocks[threadIdx.x] = upto_b - blocks;
        if (lane == 31) {
            w_units[warp] = upto;
            w_blocks[warp] = upto_b;
            w_most[warp] = most;
        }
    }
    if (threadIdx.x == 128) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
            mbar_init(&o_empty[i], 32);
        }
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], 1);
            mbar_init(&v_full[i], 1);
            mbar_init(&v_empty[i], 1);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], kRows);
        }
#pragma unroll
        for (int i = 0; i < kDescs; ++i) {
            mbar_init(&desc_full[i], 1);
            mbar_init(&desc_empty[i], kDescReaders);
        }
        tmem_slot[1] = 0;
        fence_barrier_init();
    }
    // The scale may have any sign (see prefill_umma.cu).
    const float sabs = p.scale == 0.f ? 1.f : fabsf(p.scale);
    const bool alibi = p.slopes != nullptr || p.scale == 0.f;
    if (alibi && threadIdx.x >= kThreads - kTN) {
        const int e = threadIdx.x - (kThreads - kTN);
        const uint32_t eb = __bfloat16_as_ushort(__float2bfloat16_rn((float)e));      // exact: e < 256
        char* row = smem + kOffKp + (e >> 3) * kExtRowGroupBytes + (e & 7) * 16;
        *reinterpret_cast<uint4*>(row) = make_uint4(eb | (eb << 16), eb, 0u, 0u);
        *reinterpret_cast<uint4*>(row + 128) = make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async();
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_proxy_async();                // c_units lies where the copies of K will land
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_dependency_launch();           // not before this CTA has its tensor memory: a later grid's could take it and wait for this one
    const uint32_t received = smem_u32(smem + L::kOffParts);
    if constexpr (kRoute == kShared) cluster_arrive();

    if (warp == 4) {
        // ------------------------------------------------------------------ the list of pieces, Q and K
        // (sequence, block, KV head), KV head fastest: with ALiBi the heads' tiles cost differently (weights that are all zero
        // need no exponentials), and workers side by side walk the same keys
        Seq x = {};
        int s = 0, kvh = 0, mt = 0, jt = 0, t0 = 0, t1 = 0;        // the item's tiles t0 .. t1 - 1, jt of them done
        long long pos = 0, end = 0;                                 // in the list: the next tile's place, and the share's end
        const int me = blockIdx.x;
        bool whole = false;                                         // items are not cut: the list counts them, not their units
        // Where the share begins in the list.  (In 32 bits where they do: N is int or long long.)
        auto locate = [&](auto total_units) {
            using N = decltype(total_units);
            const N total = total_units;
            const int W = (int)max(min((N)gridDim.x, whole ? total : total / kMinShare), (N)1);
            const int skew = !whole && total / W >= 4 * kLateCost ? kLateCost : 0;
            auto share = [&](int i) { return (N)share_at(total, i, W) + skew * min(i, W - i); };
            const N begin = share(min(me, W));
            end = share(min(me + 1, W));
            pos = end;
            if (begin >= end) return;
            // the last thread's chunk that begins at or before the share, and its begin
            const long long *warps = whole ? w_blocks : w_units, *chunks = whole ? c_blocks : c_units;
            const N sum = (N)warps[lane & 7] * p.Hkv;
            N upto = sum;
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) {
                const N v = __shfl_up_sync(kFull, upto, o, 8);
                if ((lane & 7) >= o) upto += v;
            }
            int at = __popc(__ballot_sync(kFull, upto - sum <= begin) & 0xff) - 1;
            N before = __shfl_sync(kFull, upto - sum, at);
            const N mine = before + (N)chunks[at * 32 + lane] * p.Hkv;
            const int in_warp = __popc(__ballot_sync(kFull, mine <= begin)) - 1;
            before = __shfl_sync(kFull, mine, in_warp);
            at = at * 32 + in_warp;
            int most = 0;
            for (s = at * chunk; s < p.B; ++s) {
                x = sequence<TQ>(p, s);
                const N all = (whole ? (N)(x.blocks - x.first) : (N)seq_units(x, most)) * p.Hkv;
                if (before + all > begin) break;
                before += all;
            }
            if (s >= p.B) return;                                   // (cannot happen: the shares end where the items do)
            N r = begin - before;
            int units;
            for (mt = x.first;; ++mt) {
                block_tiles<TQ>(x, mt, p.window, t0, t1);
                units = whole ? 1 : (t1 - t0) * kTileCost + item_cost(x);
                if (r < units * (N)p.Hkv || mt == x.blocks - 1) break;
                r -= units * (N)p.Hkv;
            }
            kvh = (int)(r / units);
            pos = begin;
            if (whole) return;
            // an item's tile j lies its cost + j tiles behind its begin; a share has those whose place lies in it
            const int in_item = (int)(r - (N)kvh * units) - item_cost(x);
            jt = max((in_item + kTileCost - 1) / kTileCost, 0);
            pos = begin + jt * kTileCost - in_item;
        };
        // on to the next item, where there is one
        auto next_item = [&]() {
            jt = 0;
            if (pos >= end) return;
            if (++kvh == p.Hkv) {
                kvh = 0;
                if (++mt == x.blocks) {
                    for (++s; s < p.B; ++s) {
                        x = sequence<TQ>(p, s);
                        if (x.first < x.blocks) break;
                    }
                    if (s == p.B) pos = end;            // cannot happen: the shares end where the items do
                    mt = x.first;
                }
                block_tiles<TQ>(x, mt, p.window, t0, t1);
            }
            if (!whole) pos += item_cost(x);
        };
        if constexpr (kRoute != kList) {
            const int split = kRoute == kShared ? p.split : 1;
            s = blockIdx.z;
            kvh = blockIdx.y;
            x = sequence<TQ>(p, s);
            mt = blockIdx.x / split;
            if (mt >= x.first && mt < x.blocks) {
                block_tiles<TQ>(x, mt, p.window, t0, t1);
                // this CTA's share of them
                const int parts = min(split, t1 - t0), part = blockIdx.x % split;
                if (part < parts) {
                    jt = (t1 - t0) * part / parts;
                    end = ((t1 - t0) * (part + 1) / parts - jt) * kTileCost;
                }
            }
        } else {
            long long total = 0, items = 0;
            int most = 0;
            for (int w = 0; w < kThreads / 32; ++w) {
                total += w_units[w];
                items += w_blocks[w];
                most = max(most, w_most[w]);
            }
            total *= p.Hkv;
            items *= p.Hkv;
            const int alone = 2 * items <= gridDim.x ? most - most / 5 : most;
            whole = items <= gridDim.x && alone <= total / gridDim.x + (p.max_q > kNarrowRows / G ? kCutCostFull : kCutCost);
            if (whole) total = items;
            if (total < 0x40000000) locate((int)total);
            else locate(total);
            if (jt > 0 && jt == t1 - t0) next_item();                  // the share begins inside an item's last tile
        }
        fence_proxy_async();
        __syncwarp();
        const int slices = kTN >> p.bs_log2, sub = lane & (slices - 1), hf = lane >> (6 - p.bs_log2);
        const bool issues = lane < slices * L::kHalves;
        char* ring = smem + kOffK + hf * kHalfBytes + sub * p.bs * 128;
        int st = 0;
        uint32_t ph = 1;                    // parity of a stage's last release (none yet: passes)
        const uint64_t read_once = l2_policy_evict_first(), read_again = l2_policy_evict_normal();
        uint32_t owner = 0xffff, q_ph = 0;  // per quarter of Q (4 bits) whose block it holds (by its first row warp; f: none that
                                            // has not been seen done), and the parity of that barrier's next release
        int next_warp = 0;
        // what the merge needs to know: the parts of items at the share's begin and end
        int4 first_item = make_int4(0, 0, 0, 0), last_item = first_item;
        int flags = 0;
        bool waited = false;
        for (int pc = 0;; ++pc) {
            const unsigned room = (unsigned)max(min((end - pos + kTileCost - 1) / kTileCost, (long long)0x3fffffff), 0ll);
            const int len = whole ? (pos < end ? t1 - t0 : 0) : (int)min((unsigned)(t1 - t0 - jt), room);    // 0: the end
            const int rows = min(TQ, x.q - mt * TQ) * G, wide = rows > 32 ? 4 : rows > 16 ? 2 : 1;
            const bool opens = jt == 0, closes = jt + len == t1 - t0, once = x.blocks - x.first <= 1;
            const int tile_hi = t0 + jt + len - 1, q0 = x.q0 + mt * TQ, pos0 = x.pos0 + mt * TQ;
            // the row warps in turns
            const int warp0 = ((next_warp + wide - 1) & ~(wide - 1)) & 3;
            next_warp = warp0 + wide;
            bool ok = __all_sync(kFull, wait_for(&desc_empty[pc % kDescs], ((pc / kDescs) & 1) ^ 1, p.status));
            if (!ok) break;
            const int slot = opens && closes ? -1 : 2 * me + (opens ? 1 : 0);
            if (lane == 0) {
                int4* d = reinterpret_cast<int4*>(smem + L::kOffDesc + kDescBytes * (pc % kDescs));
                d[0] = make_int4(q0, rows, kvh, s);
                d[1] = make_int4(tile_hi, len, x.n, slot);
                d[2] = make_int4(pos0, warp0, once, 0);
                mbar_arrive(&desc_full[pc % kDescs]);
            }
            if (len == 0) break;
            if (!opens) flags = closes ? kCloses : kContinues, first_item = make_int4(q0, rows, kvh, pos0);
            else if (!closes) flags |= kOpens, last_item = make_int4(q0, rows, kvh, pos0);
            const int32_t* table = p.block_tables + (size_t)s * p.max_blocks;
            const int pages = min((x.n + p.bs - 1) >> p.bs_log2, p.max_blocks);       // the table is not read past them
            auto page_of = [&](int j) {
                const int i = (tile_hi - j) * slices + sub;
                return issues && i < pages ? __ldg(table + i) : 0;
            };
            int page = page_of(0);
#pragma unroll 1
            for (int j = 0; j < len; ++j) {
                const int row = (page * p.Hkv + kvh) * p.bs;                       // row of the [rows, D] view
                const int live = min(slices, (x.n - (tile_hi - j) * kTN + p.bs - 1) >> p.bs_log2);    // slices that hold keys
                page = j + 1 < len ? page_of(j + 1) : 0;
                ok = __all_sync(kFull, wait_for(&k_empty[st], ph, p.status));
                if (!ok) break;
                // q and the cache may still be written, the workspace still read, by the preceding kernel
                if (!waited) grid_dependency_wait();
                waited = true;
                if (lane == 0) mbar_expect_tx(&k_full[st], (uint32_t)(live * p.bs * D * 2));
                __syncwarp();
                if (issues && sub < live) tma_load_2d_hint(ring + st * kTileBytes, &map_k, 64 * hf, row, &k_full[st], once ? read_once : read_again);
                if (++st == kStages) st = 0, ph ^= 1;
                if (j == 0) {
                    // Q behind the first K tile, once the scores of the blocks whose rows lie there are done
#pragma unroll 1
                    for (int w = warp0; w < warp0 + wide; ++w) {
                        const uint32_t o = owner >> (4 * w) & 15;
                        if (o == 15) continue;
                        ok = ok && __all_sync(kFull, wait_for(&q_empty[o], q_ph >> o & 1, p.status));
                        q_ph ^= 1u << o;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if ((owner >> (4 * i) & 15) == o) owner |= 15u << (4 * i);
                    }
                    if (!ok) break;
#pragma unroll 1
                    for (int w = warp0; w < warp0 + wide; ++w) owner = (owner & ~(15u << (4 * w))) | (uint32_t)warp0 << (4 * w);
                    if (lane == 0) {
                        // boxes of 16 rows (or 32): rows past the block's are others' or zeros and reach no live row
                        const bool narrow = rows <= kNarrowRows;
                        const int box = narrow ? 16 : 32;
                        mbar_expect_tx(&q_full[warp0], (uint32_t)(wide * box * D * 2));
#pragma unroll 1
                        for (int w = 0; w < wide; ++w)
#pragma unroll
                            for (int h = 0; h < L::kHalves; ++h)
                                tma_load_3d(smem + kOffQ + h * kQHalfBytes + warp0 * kQuarterBytes + w * box * 128, narrow ? &map_q16 : &map_q32,
                                            64 * h, kvh * G, q0 + w * (box / G), &q_full[warp0]);
                    }
                }
            }
            if (!ok) break;
            pos += whole ? 1 : len * kTileCost;
            next_item();
        }
        if (!waited) grid_dependency_wait();
        if (kRoute == kList && lane == 0) {
            p.flags[me] = flags;
            p.items[2 * me] = first_item;
            p.items[2 * me + 1] = last_item;
        }
    } else {
        // before any wait with a limit: what the producers wait for may take as long as it likes
        grid_dependency_wait();
        Piece d;
        auto read_piece = [&](int pc) {
            const uint32_t at = smem_u32(smem + L::kOffDesc) + kDescBytes * (pc % kDescs);
            auto load = [&](uint32_t from, int& x, int& y, int& z, int& w) {
                asm volatile("ld.volatile.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(x), "=r"(y), "=r"(z), "=r"(w) : "r"(from));
            };
            load(at, d.q0, d.rows, d.kvh, d.s);
            load(at + 16, d.tile_hi, d.len, d.n, d.slot);
            load(at + 32, d.pos0, d.warp0, d.once, d.pad);
        };
        auto release_piece = [&](int pc) {
            __syncwarp();
            if (lane == 0) mbar_arrive(&desc_empty[pc % kDescs]);
        };
        // what every other warp does first with the next piece; false at the end of the list
        auto next_piece = [&](int pc, bool& ok, bool keep = false) -> bool {
            ok = __all_sync(kFull, wait_for(&desc_full[pc % kDescs], (pc / kDescs) & 1, p.status));
            if (!ok) return false;
            read_piece(pc);
            if (!keep) release_piece(pc);
            return d.len > 0;
        };
        bool ok = true;
        if (warp == 6) {
            // -------------------------------------------------------------- V
            // A box is all of a slice (the bs tokens of a page), half after half: see the issuing thread for the layout.
            const int slices = kTN >> p.bs_log2, sub = lane & (slices - 1);
            const bool issues = lane < slices;
            char* ring = smem + kOffV + sub * p.bs * (D * 2);
            int st = 0;
            uint32_t ph = 1;
            for (int pc = 0; next_piece(pc, ok); ++pc) {
                const uint64_t policy = d.once ? l2_policy_evict_first() : l2_policy_evict_normal();
                const int32_t* table = p.block_tables + (size_t)d.s * p.max_blocks;
                const int pages = min((d.n + p.bs - 1) >> p.bs_log2, p.max_blocks);
                auto page_of = [&](int j) {
                    const int i = (d.tile_hi - j) * slices + sub;
                    return issues && i < pages ? __ldg(table + i) : 0;
                };
                int page = page_of(0);
#pragma unroll 1
                for (int j = 0; j < d.len; ++j) {
                    const int row = (page * p.Hkv + d.kvh) * p.bs;
                    const int live = min(slices, (d.n - (d.tile_hi - j) * kTN + p.bs - 1) >> p.bs_log2);
                    page = j + 1 < d.len ? page_of(j + 1) : 0;
                    ok = __all_sync(kFull, wait_for(&v_empty[st], ph, p.status));
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(&v_full[st], (uint32_t)(live * p.bs * D * 2));
                    __syncwarp();
                    if (issues && sub < live) tma_load_3d_hint(ring + st * kTileBytes, &map_v, 0, row, 0, &v_full[st], policy);
                    if (++st == kStages) st = 0, ph ^= 1;
                }
                if (!ok) break;
            }
        } else if (warp == 5) {
            // -------------------------------------------------------------- one thread issues S = Q K^T
            const bool negate = p.scale < 0.f;
            const bool dots = p.scale != 0.f;
            const uint64_t q_desc0 = smem_desc(smem_u32(smem + kOffQ), 16, 1024);
            const uint64_t k_desc0 = smem_desc(smem_u32(smem + kOffK), 16, 1024);
            const uint64_t qx_desc = smem_desc_plain(smem_u32(smem + kOffQx), 128, kExtRowGroupBytes);
            const uint64_t kp_desc = smem_desc_plain(smem_u32(smem + kOffKp), 128, kExtRowGroupBytes);
            int it = 0, st = 0, qx_kvh = -1;
            uint32_t ph = 0, q_ph = 0;          // q_ph: per quarter of Q the parity of its next filling
            uint64_t* last_q = nullptr;         // where the piece before says that its scores are done, and the parity of that
            uint32_t last_ph = 0;
            for (int pc = 0; next_piece(pc, ok); ++pc) {
                const int w0 = d.warp0;
                if (alibi && d.kvh != qx_kvh) {
                    // The ALiBi step's operand for this KV head: slope / |scale| as a sum of three bf16 values, the rows a head
                    // each in turn.  Nothing reads the one before once that piece's last scores are there.
                    if (pc > 0) ok = __all_sync(kFull, wait_for(last_q, last_ph, p.status));
                    if (!ok) break;
                    qx_kvh = d.kvh;
#pragma unroll 1
                    for (int r = lane; r < kRows; r += 32) {
                        const float a = p.slopes ? __ldg(p.slopes + d.kvh * G + r % G) / sabs : 0.f;
                        const __nv_bfloat16 a0 = __float2bfloat16_rn(a);
                        const __nv_bfloat16 a1 = __float2bfloat16_rn(a - __bfloat162float(a0));
                        const __nv_bfloat16 a2 = __float2bfloat16_rn(a - __bfloat162float(a0) - __bfloat162float(a1));
                        char* row = smem + kOffQx + (r >> 3) * kExtRowGroupBytes + (r & 7) * 16;
                        *reinterpret_cast<uint4*>(row) = make_uint4((uint32_t)__bfloat16_as_ushort(a0) | ((uint32_t)__bfloat16_as_ushort(a1) << 16),
                                                                    (uint32_t)__bfloat16_as_ushort(a2), 0u, 0u);
                        *reinterpret_cast<uint4*>(row + 128) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    fence_proxy_async();
                    __syncwarp();
                }
                // products of 64 rows: Q begins so that their rows 16 w0 .. 16 w0 + 15 are the quarter's first
                const bool narrow = d.rows <= kNarrowRows;
                const uint64_t qd = desc_advance(q_desc0, narrow ? w0 * (kQuarterBytes - 16 * 128) : 0);
                const uint32_t idesc_s = narrow ? instr_desc(false, kTN, false, 64) : instr_desc(false, kTN);
                const uint32_t idesc_qk = idesc_s | (negate ? instr_desc(false, kTN, true) ^ instr_desc(false, kTN) : 0u);
                if (lane == 0) {
                    ok = wait_for(&q_full[w0], q_ph >> w0 & 1, p.status);
#pragma unroll 1
                    for (int j = 0; ok && j < d.len; ++j, ++it) {
                        const int sb = it & 1;
                        // the score buffer is free once the P V of the tile before the last one has read its weights there
                        // (kStages is 2: that tile's V stage is this tile's)
                        if (it >= 2) ok = wait_for(&v_empty[st], ph ^ 1, p.status);
                        ok = ok && wait_for(&k_full[st], ph, p.status);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t kd = desc_advance(k_desc0, st * kTileBytes);
                        const uint32_t s_tmem = tmem_base + kColS + sb * kTN;
                        if (dots) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                umma_ss(s_tmem, desc_advance(qd, (ks >> 2) * kQHalfBytes + (ks & 3) * 32),
                                        desc_advance(kd, (ks >> 2) * kHalfBytes + (ks & 3) * 32), idesc_qk, ks > 0);
                        }
                        if (alibi) umma_ss(s_tmem, qx_desc, kp_desc, idesc_s, dots);
                        tc_commit(&s_full[sb]);
                        tc_commit(&k_empty[st]);
                        if (j == d.len - 1) tc_commit(&q_empty[w0]);
                        if (++st == kStages) st = 0, ph ^= 1;
                    }
                }
                ok = __all_sync(kFull, ok);
                if (!ok) break;
                last_q = &q_empty[w0];
                last_ph = q_ph >> w0 & 1;
                q_ph ^= 1u << w0;
            }
        } else if (warp == 7) {
            // -------------------------------------------------------------- one thread issues O (+)= P V
            // V is MN-major, in slices of bs keys with the 64-dim halves of a slice side by side: halves bs * 128 bytes
            // apart (leading offset), groups of 8 keys 1 KiB apart (stride offset), slices bs * D * 2 bytes.
            const uint64_t v_desc0 = smem_desc(smem_u32(smem + kOffV), p.bs * 128, 1024);
            const uint32_t half_slice = p.bs == 16 ? 16 * D * 2 : 2048;     // from 16 keys to the next 16 of the same 32
            int it = 0, st = 0;
            uint32_t ph = 0;
            uint32_t reading = 0, o_ph = 0;     // row warps that read the piece before; per row warp the parity of its next reading
            for (int pc = 0; next_piece(pc, ok); ++pc) {
                const uint32_t idesc_pv = d.rows <= kNarrowRows ? instr_desc(true, D, false, 64) : instr_desc(true, D);
#pragma unroll 1
                for (int j = 0; j < d.len; ++j, ++it) {
                    const int sb = it & 1, live = d.n - (d.tile_hi - j) * kTN;      // keys of the tile that exist
                    ok = __all_sync(kFull, wait_for(&v_full[st], ph, p.status));
                    if (!ok) break;
                    if (live < kTN) {
                        // Rows past the sequence's end hold whatever the page held, or stale shared memory where no page
                        // exists: zero them, so that a weight of 0 times garbage cannot be NaN.
#pragma unroll 1
                        for (int r = live + (lane >> 3); r < kTN; r += 4) {
                            char* vrow = smem + kOffV + st * kTileBytes + (r >> p.bs_log2 << p.bs_log2) * (D * 2) + (r & (p.bs - 1)) * 128 + (lane & 7) * 16;
#pragma unroll
                            for (int b = 0; b < L::kHalves; ++b)
                                *reinterpret_cast<uint4*>(vrow + b * p.bs * 128) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async();
                        __syncwarp();
                    }
                    if (lane == 0) {
                        ok = wait_for(&p_full[sb], (it >> 1) & 1, p.status);
                        if (j == 0) {           // O of the piece before has been read
#pragma unroll 1
                            for (int w = 0; w < 4; ++w)
                                if (reading >> w & 1) ok = ok && wait_for(&o_empty[w], o_ph >> w & 1, p.status);
                            o_ph ^= reading;
                        }
                        if (ok) {
                            tc_fence_after();
                            const uint64_t vd = desc_advance(v_desc0, st * kTileBytes);
                            const uint32_t p_tmem = tmem_base + kColS + sb * kTN;
#pragma unroll
                            for (int kk = 0; kk < kTN / 16; ++kk) {
                                const uint32_t at = (kk >> 1) * 32 * (D * 2) + (kk & 1) * half_slice;
                                umma_ts(tmem_base + kColO, p_tmem + kk * 8, desc_advance(vd, at), idesc_pv, j > 0 || kk > 0);
                            }
                            tc_commit(&v_empty[st]);
                        }
                    }
                    ok = __all_sync(kFull, ok);
                    if (!ok) break;
                    if (++st == kStages) st = 0, ph ^= 1;
                }
                if (!ok) break;
                reading = ((1u << (d.rows <= kNarrowRows ? (d.rows + 15) / 16 : (d.rows + 31) / 32)) - 1) << d.warp0;
            }
        } else {
            // -------------------------------------------------------------- one thread per row: softmax, rescale, store
            const int hg = lane % G;                     // (16 is a multiple of G)
            if constexpr (kRoute == kShared) cluster_wait();        // every CTA is there to be written to
            // the thread's row of the block, -1: none
            auto row_of = [&]() {
                const int w = warp - d.warp0;
                const int rr = d.rows > kNarrowRows ? (int)threadIdx.x : lane < 16 && w >= 0 ? 16 * w + lane : -1;
                return rr < d.rows ? rr : -1;
            };
            // rows before position 0 (more new tokens than context: padding) see nothing and are zero
            const int cta = linear_cta(), ctas = gridDim.x * gridDim.y * gridDim.z;
            for (int s = cta * 4 + warp; s < p.B; s += ctas * 4) {
                const Seq x = sequence<TQ>(p, s);
                const int none = min(x.q, -x.pos0);
                uint4* o = reinterpret_cast<uint4*>(p.out + (size_t)x.q0 * p.Hq * D);
                for (long long i = lane; i < (long long)none * p.Hq * (D / 8); i += 32) o[i] = make_uint4(0u, 0u, 0u, 0u);
            }
            const float qscale = sabs * kLog2e;
            const uint32_t lane_addr = tmem_base + ((uint32_t)(warp * 32) << 16);
            int it = 0, st = 0;                     // tile, and the stage and parity of its V
            uint32_t ph = 0;
            // waits for the P V of the tile before this one
            auto prev_pv_done = [&]() {
                const int ps = st == 0 ? kStages - 1 : st - 1;
                return __all_sync(kFull, wait_for(&v_empty[ps], st == 0 ? ph ^ 1 : ph, p.status));
            };
            for (int pc = 0; next_piece(pc, ok, true); ++pc) {
                // the row's position, and the last key before those it sees; a row that is not there sees none
                int pos = -1, lo = -1;
                {
                    const int rr = row_of();
                    if (rr >= 0) {
                        pos = d.pos0 + rr / G;
                        if (p.window > 0) lo = max(max(pos, 0) - p.window, -1);
                    }
                }
                const float slope2 = p.slopes ? __ldg(p.slopes + d.kvh * G + hg) * kLog2e : 0.f;
                float m_used = -INFINITY, l = 0.f;
                bool begun = false;                 // the row saw a tile of the piece
                auto next_tile = [&]() {
                    ++it;
                    if (++st == kStages) st = 0, ph ^= 1;
                };
                for (int j = 0; j < d.len; ++j, next_tile()) {
                    const int sb = it & 1, j0 = (d.tile_hi - j) * kTN;
                    ok = __all_sync(kFull, wait_for(&s_full[sb], (it >> 1) & 1, p.status));
                    if (!ok) break;
                    tc_fence_after();
                    const bool sees = j0 <= pos && j0 + kTN - 1 > lo;
                    if (!__any_sync(kFull, sees || begun)) {
                        // no row of the warp has begun: what the tensor core adds to their O from this tile's scores,
                        // read as if they were weights, is discarded when they do
                        tc_fence_before();
                        mbar_arrive(&p_full[sb]);
                        continue;
                    }
                    const uint32_t s_addr = lane_addr + kColS + sb * kTN;
                    const float bias0 = slope2 * (float)(j0 - pos);       // ALiBi term of the tile's first key
                    float v[kTN / 32][32];
                    {
                        uint32_t raw[kTN / 32][32];
#pragma unroll
                        for (int c = 0; c < kTN / 32; ++c) tmem_ld32_issue(s_addr + c * 32, raw[c]);
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < kTN / 32; ++c) {
                            tmem_pin(raw[c]);
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[c][e] = __uint_as_float(raw[c][e]);
                        }
                    }
                    if (__any_sync(kFull, (sees || begun) && (j0 + kTN - 1 > pos || j0 <= lo))) {
                        // -inf in the place of what the row does not see: both passes then run as they are.  (Rows that have not
                        // begun, or are not there, may weigh what they like: see above.  Without the first condition every tile of a
                        // block whose last warp is part full came here.)
                        const int top = pos - j0, bottom = lo - j0;
#pragma unroll
                        for (int e = 0; e < kTN; ++e)
                            if (e > top || e <= bottom) v[e / 32][e % 32] = -INFINITY;
                    }
                    // (NaN where a score is, so that such a tile is never taken for one whose weights are all zero: its sum
                    // is NaN, and with it the row)
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < kTN / 32; ++c) chunk_max<false, true>(v[c], 0, 0, 0, mx);
                    const float m_tile = fmaf(max3_nan(max3_nan(mx[0], mx[1], mx[2]), mx[3], mx[3]), qscale, bias0);
                    // the running maximum moves (and l and O are rescaled) only when it grew by more than the threshold,
                    // and at the row's first tile
                    const bool begins = sees && m_used == -INFINITY;
                    const bool need = sees && m_tile > m_used + kRescaleThreshold;
                    const float m_new = need ? m_tile : m_used;
                    const float f = need ? ex2(m_used - m_new) : 1.f;
                    if (j > 0 && __any_sync(kFull, need || begins)) {
                        ok = prev_pv_done();
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            float o[32];
                            uint32_t w[32];
                            tmem_ld32(lane_addr + kColO + c * 32, o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) w[e] = begins ? 0u : __float_as_uint(o[e] * f);
                            tmem_st32(lane_addr + kColO + c * 32, w);
                        }
                    }
                    begun |= sees;
                    m_used = m_new;
                    l *= f;
                    const float m_sub = m_used == -INFINITY ? 0.f : m_used;
                    const float bias_m = bias0 - m_sub;
                    // every weight of the tile is exactly zero (see prefill_umma.cu), or the row does not see it
                    const bool all_zero = __all_sync(kFull, !sees || m_tile - m_used < -127.f);
                    if (all_zero) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[e] = 0u;
#pragma unroll
                        for (int c = 0; c < kTN / 32; ++c) tmem_st16(s_addr + c * 16, w);
                    } else {
                        float sum = 0.f;
#pragma unroll
                        for (int c = 0; c < kTN / 32; ++c) {
                            uint32_t w[16];
                            sum += chunk_exp<false, true>(v[c], qscale, bias_m, 0, 0, 0, w);
                            tmem_st16(s_addr + c * 16, w);
                        }
                        if (sees) l += sum;
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&p_full[sb]);
                }
                if (!ok) break;

                // ---- the piece is complete once its last P V is: normalise, store, hand O back
                read_piece(pc);             // (again, rather than in registers meanwhile)
                const int rr = row_of();
                const bool valid = rr >= 0;
                if (__any_sync(kFull, valid)) {
                    ok = prev_pv_done();
                    if (!ok) break;
                    tc_fence_after();
                    const float inv = 1.f / l;
                    __nv_bfloat16* orow = p.out + ((size_t)(d.q0 + rr / G) * p.Hq + d.kvh * G + hg) * D;
                    const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31) == 0;
                    // a part is [D][rows], so that 32 neighbouring rows are one line
                    float* part = p.part + (size_t)d.slot * D * p.slot_rows + rr;
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        float o[32];
                        tmem_ld32(lane_addr + kColO + c * 32, o);
                        if (c == D / 32 - 1) {                      // the next piece may overwrite O
                            tc_fence_before();
                            mbar_arrive(&o_empty[warp]);
                        }
                        if (begun && d.slot < 0) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                uint32_t w[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) w[i] = pack2(o[16 * e + 2 * i] * inv, o[16 * e + 2 * i + 1] * inv);
                                st_global_32(orow + c * 32 + e * 16, w, wide);
                            }
                        } else if (begun && kRoute == kShared) {
                            send_columns<D>(received, blockIdx.x % p.split, p.split, p.recv_rows, rr, c * 32, o, inv);
                        } else if (begun) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) part[(size_t)(c * 32 + e) * p.slot_rows] = o[e] * inv;
                        }
                    }
                    // a row that saw nothing of the piece: weight zero
                    if (valid && d.slot >= 0) {
                        const float lse = begun ? (m_used + lg2(l)) * kLn2 : -INFINITY;
                        if constexpr (kRoute == kShared) {
                            const uint32_t at = received + p.recv_rows * D * 4 + (blockIdx.x % p.split * p.recv_rows + rr) * 4;
                            for (int c = 0; c < p.split; ++c) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(in_cta(at, c)), "f"(lse) : "memory");
                        } else {
                            p.lse[(size_t)d.slot * p.slot_rows + rr] = lse;
                        }
                    }
                }
                release_piece(pc);
            }
        }
    }

    if constexpr (kRoute == kShared) {
        __syncwarp();
        if (warp >= 4) cluster_wait();
        cluster_arrive();                   // (this warp's rows are where they are merged)
    }
    // ---- every role is done with tensor memory: give it back (after a wait that gave up, let what is in flight drain)
    if (*reinterpret_cast<volatile int*>(p.status) != 0) tmem_slot[1] = 1;
    tc_fence_before();
    __syncthreads();
    if (tmem_slot[1]) {
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
    }

    if constexpr (kRoute == kShared) {
        const Seq x = sequence<TQ>(p, blockIdx.z);
        const int mt = blockIdx.x / p.split;
        int t0 = 0, t1 = 0;
        if (mt >= x.first && mt < x.blocks) block_tiles<TQ>(x, mt, p.window, t0, t1);
        const int parts = min(p.split, t1 - t0);
        __syncwarp();
        cluster_wait();                     // (and only then may a CTA end: the others write into it)
        if (parts > 1)
            merge_cluster<D, G>(smem + L::kOffParts, p.out, blockIdx.x % p.split, p.split, parts, p.recv_rows, min(TQ, x.q - mt * TQ) * G,
                                x.q0 + mt * TQ, x.pos0 + mt * TQ, blockIdx.y, p.Hq, p.total_q);
    }
}

// ----------------------------------------------------------------------------- merge
// An item in parts is the last piece of one worker, the leader, and the first ones of the workers behind it up to the one that
// closes it.  A CTA stands in the place of each worker (so that the grid is one wave, and the next kernel's CTAs may begin beside
// it), half its warps for the item of the worker's first piece, half for that of its last; an item is merged by the warps of all its
// parts together, in units of 32 rows times 4 C columns.  A thread has four rows and C columns; kBatch parts are requested together.
constexpr int kMergeWarps = 16;

struct ChunkMergeParams {
    __nv_bfloat16* out;
    const int32_t* flags;
    const int4* items;
    const float* lse;
    const float* part;
    int W, Hq, total_q, slot_rows;
};

template <int D, int G, int C, int kBatch>
__device__ __forceinline__ void merge_units(const ChunkMergeParams& p, int leader, int parts, int first_unit, int step, const int4& item) {
    const int lane = threadIdx.x & 31, slabs = (item.y + 31) / 32;
    for (int unit = first_unit; unit < slabs * (D / (4 * C)); unit += step) {
        const int row = unit % slabs * 32 + (lane & 7) * 4, d0 = unit / slabs * (4 * C) + (lane >> 3) * C;
        float M[4], den[4], num[C][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            M[i] = -INFINITY;
            den[i] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) num[c][i] = 0.f;
        }
        for (int first = 0; first < parts; first += kBatch) {
            __align__(16) float lw[kBatch][4], x[kBatch][C][4];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                // (the workspace has less than 2^32 numbers)
                const unsigned slot = first + u == 0 ? 2 * leader + 1 : 2 * (leader + min(first + u, parts - 1));
                *reinterpret_cast<float4*>(lw[u]) = *reinterpret_cast<const float4*>(p.lse + slot * p.slot_rows + row);
                const unsigned at = (slot * D + d0) * p.slot_rows + row;
#pragma unroll
                for (int c = 0; c < C; ++c) *reinterpret_cast<float4*>(x[u][c]) = *reinterpret_cast<const float4*>(p.part + at + c * p.slot_rows);
                if (kBatch > 1 && first + u >= parts) lw[u][0] = lw[u][1] = lw[u][2] = lw[u][3] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float top = M[i];
#pragma unroll
                for (int u = 0; u < kBatch; ++u) top = fmaxf(top, lw[u][i]);
                const float f = top > M[i] ? ex2((M[i] - top) * kLog2e) : 1.f;       // 0 the first time
                M[i] = top;
                den[i] *= f;
#pragma unroll
                for (int c = 0; c < C; ++c) num[c][i] *= f;
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    // -inf: no part, or one the row saw nothing of and whose values mean nothing (a NaN is carried on)
                    const bool holds = lw[u][i] != -INFINITY;
                    const float w = holds ? ex2((lw[u][i] - top) * kLog2e) : 0.f;
                    den[i] += w;
#pragma unroll
                    for (int c = 0; c < C; ++c) num[c][i] = fmaf(w, holds ? x[u][c][i] : 0.f, num[c][i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = row + i, t = item.x + r / G;
            if (r >= item.y || item.w + r / G < 0 || (unsigned)t >= (unsigned)p.total_q) continue;
            const float inv = 1.f / den[i];
            __nv_bfloat16* o = p.out + ((size_t)t * p.Hq + item.z * G + r % G) * D + d0;
            if constexpr (C == 4) *reinterpret_cast<uint2*>(o) = make_uint2(pack2(num[0][i] * inv, num[1][i] * inv), pack2(num[2][i] * inv, num[3][i] * inv));
            else *reinterpret_cast<uint32_t*>(o) = pack2(num[0][i] * inv, num[1][i] * inv);
        }
    }
}

template <int D, int G>
__global__ void __launch_bounds__(kMergeWarps * 32, 2)
chunk_merge_kernel(const ChunkMergeParams p) {
    __shared__ int flags[kChunkMaxWorkers];
    grid_dependency_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, me = blockIdx.x;
    const int last = warp / (kMergeWarps / 2);                  // in the place of the worker's first piece, or of its last
    grid_dependency_wait();
    for (int i = threadIdx.x; i < p.W; i += kMergeWarps * 32) flags[i] = p.flags[i];
    const int4 item = p.items[2 * me + last];
    __syncthreads();
    if (!(flags[me] & (last ? kOpens : kContinues | kCloses))) return;
    int leader = me;
    if (!last) {                                                // the last one before this that opens
        for (int hi = me - 1;; hi -= 32) {
            const unsigned found = __ballot_sync(kFull, hi - lane >= 0 && (flags[max(hi - lane, 0)] & kOpens));
            leader = hi - (__ffs(found) - 1);
            if (found || hi < 32) break;
        }
        leader = max(min(leader, me - 1), 0);
    }
    int parts = 1;
    for (int at = leader + 1;; at += 32) {
        const unsigned run = __ballot_sync(kFull, at + lane < p.W && (flags[min(at + lane, p.W - 1)] & kContinues));
        if (run != kFull) {
            parts += __ffs(~run);                               // and the one that closes it
            break;
        }
        parts += 32;
    }
    parts = min(parts, p.W - leader);
    const int mine = (me - leader) * (kMergeWarps / 2) + warp % (kMergeWarps / 2), all = parts * (kMergeWarps / 2);
    if (parts <= 4) merge_units<D, G, 4, 1>(p, leader, parts, mine, all, item);
    else merge_units<D, G, 2, 2>(p, leader, parts, mine, all, item);
}

// ----------------------------------------------------------------------------- host
// q [tokens, Hq, D] as a 3-D tensor; a box is 64 dims x the G heads of a group x `box` tokens.
bool make_q_map(CUtensorMap* map, const void* q, int64_t stride, int tokens, int Hq, int G, int D, int box_tokens) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)Hq, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)box_tokens};
    return make_bf16_map(map, q, 3, dims, strides, box);
}

struct Maps {
    CUtensorMap q32, q16, k, v;
};

// Shared memory of a launch whose items have `split` CTAs each.
size_t chunk_smem(int D, int split, int recv_rows) {
    return (D == 128 ? ChLayout<128>::kSmemBytes : ChLayout<64>::kSmemBytes) + (split > 1 ? (size_t)recv_rows * (D + split) * 4 : 0);
}

// Clusters of 2^k of the kernel's CTAs that are resident together, of one CTA per multiprocessor (148, 74, 33, 15: a cluster's lie in
// one part of the GPU); 0 where that cannot be found out.
int resident_clusters(int k) {
    static std::atomic<int> known[kMaxDevices][4];
    static std::atomic<bool> configured[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
    int n = known[dev][k].load(std::memory_order_relaxed);
    if (n == 0) {
        if (!ensure_smem_limit(chunk_kernel<128, 1, kShared>, ChLayout<128>::kMostBytes, configured)) return 0;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        cfg.gridDim = dim3(8);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = ChLayout<128>::kMostBytes;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 1u << k;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, chunk_kernel<128, 1, kShared>, &cfg) != cudaSuccess || n <= 0) {
            (void)cudaGetLastError();       // not the call's: it goes without clusters
            return 0;
        }
        known[dev][k].store(n, std::memory_order_relaxed);
    }
    return n;
}

// How many CTAs every item gets: one, or a cluster that shares its tiles; 0: the list.  items, seq_items (of one sequence) and tiles (of the
// longest) are what the host can bound them by; wide: blocks of more than 64 rows; wave: the CTAs that are resident together.
//
// The list takes a prologue and a launch for the merge, and cuts evenly; clusters cost their barriers and the exchange, 3 us, and go
// with the longest item.  In a graph, us, the list against 1, 2, 4 and 8 CTAs an item:
//   8 items of 5, 9, 17, 33, 65, 129 and 257 tiles: 8.6 11.7 13.0 16.0 21.3 26.4 32.4 against 7.4 10.4 16.5 28.4 .. (1), 7.9 8.4 10.1 13.2
//     19.3 31.2 55 (4) and 8.4 8.9 9.4 11.0 14.1 20.1 32.2 (8);
//   32 items of 5, 9, 17, 33 and 65: 10.3 14.3 15.5 19.5 23.9 against 7.7 10.9 17.4 30 56 (1), 8.8 10.4 13.6 19.6 31.7 (2), 9.8 10.3 11.8
//     15.0 21.2 (4); wide 12.5 15.9 18.1 20.7 25.4 against 9.5 13.4 20.7 35 64 (1) and 11.5 12.2 13.9 17.3 23.9 (4);
//   128 items of 9, 17 and 33: 15.8 22.0 33.7 against 12.2 19.2 33.4 (1) and 13.2 17.6 27.1 (2);
//   64-dim heads, 128 items of 66 rows and 18 tiles: 23.3 against 23.9 (1) and 20.2 (2).
// So: by estimates in us, a CTA 4.3 and 0.8 a tile (wide 6 and 0.9), a cluster 6.8 (8.7) and 0.013 per CTA of all, where they fit the GPU at
// once -- 16 clusters of 8 with a multiprocessor for each CTA, in two waves, took 16.1 us where 8 took 8.2 -- and a CTA has few tiles:
// up to 8 and one more per 16 items of one CTA, 16 and one more per 32 CTAs of clusters.
//
// More items than a wave: a CTA each against the list that is cut, 320 items of 2, 4, 8 and 16 tiles 13.1 17.0 24.8 41.7 against 17.6 21.2
// 26.9 37.1; 448 14.6 18.2 26.9 45.0 against 17.6 25.3 32.5 46.9; 600 of 2, 4 and 8 19.5 25.1 37.9 against 22.7 28.2 37.1; 896 25.9 33.7 51.0
// against 25.2 33.1 48.0; wide, 448 of 2, 4, 8 and 16 18.3 22.5 31.7 51.5 against 23.7 31.9 40.3 58.9, 600 26.7 32.8 45.7 74.7 against 28.2
// 36.7 48.7 72.9, 896 36.5 46.3 63.9 103.6 against 35.3 46.3 64.7 101.3.  There it goes by estimates of both, in us.  Up to two waves:
// a wave 6 and 1.06 a tile (wide 8.3 and 1.2), a last one that is not full counting 0.8, and the list 17 (12 where nothing can be cut)
// and of each worker's items 1.2 and 1.06 a tile (wide 3.4 and 1.25); from there on straight lines in the number of items.
//
// far: the batch's keys and values are more than L2 holds and the sequences have several blocks, which read the same ones.  Side by side
// as the grid has them they find them there, over the list's ranges not: 4 blocks each behind 1024 tokens, 172, 264 and 403 MB, 117 170 253
// against 128 194 289 us; 8 blocks, 130 and 197 MB, 164 243 against 166 280 (65 MB: 103 against 95).
//
// Both take every context for the longest, and what the host knows of that is the tables' width.  Where a batch is not so, the longest
// item is walked by one CTA alone.  So they hold up to kOneTiles and kFarTiles, where that costs little -- one item of 8, 16, 24, 32 and
// 48 tiles among 320 of 1, a CTA each against the list, 11.7 17.4 23.3 29.1 41.1 against 16.0 15.9 16.8 17.6 19.0, among 560 of 4 18.9 20.2 26.4
// 32.4 44.4 against 26.4 26.9 27.1 27.9 27.8; of 16, 24, 32 and 48 among 768 wide ones of 4 35 41 48 62 against 39 42 43 45; but one of 512
// among 560 of 16 403 against 76 -- and beyond where a sequence's items alone are a third of a wave, which leaves few CTAs without work:
// with 16, 32, 64, 128 and 256 items one sequence of 32768 tokens among others of 1024 took 490 603 733 752 763 against 116 232 327 432 1009,
// all of 8192 431 466 568 1091 1152 against 457 504 657 1348 1262, all of 32768 (32 to 256) 1925 2301 4661 4675 against 2129 3257 6431 6346.
// (Short of that, batches of long and like contexts would gain: 592 items of 20, 32, 64 and 128 tiles 59 94 180 354 against 65 99 188 363.)
int ctas_per_item(long long items, long long seq_items, long long wave, long long tiles, bool wide, bool far, int D, int recv_rows) {
    const double t = (double)tiles, share = (double)items / (double)wave;
    if (items > wave) {
        const bool fills = 3 * seq_items >= wave;
        if (far && (fills || tiles <= kFarTiles)) return 1;
        if (items > 4 * wave || !(fills || tiles <= kOneTiles)) return 0;
        double direct, list;
        if (items <= 2 * wave) {
            direct = (1.0 + 0.8) * (wide ? 8.3 + 1.2 * (t - 1) : 6.0 + 1.06 * (t - 1));
            list = (tiles > 1 ? 17.0 : 12.0) + share * (wide ? 3.4 + 1.25 * t : 1.2 + 1.06 * t);
        } else {
            direct = wide ? 3.0 + 0.9 * t + share * (6.2 + 1.17 * t) : 4.0 + 0.8 * t + share * (3.3 + t);
            list = wide ? (tiles > 2 ? 17.0 : 10.0) + share * (2.2 + 1.35 * t) : (tiles > 2 ? 15.0 : 11.0) + share * (1.25 * t - 0.5);
        }
        return direct < list;
    }
    const double per_tile = wide ? 0.9 : 0.8;
    double best = (wide ? 6.0 : 4.3) + per_tile * t;
    int split = 1;
    for (int k = 1; k <= 3; ++k) {
        const int C = 1 << k, per_sm = 2 * (chunk_smem(D, C, recv_rows) + 1024) <= kSmemPerSm ? 2 : 1;
        if (items * C > wave || tiles < C) break;
        const double time = (wide ? 8.7 : 6.8) + 0.013 * (double)(items * C) + per_tile * (double)((tiles + C - 1) / C);
        if (time < best && items <= (long long)per_sm * resident_clusters(k)) best = time, split = C;
    }
    const long long each = (tiles + split - 1) / split;
    return each <= (split == 1 ? 8 + items / 16 : 16 + items * split / 32) ? split : 0;
}

template <int D, int G>
int launch_both(const Maps& maps, const ChunkParams& p, const ChunkMergeParams& m, dim3 grid, cudaStream_t stream) {
    static std::atomic<bool> configured[3][kMaxDevices];
    const size_t smem = chunk_smem(D, p.split, p.recv_rows);
    if (p.split > 1) {
        if (!ensure_smem_limit(chunk_kernel<D, G, kShared>, ChLayout<D>::kMostBytes, configured[kShared])) return OPT_GQA_ERR_CUDA;
        return launch_clusters(chunk_kernel<D, G, kShared>, grid, dim3(kThreads), p.split, smem, stream, maps.q32, maps.q16, maps.k, maps.v, p);
    }
    if (p.split == 1) {
        if (!ensure_smem_limit(chunk_kernel<D, G, kOne>, smem, configured[kOne])) return OPT_GQA_ERR_CUDA;
        return launch_dependent(chunk_kernel<D, G, kOne>, grid, dim3(kThreads), smem, stream, maps.q32, maps.q16, maps.k, maps.v, p);
    }
    if (!ensure_smem_limit(chunk_kernel<D, G, kList>, smem, configured[kList])) return OPT_GQA_ERR_CUDA;
    const int rc = launch_dependent(chunk_kernel<D, G, kList>, grid, dim3(kThreads), smem, stream, maps.q32, maps.q16, maps.k, maps.v, p);
    if (rc != OPT_GQA_OK || m.W <= 1) return rc;            // (one worker has nothing to merge)
    return launch_dependent(chunk_merge_kernel<D, G>, dim3((unsigned)m.W), dim3(kMergeWarps * 32), 0, stream, m);
}

template <int D>
int launch_g(const Maps& maps, const ChunkParams& p, const ChunkMergeParams& m, int G, dim3 grid, cudaStream_t stream) {
    switch (G) {
        case 1: return launch_both<D, 1>(maps, p, m, grid, stream);
        case 2: return launch_both<D, 2>(maps, p, m, grid, stream);
        case 4: return launch_both<D, 4>(maps, p, m, grid, stream);
        case 8: return launch_both<D, 8>(maps, p, m, grid, stream);
    }
    return OPT_GQA_ERR_SHAPE;
}

}  // namespace

int launch_chunk(void* out, const void* q, int64_t q_stride, const int32_t* q_start_loc, int total_q_tokens, int max_q_len,
                 const void* k_cache, const void* v_cache, const int32_t* block_tables, int max_blocks_per_seq,
                 const int32_t* context_lens, const float* alibi_slopes, float scale, int B, int Hq, int Hkv, int D, int bs,
                 int64_t num_blocks, int window, void* workspace, int* device_status, cudaStream_t stream) {
    const uint64_t rows = (uint64_t)num_blocks * (uint64_t)Hkv * (uint64_t)bs;
    if (rows == 0 || rows > 0x7fffffffull) return OPT_GQA_ERR_SHAPE;
    const int G = Hq / Hkv, sms = sm_count();
    if (sms <= 0) return OPT_GQA_ERR_CUDA;
    Maps maps;
    if (!make_q_map(&maps.q16, q, q_stride, total_q_tokens, Hq, G, D, 16 / G) || !make_cache_map(&maps.k, k_cache, rows, D, bs) ||
        !make_slice_map(&maps.v, v_cache, rows, D, bs))
        return OPT_GQA_ERR_CUDA;
    maps.q32 = maps.q16;                // blocks of more than kNarrowRows take boxes of 32 rows
    if ((long long)max_q_len * G > kNarrowRows && !make_q_map(&maps.q32, q, q_stride, total_q_tokens, Hq, G, D, 32 / G))
        return OPT_GQA_ERR_CUDA;
    const ChunkLayout L = chunk_layout(Hq, Hkv, D, max_q_len);
    char* ws = static_cast<char*>(workspace);
    ChunkParams p;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.q_start_loc = q_start_loc;
    p.block_tables = block_tables;
    p.context_lens = context_lens;
    p.slopes = alibi_slopes;
    p.flags = reinterpret_cast<int32_t*>(ws + L.flags);
    p.items = reinterpret_cast<int4*>(ws + L.items);
    p.lse = reinterpret_cast<float*>(ws + L.lse);
    p.part = reinterpret_cast<float*>(ws + L.part);
    p.status = device_status;
    p.scale = scale;
    p.B = B;
    p.total_q = total_q_tokens;
    p.max_q = max_q_len;
    p.max_blocks = max_blocks_per_seq;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.bs = bs;
    p.bs_log2 = bs == 32 ? 5 : 4;
    p.window = window;
    p.slot_rows = L.slot_rows;
    p.recv_rows = (long long)max_q_len * G <= 16 ? 16 : L.slot_rows;
    ChunkMergeParams m;
    m.out = p.out;
    m.flags = p.flags;
    m.items = p.items;
    m.lse = p.lse;
    m.part = p.part;
    m.Hq = Hq;
    m.total_q = total_q_tokens;
    m.slot_rows = L.slot_rows;
    const long long blocks = ((long long)max_q_len * G + kRows - 1) / kRows, items = blocks * Hkv * B;
    long long tiles = (long long)max_blocks_per_seq * bs / kTN + 1;
    if (window > 0) {
        const long long seen = ((long long)window + kRows / G + kTN - 2) / kTN + 1;
        if (seen < tiles) tiles = seen;
    }
    const long long wave = (long long)sms * kCtasPerSm < kChunkMaxWorkers ? (long long)sms * kCtasPerSm : kChunkMaxWorkers;
    // several blocks of most sequences, by the number of new tokens, and more than kFarBytes of keys and values, by the tables' width
    const bool far = blocks > 1 && blocks * B <= 2 * ((long long)total_q_tokens * G / kRows + B) &&
                     (double)B * Hkv * D * 4 * kTN * (double)tiles > kFarBytes;
    p.split = blocks <= 65535 ? ctas_per_item(items, blocks * Hkv, wave, tiles, (long long)max_q_len * G > kNarrowRows, far, D, p.recv_rows) : 0;
    dim3 grid((unsigned)blocks * (p.split > 1 ? p.split : 1), (unsigned)Hkv, (unsigned)B);
    m.W = 1;
    if (!p.split) {
        // one resident wave, and no more workers than there can be tiles
        const long long most = Hkv * ((long long)total_q_tokens * G / kRows + B) * tiles;
        m.W = (int)(most < wave ? most : wave);
        grid = dim3((unsigned)m.W);
    }
    return D == 128 ? launch_g<128>(maps, p, m, G, grid, stream) : launch_g<64>(maps, p, m, G, grid, stream);
}

}  // namespace optgqa
