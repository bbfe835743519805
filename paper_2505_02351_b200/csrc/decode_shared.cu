// Decode attention for a batch whose sequences share long prefixes (one prompt, many continuations): the keys and values
// of a shared prefix are brought on-chip once for all sequences of its group instead of once per sequence.
//
// Softmax over disjoint sets of keys merges exactly from each set's normalised result and log-sum-exp, so
//     out = (e^{lse_P} o_P + e^{lse_S} o_S) / (e^{lse_P} + e^{lse_S}),
// P the keys a sequence shares, S its own.  Both are items of one kernel: over the shared keys of a group the n_g sequences
// times the G query heads of a KV head are the rows (in blocks of 128), a real matrix product with 2 n_g G flops per byte
// of the cache; over a sequence's own keys the G heads are the rows.  Per item S = Q K^T and O += P V run on tcgen05 over
// 64-key tiles, accumulators in tensor memory, as a query block of the chunked prefill does.  For an own item most of the
// rows of a product (64, the fewest the instruction has) are idle, and that costs little that counts: a 32 KB tile takes an
// SM's share of the memory bandwidth 1480 cycles, and the two resident CTAs need 1000 for its arithmetic, idle rows or not
// (warps none of whose rows are live skip the softmax).  So own contexts and prefixes of up to 128 rows are bound by reading the
// cache; prefixes of more rows by the special-function unit and the tensor core, as the prefill is (1.07 PFLOP/s).
// (Products with the keys as rows and the G heads as columns, S^T = K Q^T and O^T = V^T P, waste nothing and spread the
// exponentials over all warps, but take 80 cycles an instruction and, V^T being transposed, 160: 256 sequences in 12 groups
// 119.6 us against 94.  128 rows instead of 64 cost power: 108.7 us against 104.3 when run without a pause.)
//
// The tiles of the groups' items, laid end to end, are cut into one contiguous range per worker (a CTA, two per SM), and so
// are those of the sequences' own, as many workers for the one as for the other as they are worth, so that one long prefix
// fills the GPU as well as many short ones, whatever the mix.  A worker's part of an item is a piece: normalised partial rows
// and log-sum-exps in the workspace, merged by merge_shared_kernel.  (The own contexts were first left to decode_stream.cu:
// its mma.sync work takes issue slots and tensor cycles from the group pass beside it, and its workers drain between two
// 16-token tiles: 28.6 us for 32 sequences behind 1500 tokens, where this took 19.3.  Workers that take of both lists make more
// pieces: 22.3.)
//
// 32/8 heads, 32 sequences of 64 to 548 tokens behind 1500 shared ones: 18.3 us (37 MB: 5.7 us of copy bandwidth); 32/4
// heads, 8 behind 32768: 23.9 us (78 MB, 12.1); 64/8 heads, 256 in 12 groups: 89 us (383 MB, 59; DRAM reads 419 MB; 100 to 104
// where it runs without a pause and the power limit takes the clock down to 1.75 GHz); 32/8 heads, 128 behind 16384: 61 to 68
// us (34.5 GFLOP, 20 at the burst rate, 24 at the sustained one).  The weights are rounded to bf16 for P V, as in the other
// decode kernels, and the denominator sums the rounded ones: 0.2 to 2 us of that (18.1, 24.1, 89.2, 61.0 against 17.7, 23.9,
// 87.9, 59.5), for a value that all keys have to come out as it went in.  Besides the main phase each has 5 to 7 us from the launch to
// the first copy (the list is computed from cold memory and cold code; one CTA per SM does that while a preceding call's merge
// runs, the other behind it), 3 to 5 us between a worker's mean end and the last one's, 1.5 to 2.5 us until the merge may read,
// and 3 to 10 us of merge.  The row warps' loop fills their 128 registers: 24 bytes spilled cost 4 %.
//
// A sequence sees whole tiles of its group only: the first e_s = floor(min(prefix, n_s) / 64) * 64 tokens, the rest is its
// own.  So no group tile is masked inside, and where sequences of a group differ in e_s (the tiles are taken from the last
// one backwards) a row that has not begun simply discards what it accumulated: its O is set to zero, not multiplied by zero,
// at its first tile, and nothing it does not see can reach it, not even a NaN.
//
// Eight warps: 0-3 one thread per row (softmax), 4 the list of pieces and the TMA copies of Q and K, 6 those of V, 5 and 7
// issue S = Q K^T and O += P V.  (One producer was what everything waited for: a copy of 16 rows costs its warp about 90
// cycles, 16 of them a tile; and one issuing thread adds the waits for K, V and P up, 1690 cycles a tile.)  Every wait is a
// bounded mbarrier wait.
#include "umma.cuh"

namespace optgqa {

namespace {

constexpr int kRows = kSharedRows;
constexpr int kTN = kSharedTile;
constexpr int kStages = 2;                 // of the K ring and of the V ring
constexpr int kCtasPerSm = 2;
constexpr int kThreads = 256;
// The cut counts tiles, and for an item besides (the next one's Q, which takes the place of this one's, the wait for its last
// P V, storing the piece) as many of them as it costs time: fitted to the times of 296 workers with different numbers of
// tiles and pieces, a group's tile and one of a sequence's own last alike (1.06 us, two CTAs per SM), a group's item 2.4 to 3.7
// of them, an own item about one.
constexpr int kGroupItem = 3, kOwnItem = 1;
// A worker's share of the groups' list at least (a piece of theirs is 64 KB), and of the own one.
constexpr int kMinGroupShare = 4, kMinOwnShare = 2;
constexpr int kOwnRows = 64;              // M of an own item's products: row 16 w + h lies in lane 32 w + h of tensor memory
constexpr int kDescs = 4;                  // pieces described ahead
constexpr unsigned kFull = 0xffffffffu;
constexpr float kRescaleThreshold = 8.f;   // log2 units: O is rescaled only when a row's maximum grew by more

constexpr int kHalfBytes = kTN * 128;      // one 64-dim column half of a K tile
constexpr int kQHalfBytes = kRows * 128;   // one 64-dim column half of the Q tile
// The ALiBi term inside a tile rides on the tensor core as one more k-step (see prefill_umma.cu): slope / |scale| as
// three bf16 values against the key's index in the tile.
constexpr int kExtRowGroupBytes = 256;
constexpr int kQxBytes = kRows / 8 * kExtRowGroupBytes;
constexpr int kKpBytes = kTN / 8 * kExtRowGroupBytes;
// barriers: q_full[4], q_empty[4], o_empty[4], k_full[], k_empty[], v_full[], v_empty[], s_full[2], p_full[2],
// desc_full[], desc_empty[]
constexpr int kNumBars = 12 + 4 * kStages + 4 + 2 * kDescs;
constexpr int kDescReaders = 7;            // warps that read a descriptor: all but the one that writes it

template <int D>
struct ShLayout {
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
    static constexpr int kOffGroups = kOffDesc + kDescs * 48;           // units before (8 B), tiles, leader, items before (2 B)
    static constexpr int kSmemBytes = kOffGroups + kMaxGroups * 18 + 1024;
};

constexpr uint32_t kColS = 0;              // S buffers at 0 and kTN, P over the first half of its S
constexpr uint32_t kColO = 2 * kTN;
constexpr uint32_t kTmemCols = 256;

struct SharedParams {
    const int32_t* block_tables;
    const int32_t* context_lens;
    const int32_t* prefix_lens;
    const int32_t* group_start;
    const float* slopes;
    int32_t* info;              // see SharedLayout, as the pieces below
    float* group_lse;
    float* group_out;
    float* own_lse;
    float* own_out;
    int* status;
    float scale;
    int num_groups, B, max_blocks, Hkv, bs, bs_log2, lanes_log2;
};

// mbar_wait with its waiting loop in one place: this kernel waits at some twenty, its warps run all over it, and its time
// goes with the instruction cache's misses (as inlined: 86 KB, the caches' shared port busy 74 % of the time).
__noinline__ __device__ bool wait_long(uint64_t* bar, uint32_t parity, int* status) { return mbar_wait(bar, parity, status); }
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, int* status) {
    return mbar_try_wait(bar, parity) || wait_long(bar, parity, status);
}

// Where the share of worker i of W begins in a list of `total`: rounded down, so that the shares follow one another.
__device__ __forceinline__ long long share_at(long long total, int i, int W) {
    return total < (1 << 22) ? (long long)((unsigned)total * (unsigned)i / (unsigned)W) : total * i / W;      // (W < 512)
}

// What the other warps need to know of a piece.
struct Piece {
    int s0, rows, kvh, table;       // first sequence, live rows, KV head, sequence whose page table is walked
    int tile_hi, len, n, piece;     // last tile (of the sequence's 64-key tiles) and how many, keys there are, number
    int own, opens, closes, warp0;  // own item or a group's; whether the piece holds the item's first and last tile; the row
                                    // warp whose lanes are the first rows
};

template <int D, int G>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
decode_shared_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_q1,
                     const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                     const SharedParams p) {
    using L = ShLayout<D>;
    constexpr int kTileBytes = L::kTileBytes, kOffQ = L::kOffQ, kOffK = L::kOffK, kOffV = L::kOffV, kOffQx = L::kOffQx,
                  kOffKp = L::kOffKp;
    constexpr int TQ = kRows / G;          // sequences per row block
    extern __shared__ char smem_raw[];
    char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
    uint64_t* q_full = bars;                    // [4], per quarter of Q: an own item's rows lie in one, a group's use the first
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
    long long* g_units = reinterpret_cast<long long*>(smem + L::kOffGroups);     // of the groups before (one head)
    int* g_kt = reinterpret_cast<int*>(g_units + kMaxGroups);
    int* g_lead = g_kt + kMaxGroups;
    uint16_t* g_items = reinterpret_cast<uint16_t*>(g_lead + kMaxGroups);        // at most kMaxGroups + 65535 * 8 / 128
    // units of the own items (one head) of the sequences before each thread's chunk, from its warp's first on, and of each
    // warp's chunks; gone once the K ring is in use
    long long* c_units = reinterpret_cast<long long*>(smem + kOffK);
    long long* w_units = c_units + kThreads;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int N = p.num_groups;
    if (threadIdx.x == 192) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q1) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    auto group_lo = [&](int g) { return min(max(__ldg(p.group_start + g), 0), p.B); };
    auto blocks_of = [&](int g) {
        const int rows = max(group_lo(g + 1) - group_lo(g), 0) * G;
        return rows / kRows + (rows % kRows != 0);
    };
    const int grouped_lo = __ldg(p.group_start), grouped_hi = __ldg(p.group_start + N);
    // tiles of sequence s (of length n) at which its own begin and end
    auto own_begin = [&](int s, int n) {
        const int e = shared_tokens(__ldg(p.prefix_lens + s), n) / kTN;
        return s >= grouped_lo && s < grouped_hi ? e : 0;
    };
    auto own_end = [&](int n) { return (max(n, 0) + kTN - 1) / kTN; };
    auto item_units = [&](int tiles) { return tiles > 0 ? tiles + kOwnItem : 0; };

    // ------------------------------------------------------------------ the items (the index arrays are read before the
    // wait for the preceding kernel: see the ordering contract in the header)
    const int chunk = (p.B + kThreads - 1) / kThreads;          // sequences per thread
    {
        long long sum = 0;
        for (int s = threadIdx.x * chunk; s < min((int)(threadIdx.x + 1) * chunk, p.B); ++s) {
            const int n = __ldg(p.context_lens + s);
            sum += item_units(own_end(n) - own_begin(s, n));
        }
        long long incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += v;
        }
        c_units[threadIdx.x] = incl - sum;
        if (lane == 31) w_units[warp] = incl;
    }
    {
        // of each group the longest shared run, whose it is, and the row blocks: 2^lanes_log2 lanes per group
        const int lanes = 1 << p.lanes_log2, sub = lane & (lanes - 1), per_warp = 32 >> p.lanes_log2;
        for (int g0 = warp * per_warp; g0 < N; g0 += kThreads / 32 * per_warp) {
            const int g = g0 + (lane >> p.lanes_log2);
            int best = 0, lead = 0;
            if (g < N) {
                const int hi = group_lo(g + 1);
                for (int s = group_lo(g) + sub; s < hi; s += lanes) {
                    const int e = shared_tokens(__ldg(p.prefix_lens + s), __ldg(p.context_lens + s));
                    if (e > best) best = e, lead = s;
                }
            }
            for (int o = lanes >> 1; o >= 1; o >>= 1) {
                const int e = __shfl_xor_sync(kFull, best, o), l = __shfl_xor_sync(kFull, lead, o);
                if (e > best || (e == best && l < lead)) best = e, lead = l;
            }
            if (g < N && sub == 0) {
                g_kt[g] = best / kTN;
                g_lead[g] = lead;
                g_items[g] = best > 0 ? (uint16_t)blocks_of(g) : 0;     // (at most 65535 * 8 / 128)
            }
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

    if (warp == 4) {
        // ------------------------------------------------------------------ the list of pieces, Q and K
        // Exclusive sums over the groups.  A group_start that is not increasing may name more row blocks than the workspace
        // has room for: the groups past it are left out (a wrong row, never a write outside).
        long long group_total = 0, own_total = 0;
        {
            int items = 0;
            const int most = N + (int)((long long)p.B * G / kRows);
            for (int g0 = 0; g0 < N; g0 += 32) {
                const int g = g0 + lane;
                int b = g < N ? g_items[g] : 0, kt = g < N ? g_kt[g] : 0;
                int incl = b;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(kFull, incl, o);
                    if (lane >= o) incl += v;
                }
                if (items + incl > most) b = 0, kt = 0;       // (items + incl only grows: all later ones too)
                const long long units = b * (long long)(kt + kGroupItem);
                long long incl_t = units;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const long long v = __shfl_up_sync(kFull, incl_t, o);
                    if (lane >= o) incl_t += v;
                }
                if (g < N) {
                    g_units[g] = group_total + incl_t - units;
                    g_items[g] = (uint16_t)min(items + incl - b, most);
                    g_kt[g] = kt;
                }
                group_total += __shfl_sync(kFull, incl_t, 31);
                items += __shfl_sync(kFull, incl, 31);
            }
            group_total *= p.Hkv;
            for (int w = 0; w < kThreads / 32; ++w) own_total += w_units[w];
            own_total *= p.Hkv;
            __syncwarp();
        }
        // This worker's share: as many workers as they are worth take the groups' units (fewer where a share would have less than
        // kMinGroupShare), the others the own ones (kMinOwnShare each at least).
        const int W = gridDim.x, me = blockIdx.x;
        const long long units = group_total + own_total;
        // (rounded in fp32: which way matters to nobody, all workers round alike)
        int gw = units > 0 ? __float2int_rn(__ll2float_rn(group_total) / __ll2float_rn(units) * W) : 0;
        gw = max(min(gw, own_total > 0 && W > 1 ? W - 1 : W), group_total > 0 ? 1 : 0);
        gw = (int)min((long long)gw, (group_total + kMinGroupShare - 1) / kMinGroupShare);
        const int o0 = W > 1 ? gw : 0, ow = (int)max(min((long long)(W - o0), own_total / kMinOwnShare), 1ll), oi = min(max(me - o0, -1), ow);
        // four lanes one bound each: the groups' share's begin and end, the own one's
        const bool of_own = lane & 2;
        const int at = of_own ? min(max(oi + (lane & 1), 0), ow) : min(me + (lane & 1), gw);
        const long long bound = share_at(of_own ? own_total : group_total, at, of_own ? ow : max(gw, 1));
        const long long g_lo = __shfl_sync(kFull, bound, 0), g_hi = __shfl_sync(kFull, bound, 1);
        const long long o_lo = __shfl_sync(kFull, bound, 2), o_hi = __shfl_sync(kFull, bound, 3);
        // the place in the list: (group, KV head, row block), row block fastest, so that the blocks of one prefix are worked on
        // at the same time and its tiles come from L2 after their first reading; then (sequence, KV head)
        int g = 0, kvh = 0, mt = 0, blocks = 1, s = 0, n = 0, jt = 0, t0 = 0, t1 = 0;    // the item's tiles t0 .. t1 - 1
        long long item = 0;
        auto enter_group = [&]() {
            t0 = 0;
            t1 = g_kt[g];
            blocks = blocks_of(g);
        };
        long long pos = 0, hi = 0;          // in the list at hand: the next tile's place and the end of the share
        // a group item's tile j lies kGroupItem + j behind the item's begin
        auto locate_group = [&]() {
            pos = g_lo;
            hi = g_hi;
            if (pos >= hi) return;
            int a = 0, b = N - 1;           // the last group that begins at or before it (and so one that has tiles)
            while (a < b) {
                const int m = (a + b + 1) >> 1;
                if (g_units[m] * p.Hkv <= pos) a = m;
                else b = m - 1;
            }
            g = a;
            enter_group();
            const int u = t1 + kGroupItem;
            const long long r = pos - g_units[g] * p.Hkv;
            const int in_group = r < 0x7fffffff ? (int)r / u : (int)(r / u);
            const int in_item = (int)(r - (long long)in_group * u) - kGroupItem;
            jt = max(in_item, 0);
            pos += jt - in_item;
            kvh = in_group / blocks;
            mt = in_group - kvh * blocks;
            item = (long long)g_items[g] * p.Hkv + in_group;
        };
        // an own item's tile j lies kOwnItem + j behind the item's begin
        int own_chunk = 0;                  // the last thread's chunk that begins at or before o_lo, and its begin
        long long chunk_begin = 0;
        if (o_lo < o_hi) {
            while (own_chunk < kThreads / 32 - 1 && chunk_begin + w_units[own_chunk] * p.Hkv <= o_lo)
                chunk_begin += w_units[own_chunk++] * p.Hkv;
            own_chunk = own_chunk * 32 + __popc(__ballot_sync(kFull, chunk_begin + c_units[own_chunk * 32 + lane] * p.Hkv <= o_lo)) - 1;
            chunk_begin += c_units[own_chunk] * p.Hkv;
        }
        fence_proxy_async();
        __syncwarp();
        const int slices = kTN >> p.bs_log2, sub = lane & (slices - 1), hf = lane >> (6 - p.bs_log2);
        const bool issues = lane < slices * L::kHalves;
        char* ring = smem + kOffK + hf * kHalfBytes + sub * p.bs * 128;
        int st = 0;
        uint32_t ph = 1;                    // parity of a stage's last release (none yet: passes)
        // a sequence's own tiles are read once, a group's by all its row blocks
        const uint64_t read_once = l2_policy_evict_first(), read_again = l2_policy_evict_normal();
        // (One place for each of the steps below, for the sake of the instruction cache.)
        bool own = false, open_list = true, step = false, walk = false, seek = false;
        int lists = 0;                      // lists done
        uint32_t q_used = 0, q_ph = 0;      // quarters of Q not yet seen free again, and the parity of their next release
        bool q_group = false;               // the first of them stands for all of Q
        long long before = 0;
        for (int pc = 0;;) {
            if (open_list) {
                open_list = false;
                if (own) {
                    pos = hi = o_hi;
                    if (o_lo < o_hi) {
                        walk = seek = true;
                        s = own_chunk * chunk;
                        before = chunk_begin;
                    }
                } else {
                    locate_group();
                }
            }
            if (step) {                     // to the next item, where there is one
                step = false;
                if (pos >= hi) {
                } else if (own) {
                    if (++kvh == p.Hkv) {
                        kvh = 0;
                        ++s;
                        walk = true;
                    }
                } else {
                    ++item;
                    if (++mt == blocks) {
                        mt = 0;
                        if (++kvh == p.Hkv) {
                            kvh = 0;
                            do ++g;
                            while (g < N - 1 && g_kt[g] == 0);
                            enter_group();
                            item = (long long)g_items[g] * p.Hkv;
                        }
                    }
                }
            }
            if (walk) {                     // s, or the first one behind it that has tiles of its own -- or holds o_lo
                walk = false;
                for (; s < p.B; ++s) {
                    n = __ldg(p.context_lens + s);
                    t0 = own_begin(s, n);
                    t1 = own_end(n);
                    if (t1 <= t0) continue;
                    if (!seek || before + item_units(t1 - t0) * (long long)p.Hkv > o_lo) break;
                    before += item_units(t1 - t0) * (long long)p.Hkv;
                }
                if (s >= p.B) {
                    pos = hi;               // cannot happen: the shares end where the items do
                } else if (seek) {
                    seek = false;
                    const long long r = o_lo - before;
                    const int u = item_units(t1 - t0);
                    kvh = r < 0x7fffffff ? (int)r / u : (int)(r / u);
                    const int in_item = (int)(r - (long long)kvh * u) - kOwnItem;
                    jt = max(in_item, 0);
                    pos = o_lo + jt - in_item;
                }
            }
            if (pos >= hi && ++lists < 2) {
                own = !own;
                open_list = true;
                continue;
            }
            const unsigned room = (unsigned)max(min(hi - pos, (long long)0x3fffffff), 0ll);
            const int len = (int)min((unsigned)(t1 - t0 - jt), room);    // 0: the end
            const int s0 = own ? s : group_lo(g) + mt * TQ;
            const int rows = own ? G : min(kRows, (group_lo(g + 1) - s0) * G);
            // Own items take the row warps in turns: while one waits for its item's last P V and stores the piece, the next is
            // at the next item's weights.
            const int warp0 = own ? pc & 3 : 0;
            const int table_of = own ? s : g_lead[g], tile_hi = t0 + jt + len - 1, keys = own ? n : t1 * kTN;
            bool ok = __all_sync(kFull, wait_for(&desc_empty[pc % kDescs], ((pc / kDescs) & 1) ^ 1, p.status));
            if (!ok) break;
            if (lane == 0) {
                int4* d = reinterpret_cast<int4*>(smem + L::kOffDesc) + 3 * (pc % kDescs);
                d[0] = make_int4(s0, rows, kvh, table_of);
                d[1] = make_int4(tile_hi, len, keys, (int)((own ? (long long)s * p.Hkv + kvh : item) + me));
                d[2] = make_int4(own, jt == 0, jt + len == t1 - t0, warp0);
                mbar_arrive(&desc_full[pc % kDescs]);
            }
            if (len == 0) break;
            const int32_t* table = p.block_tables + (size_t)table_of * p.max_blocks;
            const int pages = min((keys + p.bs - 1) >> p.bs_log2, p.max_blocks);       // the table is not read past them
            auto page_of = [&](int j) {
                const int i = (tile_hi - j) * slices + sub;
                return issues && i < pages ? __ldg(table + i) : 0;
            };
            int page = page_of(0);
#pragma unroll 1
            for (int j = 0; j < len; ++j) {
                const int row = (page * p.Hkv + kvh) * p.bs;                       // row of the [rows, D] view
                const int live = min(slices, (keys - (tile_hi - j) * kTN + p.bs - 1) >> p.bs_log2);    // slices that hold keys
                page = j + 1 < len ? page_of(j + 1) : 0;
                ok = __all_sync(kFull, wait_for(&k_empty[st], ph, p.status));
                if (!ok) break;
                // q and the cache may still be written, the workspace still read, by the preceding kernel
                if (pc == 0 && j == 0) grid_dependency_wait();
                if (lane == 0) mbar_expect_tx(&k_full[st], (uint32_t)(live * p.bs * D * 2));
                __syncwarp();
                if (issues && sub < live) tma_load_2d_hint(ring + st * kTileBytes, &map_k, 64 * hf, row, &k_full[st], own ? read_once : read_again);
                if (++st == kStages) st = 0, ph ^= 1;
                if (j == 0) {
                    // Q behind the first K tile.  Own items lie in different quarters, so that the next one's rows are fetched
                    // while the piece before is still at work; a group's need all of Q.
                    uint32_t wait = own && !q_group ? q_used & (1u << warp0) : q_used;
                    q_used = own && !q_group ? q_used & ~wait : 0u;
#pragma unroll 1
                    for (int w = 0; wait; ++w, wait >>= 1)
                        if (wait & 1) {
                            ok = ok && __all_sync(kFull, wait_for(&q_empty[w], q_ph >> w & 1, p.status));
                            q_ph ^= 1u << w;
                        }
                    if (!ok) break;
                    q_used |= 1u << warp0;
                    q_group = !own;
                    if (lane == 0) {
                        // an own item's G rows alone: what the other rows of the tile hold reaches no live row
                        mbar_expect_tx(&q_full[warp0], own ? (uint32_t)(G * D * 2) : (uint32_t)L::kQBytes);
#pragma unroll 1
                        for (int h = 0; h < L::kHalves; ++h)
                            tma_load_3d(smem + kOffQ + h * kQHalfBytes + warp0 * (kOwnRows / 4 * 128), own ? &map_q1 : &map_q, 64 * h, kvh * G, s0, &q_full[warp0]);
                    }
                }
            }
            if (!ok) break;
            // on to the next piece
            ++pc;
            pos += len + (own ? kOwnItem : kGroupItem);
            jt = 0;
            step = true;
        }
    } else {
        // before any wait with a limit: what the producers wait for may take as long as it likes
        grid_dependency_wait();
        Piece d;
        auto read_piece = [&](int pc) {
            const uint32_t at = smem_u32(smem + L::kOffDesc) + 48 * (pc % kDescs);
            auto load = [&](uint32_t from, int& x, int& y, int& z, int& w) {
                asm volatile("ld.volatile.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(x), "=r"(y), "=r"(z), "=r"(w) : "r"(from));
            };
            load(at, d.s0, d.rows, d.kvh, d.table);
            load(at + 16, d.tile_hi, d.len, d.n, d.piece);
            load(at + 32, d.own, d.opens, d.closes, d.warp0);
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
                const uint64_t policy = d.own ? l2_policy_evict_first() : l2_policy_evict_normal();
                const int32_t* table = p.block_tables + (size_t)d.table * p.max_blocks;
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
                const uint32_t idesc_s = d.own ? instr_desc(false, kTN, false, kOwnRows) : instr_desc(false, kTN);
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
                                umma_ss(s_tmem, desc_advance(q_desc0, (ks >> 2) * kQHalfBytes + (ks & 3) * 32),
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
                const uint32_t idesc_pv = d.own ? instr_desc(true, D, false, kOwnRows) : instr_desc(true, D);
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
                reading = d.own ? 1u << d.warp0 : (1u << ((d.rows + 31) / 32)) - 1;
            }
        } else {
            // -------------------------------------------------------------- one thread per row: softmax, rescale, store
            const int r = threadIdx.x, hg = r % G;       // (32 is a multiple of G)
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
                int n = 0, e_row = 0;       // the row's context, and of that what it sees: of a group's item whole tiles
                {
                    const int rr = r - 32 * d.warp0, s = d.s0 + rr / G;     // row of the item
                    if (rr >= 0 && rr < d.rows) {
                        n = __ldg(p.context_lens + s);
                        e_row = d.own ? n : shared_tokens(__ldg(p.prefix_lens + s), n);
                    }
                }
                const float slope2 = p.slopes ? __ldg(p.slopes + d.kvh * G + hg) * kLog2e : 0.f;
                float m_used = -INFINITY, l = 0.f;
                auto next_tile = [&]() {
                    ++it;
                    if (++st == kStages) st = 0, ph ^= 1;
                };
                for (int j = 0; j < d.len; ++j, next_tile()) {
                    const int sb = it & 1, j0 = (d.tile_hi - j) * kTN;
                    ok = __all_sync(kFull, wait_for(&s_full[sb], (it >> 1) & 1, p.status));
                    if (!ok) break;
                    tc_fence_after();
                    const bool sees = j0 < e_row;
                    const bool masked = j0 + kTN > d.n;             // an own item's sequence ends inside the tile
                    if (!__any_sync(kFull, sees)) {
                        // no row of the warp has begun: what the tensor core adds to their O from this tile's scores,
                        // read as if they were weights, is discarded when they do
                        tc_fence_before();
                        mbar_arrive(&p_full[sb]);
                        continue;
                    }
                    const uint32_t s_addr = lane_addr + kColS + sb * kTN;
                    const float bias0 = slope2 * (float)(j0 - (n - 1));       // ALiBi term of the tile's first key
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
                    if (masked) {
                        // -inf in the place of what lies past the end: both passes then run as they are
                        const int live = d.n - j0;
#pragma unroll
                        for (int e = 0; e < kTN; ++e)
                            if (e >= live) v[e / 32][e % 32] = -INFINITY;
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
                const int rr = r - 32 * d.warp0, s = d.s0 + rr / G;
                const bool valid = rr >= 0 && rr < d.rows;
                if (__any_sync(kFull, valid)) {
                    ok = prev_pv_done();
                    if (!ok) break;
                    tc_fence_after();
                    const float inv = 1.f / l;
                    const bool begun = (d.tile_hi - d.len + 1) * kTN < e_row;      // the row saw a tile of the piece
                    // a group's piece is [D][128 rows], so that 32 neighbouring rows are one line; an own piece [G][D]
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        float o[32];
                        tmem_ld32(lane_addr + kColO + c * 32, o);
                        if (c == D / 32 - 1) {                      // the next piece may overwrite O
                            tc_fence_before();
                            mbar_arrive(&o_empty[warp]);
                        }
                        if (begun && d.own) {
                            float4* po = reinterpret_cast<float4*>(p.own_out + ((size_t)d.piece * G + rr) * D + c * 32);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                po[e] = make_float4(o[4 * e] * inv, o[4 * e + 1] * inv, o[4 * e + 2] * inv, o[4 * e + 3] * inv);
                        } else if (begun) {
                            float* po = p.group_out + ((size_t)d.piece * D + c * 32) * kRows + r;
#pragma unroll
                            for (int e = 0; e < 32; ++e) po[e * kRows] = o[e] * inv;
                        }
                    }
                    if (e_row > 0 && hg == 0) {
                        int32_t* info = p.info + ((size_t)s * p.Hkv + d.kvh) * kInfoWords;
                        if (d.own) {
                            if (d.opens) info[4] = d.piece;
                            if (d.closes) info[5] = d.piece;
                        } else {
                            if (d.opens) info[0] = d.piece, info[1] = r;
                            if (d.closes) info[2] = d.piece;
                        }
                    }
                    // a row that saw nothing of the piece: weight zero
                    if (valid)
                        (d.own ? p.own_lse + (size_t)d.piece * G : p.group_lse + (size_t)d.piece * kRows)[rr] = begun ? (m_used + lg2(l)) * kLn2 : -INFINITY;
                }
                release_piece(pc);
            }
        }
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
}

// ----------------------------------------------------------------------------- merge
// A CTA merges 32 rows: 32 / G consecutive sequences times the G heads of one KV head, a lane per row, so that a group's
// pieces ([D][rows]) are read as whole lines.  Per row the pieces are two runs of consecutive numbers, its group item's and its
// own.  kWP of the CTA's eight warps share the runs, the others (and the grid's z) take other columns, C of them per lane;
// a warp keeps a running maximum, so that log-sum-exps and rows are requested together, kBatch pieces at a time.
constexpr int kMergeWarps = 8;

struct MergeParams {
    __nv_bfloat16* out;
    const int32_t* context_lens;
    const int32_t* prefix_lens;
    const int32_t* group_start;
    const int32_t* info;
    const float* group_lse;
    const float* group_out;
    const float* own_lse;
    const float* own_out;
    int num_groups, B, Hq, Hkv, group_pieces, own_pieces;
};

template <int D, int G, int kWP, int C>
__global__ void __launch_bounds__(kMergeWarps * 32)
merge_shared_kernel(const MergeParams p) {
    constexpr int kSeqs = 32 / G, kBatch = 32 / C;      // (C 4, 8 or 16)
    __shared__ float s_max[kWP > 1 ? kMergeWarps : 1][32];
    __shared__ float s_den[kWP > 1 ? kMergeWarps : 1][32];
    __shared__ float s_num[kWP > 1 ? kMergeWarps : 1][C][32];
    grid_dependency_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wp = warp % kWP, d0 = (blockIdx.z * (kMergeWarps / kWP) + warp / kWP) * C;
    const int s = blockIdx.x * kSeqs + lane / G, kvh = blockIdx.y, hh = lane % G;
    const bool active = s < p.B;
    const int n = active ? __ldg(p.context_lens + s) : 0;
    const bool grouped = active && s >= __ldg(p.group_start) && s < __ldg(p.group_start + p.num_groups);
    const int shared = grouped ? shared_tokens(__ldg(p.prefix_lens + s), n) : 0;
    const bool has1 = shared > 0, has2 = n > shared;
    grid_dependency_wait();

    const int32_t* info = p.info + ((size_t)(active ? s : 0) * p.Hkv + kvh) * kInfoWords;
    int4 i0 = *reinterpret_cast<const int4*>(info);
    int2 i1 = *reinterpret_cast<const int2*>(info + 4);
    // Always so, where the index arrays keep their promises; where they do not (a sequence that no group of a group_start
    // that does not increase covers), the words were never written and the row is wrong, but nothing outside is read.
    i0.x = min(max(i0.x, 0), p.group_pieces - 1);
    i0.y = min(max(i0.y, 0), kRows - G);
    i0.z = min(min(max(i0.z, i0.x), i0.x + kSharedMaxWorkers), p.group_pieces - 1);
    i1.x = min(max(i1.x, 0), p.own_pieces - 1);
    i1.y = min(min(max(i1.y, i1.x), i1.x + kSharedMaxWorkers), p.own_pieces - 1);

    float M = -INFINITY, den = 0.f, num[C];
#pragma unroll
    for (int c = 0; c < C; ++c) num[c] = 0.f;
    // the two runs as one, so that a group's pieces and the own ones are requested together
    const int R1 = has1 ? i0.z - i0.x + 1 : 0, R = R1 + (has2 ? i1.y - i1.x + 1 : 0);
    const float* lse1 = p.group_lse + (size_t)i0.x * kRows + i0.y + hh;
    const float* out1 = p.group_out + ((size_t)i0.x * D + d0) * kRows + i0.y + hh;
    const float* lse2 = p.own_lse + (size_t)i1.x * G + hh;
    const float* out2 = p.own_out + ((size_t)i1.x * G + hh) * D + d0;
    for (int i = wp; i < R; i += kWP * kBatch) {
        float lw[kBatch];
        __align__(16) float x[kBatch][C];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int k = i + u * kWP, k2 = k - R1;
            lw[u] = -INFINITY;
            if (k < R1) {                                               // [D][rows]
                lw[u] = lse1[(size_t)k * kRows];
#pragma unroll
                for (int c = 0; c < C; ++c) x[u][c] = out1[((size_t)k * D + c) * kRows];
            } else if (k < R) {                                         // [G][D]
                lw[u] = lse2[(size_t)k2 * G];
#pragma unroll
                for (int c = 0; c < C; c += 4)
                    *reinterpret_cast<float4*>(&x[u][c]) = *reinterpret_cast<const float4*>(out2 + (size_t)k2 * G * D + c);
            }
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) top = fmaxf(top, lw[u]);
        if (top > M) {
            const float f = ex2((M - top) * kLog2e);        // 0 the first time
            den *= f;
#pragma unroll
            for (int c = 0; c < C; ++c) num[c] *= f;
            M = top;
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            // -inf: no piece, or one the row saw nothing of and whose values mean nothing (a NaN is carried on)
            const bool holds = lw[u] != -INFINITY;
            const float w = holds ? ex2((lw[u] - M) * kLog2e) : 0.f;
            den += w;
#pragma unroll
            for (int c = 0; c < C; ++c) num[c] = fmaf(w, holds ? x[u][c] : 0.f, num[c]);
        }
    }
    if constexpr (kWP > 1) {
        s_max[warp][lane] = M;
        s_den[warp][lane] = den;
#pragma unroll
        for (int c = 0; c < C; ++c) s_num[warp][c][lane] = num[c];
        __syncthreads();
        if (wp != 0) return;
        float top = M;
#pragma unroll
        for (int w = 1; w < kWP; ++w) top = fmaxf(top, s_max[warp + w][lane]);
        const float sub = top == -INFINITY ? 0.f : top;         // nothing anywhere: 0 weights
        const float f = ex2((M - sub) * kLog2e);
        den *= f;
#pragma unroll
        for (int c = 0; c < C; ++c) num[c] *= f;
#pragma unroll
        for (int w = 1; w < kWP; ++w) {
            const float fw = ex2((s_max[warp + w][lane] - sub) * kLog2e);
            den = fmaf(fw, s_den[warp + w][lane], den);
#pragma unroll
            for (int c = 0; c < C; ++c) num[c] = fmaf(fw, s_num[warp + w][c][lane], num[c]);
        }
    }
    if (!active) return;
    const float inv = has1 || has2 ? 1.f / den : 0.f;           // an empty sequence gives a zero row
    __nv_bfloat16* o = p.out + ((size_t)s * p.Hq + kvh * G + hh) * D + d0;
    if constexpr (C % 8 == 0) {
#pragma unroll
        for (int c = 0; c < C; c += 8)
            *reinterpret_cast<uint4*>(o + c) = make_uint4(pack2(num[c] * inv, num[c + 1] * inv), pack2(num[c + 2] * inv, num[c + 3] * inv),
                                                          pack2(num[c + 4] * inv, num[c + 5] * inv), pack2(num[c + 6] * inv, num[c + 7] * inv));
    } else {
#pragma unroll
        for (int c = 0; c < C; c += 4)
            *reinterpret_cast<uint2*>(o + c) = make_uint2(pack2(num[c] * inv, num[c + 1] * inv), pack2(num[c + 2] * inv, num[c + 3] * inv));
    }
}

// ----------------------------------------------------------------------------- host
// q [B, Hq, D] as a 3-D tensor; a box is 64 dims x the G heads of a group x `seqs` sequences.
bool make_q_map(CUtensorMap* map, const void* q, int B, int Hq, int G, int D, int seqs) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)Hq, (cuuint64_t)B};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)Hq * D * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)seqs};
    return make_bf16_map(map, q, 3, dims, strides, box);
}

// The cache as a 3-D tensor [64-dim halves, rows, 64]; a box is the bs token rows of a page, half after half.
bool make_slice_map(CUtensorMap* map, const void* cache, uint64_t rows, int D, int bs) {
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(D / 64)};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, 128};
    const cuuint32_t box[3] = {64, (cuuint32_t)bs, (cuuint32_t)(D / 64)};
    return make_bf16_map(map, cache, 3, dims, strides, box);
}

struct Maps {
    CUtensorMap q, q1, k, v;
};

template <int D, int G>
int launch_both(const Maps& maps, const SharedParams& p, const MergeParams& m, unsigned ctas, cudaStream_t stream) {
    static std::atomic<bool> configured[kMaxDevices];
    if (!ensure_smem_limit(decode_shared_kernel<D, G>, ShLayout<D>::kSmemBytes, configured)) return OPT_GQA_ERR_CUDA;
    const int rc = launch_dependent(decode_shared_kernel<D, G>, dim3(ctas), dim3(kThreads), ShLayout<D>::kSmemBytes, stream,
                                    maps.q, maps.q1, maps.k, maps.v, p);
    if (rc != OPT_GQA_OK) return rc;
    const unsigned slabs = (unsigned)((p.B + 32 / G - 1) / (32 / G));
    auto merge = [&](auto kernel, unsigned z) {
        return launch_dependent(kernel, dim3(slabs, (unsigned)p.Hkv, z), dim3(kMergeWarps * 32), 0, stream, m);
    };
    // About 512 CTAs, a wave of them: of few rows many warps share the pieces and a CTA takes few columns, of many rows a
    // CTA takes all of them.
    const long long cells = (long long)slabs * p.Hkv;
    if (cells <= 16) return merge(merge_shared_kernel<D, G, 8, 4>, D / 4);
    if (cells <= 32) return merge(merge_shared_kernel<D, G, 8, 8>, D / 8);
    if (cells <= 64) return merge(merge_shared_kernel<D, G, 8, D / 8>, 8);
    if (cells <= 128) return merge(merge_shared_kernel<D, G, 4, D / 8>, 4);
    if (cells <= 256) return merge(merge_shared_kernel<D, G, 2, D / 8>, 2);
    return merge(merge_shared_kernel<D, G, 1, D / 8>, 1);
}

template <int D>
int launch_g(const Maps& maps, const SharedParams& p, const MergeParams& m, int G, unsigned ctas, cudaStream_t stream) {
    switch (G) {
        case 1: return launch_both<D, 1>(maps, p, m, ctas, stream);
        case 2: return launch_both<D, 2>(maps, p, m, ctas, stream);
        case 4: return launch_both<D, 4>(maps, p, m, ctas, stream);
        case 8: return launch_both<D, 8>(maps, p, m, ctas, stream);
    }
    return OPT_GQA_ERR_SHAPE;
}

}  // namespace

int launch_decode_shared(void* out, const void* q, const void* k_cache, const void* v_cache, const int32_t* block_tables,
                         int max_blocks_per_seq, const int32_t* context_lens, const int32_t* group_start,
                         const int32_t* prefix_lens, int num_groups, const float* alibi_slopes, float scale, int B, int Hq,
                         int Hkv, int D, int bs, int64_t num_blocks, int64_t max_context, void* workspace,
                         int* device_status, cudaStream_t stream) {
    const uint64_t rows = (uint64_t)num_blocks * (uint64_t)Hkv * (uint64_t)bs;
    if (rows == 0 || rows > 0x7fffffffull) return OPT_GQA_ERR_SHAPE;
    const int G = Hq / Hkv, N = num_groups;
    const SharedLayout L = shared_layout(B, Hq, Hkv, D, N);
    if (L.group_pieces > 0x7fffffffull || L.own_pieces > 0x7fffffffull) return OPT_GQA_ERR_SHAPE;
    const int sms = sm_count();
    if (sms <= 0) return OPT_GQA_ERR_CUDA;
    Maps maps;
    if (!make_q_map(&maps.q, q, B, Hq, G, D, kRows / G) || !make_q_map(&maps.q1, q, B, Hq, G, D, 1) ||
        !make_cache_map(&maps.k, k_cache, rows, D, bs) || !make_slice_map(&maps.v, v_cache, rows, D, bs))
        return OPT_GQA_ERR_CUDA;
    char* ws = static_cast<char*>(workspace);
    SharedParams p;
    p.block_tables = block_tables;
    p.context_lens = context_lens;
    p.prefix_lens = prefix_lens;
    p.group_start = group_start;
    p.slopes = alibi_slopes;
    p.info = reinterpret_cast<int32_t*>(ws + L.info);
    p.group_lse = reinterpret_cast<float*>(ws + L.group_lse);
    p.group_out = reinterpret_cast<float*>(ws + L.group_out);
    p.own_lse = reinterpret_cast<float*>(ws + L.own_lse);
    p.own_out = reinterpret_cast<float*>(ws + L.own_out);
    p.status = device_status;
    p.scale = scale;
    p.num_groups = N;
    p.B = B;
    p.max_blocks = max_blocks_per_seq;
    p.Hkv = Hkv;
    p.bs = bs;
    p.bs_log2 = bs == 32 ? 5 : 4;
    p.lanes_log2 = 0;           // lanes that scan one group's sequences: about the mean size of a group
    while (p.lanes_log2 < 5 && ((long long)N << p.lanes_log2) < B) ++p.lanes_log2;
    MergeParams m;
    m.out = static_cast<__nv_bfloat16*>(out);
    m.context_lens = context_lens;
    m.prefix_lens = prefix_lens;
    m.group_start = group_start;
    m.info = p.info;
    m.group_lse = p.group_lse;
    m.group_out = p.group_out;
    m.own_lse = p.own_lse;
    m.own_out = p.own_out;
    m.num_groups = N;
    m.B = B;
    m.Hq = Hq;
    m.Hkv = Hkv;
    m.group_pieces = (int)L.group_pieces;
    m.own_pieces = (int)L.own_pieces;
    // one resident wave, and no more workers than there can be tiles
    const long long most = (long long)Hkv * (N + (long long)B * G / kRows + B) * ((max_context + kTN - 1) / kTN);
    long long ctas = (long long)sms * kCtasPerSm;
    if (ctas > kSharedMaxWorkers) ctas = kSharedMaxWorkers;
    if (ctas > most) ctas = most;
    return D == 128 ? launch_g<128>(maps, p, m, G, (unsigned)ctas, stream) : launch_g<64>(maps, p, m, G, (unsigned)ctas, stream);
}

}  // namespace optgqa
