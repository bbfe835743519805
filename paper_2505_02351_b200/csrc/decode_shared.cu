// Decode attention for a batch whose sequences share long prefixes (one prompt, many continuations): the keys and values
// of a shared prefix are brought on-chip once for all sequences of its group instead of once per sequence.
//
// Softmax over disjoint sets of keys merges exactly from each set's normalised result and log-sum-exp, so
//     out = (e^{lse_P} o_P + e^{lse_S} o_S) / (e^{lse_P} + e^{lse_S}),
// P the shared keys (this file), S the sequence's own (decode_stream.cu with a first tile per sequence).  In the group
// pass the n_g sequences of a group times the G query heads of a KV head are the rows of one product with the prefix's
// keys -- a real matrix product, with 2 n_g G flops per byte of the cache -- so it runs on tcgen05: per item (group, KV head,
// block of 128 rows) S = Q K^T and O += P V over 64-key tiles, accumulators in tensor memory, exactly as a query block of
// the chunked prefill without its causal mask.  Up to 128 rows the pass is bound by reading the cache (a 32 KB tile takes
// an SM's share of the bandwidth 1480 cycles, the two resident CTAs need about 900 for its arithmetic); beyond, by the
// special-function unit and the tensor core as the prefill is.
//
// The tiles of all items are laid end to end and cut into one contiguous range per worker (two CTAs per SM), so that one
// long prefix fills the GPU as well as many short ones.  A worker's part of an item is a piece: 128 normalised partial
// rows and log-sum-exps in the workspace, merged with the own pass's pieces by merge_shared_kernel.
//
// Rows see whole tiles only: sequence s attends to the first e_s = floor(min(prefix, n_s) / 64) * 64 tokens here and to the
// rest in its own pass.  So no tile is masked inside, and where sequences of a group differ in e_s (the tiles are taken from
// the last one backwards) a row that has not begun simply discards what it accumulated: its O is set to zero, not
// multiplied by zero, at its first tile, and nothing it does not see can reach it, not even a NaN.
//
// Eight warps: 0-3 one thread per row (softmax), 4 and 6 the TMA producers of Q, K and of V, 5 and 7 issue S = Q K^T and
// O += P V.  All of them walk the same list of pieces.  Every wait is a bounded mbarrier wait.  (A single producer was what
// the pass waited for: a copy of 16 rows costs its warp about 90 cycles, 16 of them a tile; and a single issuing thread
// adds the waits for K, V and P up, 1690 cycles a tile against 1100 of softmax.)
#include "umma.cuh"

namespace optgqa {

namespace {

constexpr int kRows = kSharedRows;
constexpr int kTN = kSharedTile;
constexpr int kKStages = 3;
constexpr int kVStages = 2;
constexpr int kThreads = 256;
constexpr int kMaxRegs = 160;              // two of these warps and one of the own pass's (184) share a scheduler's 512
constexpr int kMinTiles = 2;               // tiles a worker gets at least
constexpr unsigned kFull = 0xffffffffu;
constexpr float kRescaleThreshold = 8.f;   // log2 units: O is rescaled only when a row's maximum grew by more

constexpr int kHalfBytes = kTN * 128;      // one 64-dim column half of a K or V tile
constexpr int kQHalfBytes = kRows * 128;   // one 64-dim column half of the Q tile
// The ALiBi term inside a tile rides on the tensor core as one more k-step (see prefill_umma.cu): slope / |scale| as
// three bf16 values against the key's index in the tile.
constexpr int kExtRowGroupBytes = 256;
constexpr int kQxBytes = kRows / 8 * kExtRowGroupBytes;
constexpr int kKpBytes = kTN / 8 * kExtRowGroupBytes;
// barriers: q_full, q_empty, qx_full, o_empty, k_full[], k_empty[], v_full[], v_empty[], s_full[2], p_full[2]
constexpr int kNumBars = 4 + 2 * kKStages + 2 * kVStages + 4;

template <int D>
struct ShLayout {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kQBytes = kHalves * kQHalfBytes;
    static constexpr int kOffQ = 0;
    static constexpr int kOffK = kQBytes;
    static constexpr int kOffV = kOffK + kKStages * kTileBytes;
    static constexpr int kOffQx = kOffV + kVStages * kTileBytes;
    static constexpr int kOffKp = kOffQx + kQxBytes;
    static constexpr int kOffBar = kOffKp + kKpBytes;
    static constexpr int kOffGroups = kOffBar + kNumBars * 8 + 16;      // tiles before (8 B), tiles, leader, items before (2 B)
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
    float* partial_out;
    float* partial_lse;
    int32_t* info;              // per (sequence, KV head): see SharedLayout
    int* status;
    float scale;
    int num_groups, B, max_blocks, Hq, Hkv, bs, lanes_log2;
};

// A worker's place in the items laid end to end: (group, KV head, row block), row block fastest, so that the blocks of one
// prefix are worked on at the same time and its tiles come from L2 after their first reading.
struct PieceCursor {
    int g, kvh, mt;             // the item
    int kt, blocks, jt;         // its tiles, the group's row blocks, the tile inside the item
    long long item, pos;        // number of the item, position in the tiles of all items
};

template <int D, int G>
__global__ void __maxnreg__(kMaxRegs)
decode_shared_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const SharedParams p) {
    using L = ShLayout<D>;
    constexpr int kTileBytes = L::kTileBytes, kOffQ = L::kOffQ, kOffK = L::kOffK, kOffV = L::kOffV, kOffQx = L::kOffQx,
                  kOffKp = L::kOffKp;
    constexpr int TQ = kRows / G;          // sequences per row block
    extern __shared__ char smem_raw[];
    char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
    uint64_t* q_full = bars;
    uint64_t* q_empty = bars + 1;
    uint64_t* qx_full = bars + 2;
    uint64_t* o_empty = bars + 3;
    uint64_t* k_full = bars + 4;
    uint64_t* k_empty = k_full + kKStages;
    uint64_t* v_full = k_empty + kKStages;
    uint64_t* v_empty = v_full + kVStages;
    uint64_t* s_full = v_empty + kVStages;
    uint64_t* p_full = s_full + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
    long long* g_tiles = reinterpret_cast<long long*>(smem + L::kOffGroups);     // exclusive sums over the groups, one head
    int* g_kt = reinterpret_cast<int*>(g_tiles + kMaxGroups);
    int* g_lead = g_kt + kMaxGroups;
    uint16_t* g_items = reinterpret_cast<uint16_t*>(g_lead + kMaxGroups);        // at most kMaxGroups + 65535 * 8 / 128

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int N = p.num_groups;
    if (threadIdx.x == 128) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    auto group_lo = [&](int g) { return min(max(__ldg(p.group_start + g), 0), p.B); };
    auto blocks_of = [&](int g) { return max(group_lo(g + 1) - group_lo(g), 0) * G / kRows +
                                         (max(group_lo(g + 1) - group_lo(g), 0) * G % kRows != 0); };

    // ------------------------------------------------------------------ the groups: longest shared run, whose it is
    // (the index arrays are read before the wait for the preceding kernel: see the ordering contract in the header)
    if (warp < 4) {
        const int lanes = 1 << p.lanes_log2, sub = lane & (lanes - 1), per_warp = 32 >> p.lanes_log2;
        for (int g0 = warp * per_warp; g0 < N; g0 += 4 * per_warp) {
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
            }
        }
    }
    if (threadIdx.x == 128) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        mbar_init(qx_full, kRows);
        mbar_init(o_empty, kRows);
#pragma unroll
        for (int i = 0; i < kKStages; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], 1);
        }
#pragma unroll
        for (int i = 0; i < kVStages; ++i) {
            mbar_init(&v_full[i], 1);
            mbar_init(&v_empty[i], 1);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], kRows);
        }
        tmem_slot[1] = 0;
        fence_barrier_init();
    }
    // The scale may have any sign (see prefill_umma.cu).
    const float sabs = p.scale == 0.f ? 1.f : fabsf(p.scale);
    const bool alibi = p.slopes != nullptr || p.scale == 0.f;
    if (alibi && threadIdx.x >= kRows) {
        for (int e = threadIdx.x - kRows; e < kTN; e += kThreads - kRows) {
            const uint32_t eb = __bfloat16_as_ushort(__float2bfloat16_rn((float)e));      // exact: e < 256
            char* row = smem + kOffKp + (e >> 3) * kExtRowGroupBytes + (e & 7) * 16;
            *reinterpret_cast<uint4*>(row) = make_uint4(eb | (eb << 16), eb, 0u, 0u);
            *reinterpret_cast<uint4*>(row + 128) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async();
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncthreads();
    // Exclusive sums over the groups, by one warp.  A group_start that is not increasing may name more row blocks than the
    // workspace has room for: the groups past it are left out (a wrong row, never a write outside).
    __shared__ long long s_total;
    if (warp == 0) {
        long long tiles = 0;
        int items = 0;
        const int most = N + (int)((long long)p.B * G / kRows);
        for (int g0 = 0; g0 < N; g0 += 32) {
            const int g = g0 + lane;
            int b = g < N && g_kt[g] > 0 ? blocks_of(g) : 0, kt = g < N ? g_kt[g] : 0;
            int incl = b;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(kFull, incl, o);
                if (lane >= o) incl += v;
            }
            if (items + incl > most) b = 0, kt = 0;       // (items + incl only grows: all later ones too)
            long long incl_t = (long long)b * kt;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(kFull, incl_t, o);
                if (lane >= o) incl_t += v;
            }
            if (g < N) {
                g_tiles[g] = tiles + incl_t - (long long)b * kt;
                g_items[g] = (uint16_t)min(items + incl - b, most);
                g_kt[g] = kt;
            }
            tiles += __shfl_sync(kFull, incl_t, 31);
            items += __shfl_sync(kFull, incl, 31);
        }
        if (lane == 0) s_total = tiles * p.Hkv;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const long long total = s_total, me = blockIdx.x;
    const long long by_size = total / kMinTiles > 0 ? total / kMinTiles : (total > 0 ? 1 : 0);
    const long long workers = by_size < gridDim.x ? by_size : gridDim.x;
    // The cache and q may still be written, the workspace still read, by the preceding kernel: the producer waits for it
    // before its first copy, and everything this CTA writes follows from that copy.  The kernel after this one (the own
    // pass) is let go only behind that wait: it then runs beside this grid without a wait of its own.
    if (total == 0) grid_dependency_wait();         // a grid none of whose CTAs waited could finish before its predecessor

    if (me < workers) {
        const long long lo = total * me / workers, hi = total * (me + 1) / workers;
        PieceCursor cur;
        auto enter_group = [&]() {
            cur.kt = g_kt[cur.g];
            cur.blocks = blocks_of(cur.g);
        };
        {
            int a = 0, b = N - 1;           // the last group whose tiles begin at or before lo and that has any
            while (a < b) {
                const int m = (a + b + 1) >> 1;
                if (g_tiles[m] * p.Hkv <= lo) a = m;
                else b = m - 1;
            }
            cur.g = a;
            enter_group();
            const long long r = lo - g_tiles[a] * p.Hkv;
            const int in_group = (int)(r / cur.kt);
            cur.jt = (int)(r - (long long)in_group * cur.kt);
            cur.kvh = in_group / cur.blocks;
            cur.mt = in_group - cur.kvh * cur.blocks;
            cur.item = (long long)g_items[a] * p.Hkv + in_group;
            cur.pos = lo;
        }
        auto piece_len = [&]() { return (int)min((long long)(cur.kt - cur.jt), hi - cur.pos); };
        auto next_piece = [&](int len) {
            cur.pos += len;
            cur.jt = 0;
            ++cur.item;
            if (cur.pos >= hi || ++cur.mt < cur.blocks) return;
            cur.mt = 0;
            if (++cur.kvh < p.Hkv) return;
            cur.kvh = 0;
            do ++cur.g;
            while (cur.g < N - 1 && g_kt[cur.g] == 0);
            enter_group();
            cur.item = (long long)g_items[cur.g] * p.Hkv;
        };

        if (warp == 4 || warp == 6) {
            // -------------------------------------------------------------- producers: warp 4 Q and K, warp 6 V
            // A slice is the bs tokens of a page.  K: one box of bs rows x 64 dims per slice and half, so that the 64 rows of
            // a half lie together; V: one box of all of a slice (see issue_pv for its layout).
            const bool is_k = warp == 4;
            const int slices = kTN / p.bs, sub = lane % slices, hf = lane / slices;
            const bool issues = lane < (is_k ? slices * L::kHalves : slices);
            uint64_t *full = is_k ? k_full : v_full, *empty = is_k ? k_empty : v_empty;
            const int stages = is_k ? kKStages : kVStages;
            char* ring = smem + (is_k ? kOffK + hf * kHalfBytes + sub * p.bs * 128 : kOffV + sub * p.bs * (D * 2));
            int pc = 0, st = 0;
            uint32_t ph = 1;                                    // parity of a stage's last release (none yet: passes)
            bool ok = true;
            while (ok && cur.pos < hi) {
                const int len = piece_len(), kvh = cur.kvh;
                const int32_t* table = p.block_tables + (size_t)g_lead[cur.g] * p.max_blocks;
                const int tile_hi = cur.jt + len - 1;
                auto page_of = [&](int j) {
                    return issues ? __ldg(table + min((tile_hi - j) * slices + sub, p.max_blocks - 1)) : 0;
                };
                int page = page_of(0);
                if (pc == 0) {
                    grid_dependency_wait();
                    if (is_k) grid_dependency_launch();
                }
                if (is_k) {
                    if (pc > 0) ok = __all_sync(kFull, mbar_wait(q_empty, (pc - 1) & 1, p.status));
                    if (!ok) break;
                    if (lane == 0) {
                        mbar_expect_tx(q_full, L::kQBytes);
#pragma unroll
                        for (int h = 0; h < L::kHalves; ++h)
                            tma_load_3d(smem + kOffQ + h * kQHalfBytes, &map_q, 64 * h, kvh * G, group_lo(cur.g) + cur.mt * TQ, q_full);
                    }
                }
                for (int j = 0; j < len; ++j) {
                    const int page_next = j + 1 < len ? page_of(j + 1) : 0;
                    const int row = (page * p.Hkv + kvh) * p.bs;                       // row of the [rows, D] view
                    ok = __all_sync(kFull, mbar_wait(&empty[st], ph, p.status));
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(&full[st], (uint32_t)kTileBytes);
                    __syncwarp();
                    if (issues) {
                        if (is_k) tma_load_2d(ring + st * kTileBytes, &map_k, 64 * hf, row, &full[st]);
                        else tma_load_3d(ring + st * kTileBytes, &map_v, 0, row, 0, &full[st]);
                    }
                    page = page_next;
                    if (++st == stages) st = 0, ph ^= 1;
                }
                next_piece(len);
                ++pc;
            }
        } else if (warp == 5) {
            // -------------------------------------------------------------- one thread issues S = Q K^T
            if (lane == 0) {
                constexpr uint32_t idesc_s = instr_desc(false, kTN);
                const uint32_t idesc_qk = p.scale < 0.f ? instr_desc(false, kTN, true) : idesc_s;
                const bool dots = p.scale != 0.f;
                uint64_t q_desc[D / 16];
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    q_desc[ks] = smem_desc(smem_u32(smem + kOffQ) + (ks >> 2) * kQHalfBytes + (ks & 3) * 32, 16, 1024);
                const uint64_t k_desc0 = smem_desc(smem_u32(smem + kOffK), 16, 1024);
                const uint64_t qx_desc = smem_desc_plain(smem_u32(smem + kOffQx), 128, kExtRowGroupBytes);
                const uint64_t kp_desc = smem_desc_plain(smem_u32(smem + kOffKp), 128, kExtRowGroupBytes);
                int it = 0, pc = 0, st = 0, vst = 0;
                uint32_t ph = 0, vph = 1;
                bool ok = true;
                while (ok && cur.pos < hi) {
                    const int len = piece_len();
                    ok = mbar_wait(q_full, pc & 1, p.status) && (!alibi || mbar_wait(qx_full, pc & 1, p.status));
                    for (int j = 0; ok && j < len; ++j, ++it) {
                        const int sb = it & 1;
                        // the score buffer is free once the P V of the tile before the last one has read its weights there
                        if (it >= 2) {
                            ok = mbar_wait(&v_empty[vst], vph ^ 1, p.status);
                            if (++vst == kVStages) vst = 0, vph ^= 1;
                        }
                        ok = ok && mbar_wait(&k_full[st], ph, p.status);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t kd = desc_advance(k_desc0, st * kTileBytes);
                        const uint32_t s_tmem = tmem_base + kColS + sb * kTN;
                        if (dots) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                umma_ss(s_tmem, q_desc[ks], desc_advance(kd, (ks >> 2) * kHalfBytes + (ks & 3) * 32), idesc_qk, ks > 0);
                        }
                        if (alibi) umma_ss(s_tmem, qx_desc, kp_desc, idesc_s, dots);
                        tc_commit(&s_full[sb]);
                        tc_commit(&k_empty[st]);
                        if (j == len - 1) tc_commit(q_empty);
                        if (++st == kKStages) st = 0, ph ^= 1;
                    }
                    next_piece(len);
                    ++pc;
                }
            }
        } else if (warp == 7) {
            // -------------------------------------------------------------- one thread issues O (+)= P V
            if (lane == 0) {
                constexpr uint32_t idesc_pv = instr_desc(true, D);
                // V is MN-major, in slices of bs keys with the 64-dim halves of a slice side by side: halves bs * 128 bytes
                // apart (leading offset), groups of 8 keys 1 KiB apart (stride offset), slices bs * D * 2 bytes.
                const uint64_t v_desc0 = smem_desc(smem_u32(smem + kOffV), p.bs * 128, 1024);
                int it = 0, pc = 0, st = 0;
                uint32_t ph = 0;
                bool ok = true;
                while (ok && cur.pos < hi) {
                    const int len = piece_len();
                    for (int j = 0; ok && j < len; ++j, ++it) {
                        const int sb = it & 1;
                        ok = mbar_wait(&v_full[st], ph, p.status) && mbar_wait(&p_full[sb], (it >> 1) & 1, p.status) &&
                             (j > 0 || pc == 0 || mbar_wait(o_empty, (pc - 1) & 1, p.status));    // O of the piece before is read
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t vd = desc_advance(v_desc0, st * kTileBytes);
                        const uint32_t p_tmem = tmem_base + kColS + sb * kTN;
#pragma unroll
                        for (int kk = 0; kk < kTN / 16; ++kk) {
                            const uint32_t at = p.bs == 16 ? kk * 16 * (D * 2) : (kk >> 1) * 32 * (D * 2) + (kk & 1) * 2048;
                            umma_ts(tmem_base + kColO, p_tmem + kk * 8, desc_advance(vd, at), idesc_pv, j > 0 || kk > 0);
                        }
                        tc_commit(&v_empty[st]);
                        if (++st == kVStages) st = 0, ph ^= 1;
                    }
                    next_piece(len);
                    ++pc;
                }
            }
        } else {
            // -------------------------------------------------------------- one thread per row: softmax, rescale, store
            const int r = threadIdx.x, hg = r % G;
            const float qscale = sabs * kLog2e;
            const uint32_t lane_addr = tmem_base + ((uint32_t)(warp * 32) << 16);
            // The row of the ALiBi step's operand for KV head kvh: slope / |scale| as a sum of three bf16 values.
            auto write_qx = [&](int kvh) {
                const float a = p.slopes ? p.slopes[kvh * G + hg] / sabs : 0.f;
                const __nv_bfloat16 a0 = __float2bfloat16_rn(a);
                const __nv_bfloat16 a1 = __float2bfloat16_rn(a - __bfloat162float(a0));
                const __nv_bfloat16 a2 = __float2bfloat16_rn(a - __bfloat162float(a0) - __bfloat162float(a1));
                char* row = smem + kOffQx + (r >> 3) * kExtRowGroupBytes + (r & 7) * 16;
                *reinterpret_cast<uint4*>(row) = make_uint4((uint32_t)__bfloat16_as_ushort(a0) | ((uint32_t)__bfloat16_as_ushort(a1) << 16),
                                                            (uint32_t)__bfloat16_as_ushort(a2), 0u, 0u);
                *reinterpret_cast<uint4*>(row + 128) = make_uint4(0u, 0u, 0u, 0u);
                fence_proxy_async();
                mbar_arrive(qx_full);
            };
            if (alibi) write_qx(cur.kvh);
            int it = 0, st = 0;                     // tile, and the stage and parity of its V
            uint32_t ph = 0;
            // waits for the P V of the tile before this one
            auto prev_pv_done = [&]() {
                const int ps = st == 0 ? kVStages - 1 : st - 1;
                return __all_sync(kFull, mbar_wait(&v_empty[ps], st == 0 ? ph ^ 1 : ph, p.status));
            };
            bool ok = true;
            while (ok && cur.pos < hi) {
                const int len = piece_len(), tile_hi = cur.jt + len - 1;
                const int kvh = cur.kvh;
                const long long row0 = (cur.item + me) * kRows;
                const int i = cur.mt * TQ + r / G, s = group_lo(cur.g) + i;
                const bool valid = s < group_lo(cur.g + 1);
                const int n = valid ? __ldg(p.context_lens + s) : 0;
                const int e_row = valid ? shared_tokens(__ldg(p.prefix_lens + s), n) : 0;      // keys the row sees
                const float slope2 = p.slopes ? __ldg(p.slopes + kvh * G + hg) * kLog2e : 0.f;
                const bool opens = cur.jt == 0, closes = cur.jt + len == cur.kt;
                next_piece(len);                    // `cur` is the piece after this one from here on
                float m_used = -INFINITY, l = 0.f;

                auto next_tile = [&]() {
                    ++it;
                    if (++st == kVStages) st = 0, ph ^= 1;
                };
                for (int j = 0; j < len; ++j, next_tile()) {
                    const int sb = it & 1, j0 = (tile_hi - j) * kTN;
                    ok = __all_sync(kFull, mbar_wait(&s_full[sb], (it >> 1) & 1, p.status));
                    if (!ok) break;
                    tc_fence_after();
                    // the piece's last scores are there: nothing reads its ALiBi operand any more
                    if (alibi && j == len - 1 && cur.pos < hi) write_qx(cur.kvh);
                    const bool sees = j0 < e_row;
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
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < kTN / 32; ++c) chunk_max<false>(v[c], 0, 0, 0, mx);
                    const float m_tile = fmaf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), qscale, bias0);
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
#pragma unroll
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
                            sum += chunk_exp<false>(v[c], qscale, bias_m, 0, 0, 0, w);
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
                ok = prev_pv_done();
                if (!ok) break;
                tc_fence_after();
                if (__any_sync(kFull, valid)) {
                    const float inv = 1.f / l;
                    const bool begun = (tile_hi - len + 1) * kTN < e_row;          // the row saw a tile of the piece
                    float* po = p.partial_out + row0 * D + r;                       // [D][kRows]: 32 rows are one line
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        float o[32];
                        tmem_ld32(lane_addr + kColO + c * 32, o);
                        if (begun) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) po[(c * 32 + e) * kRows] = o[e] * inv;
                        }
                    }
                    // a row that saw nothing of the piece: weight zero
                    if (e_row > 0 && hg == 0) {
                        int32_t* info = p.info + ((size_t)s * p.Hkv + kvh) * kInfoWords;
                        if (opens) info[0] = (int)(row0 / kRows), info[1] = r;
                        if (closes) info[2] = (int)(row0 / kRows);
                    }
                    if (valid) p.partial_lse[row0 + r] = begun ? (m_used + lg2(l)) * kLn2 : -INFINITY;
                }
                tc_fence_before();
                mbar_arrive(o_empty);
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
// A CTA merges 32 rows: 32 / G consecutive sequences times the G heads of one KV head, a lane per row, so that the group
// pass's pieces ([D][128 rows]) are read as whole lines.  Per row the pieces are one list: the group pass's that cover the
// sequence's item (numbers item + w, w consecutive workers), then the own pass's (consecutive rows, see reduce.cu).  kWP of
// the CTA's eight warps share the list, the others (and the grid's y) take other columns, C of them per lane.
constexpr int kMergeWarps = 8;

struct MergeParams {
    __nv_bfloat16* out;
    const int32_t* context_lens;
    const int32_t* prefix_lens;
    const int32_t* group_start;
    const int32_t* info;
    const float* sh_lse;
    const float* sh_out;
    const float* own_lse;
    const float* own_out;
    int num_groups, B, Hq, Hkv;
};

template <int D, int G, int kWP, int C>
__global__ void __launch_bounds__(kMergeWarps * 32)
merge_shared_kernel(const MergeParams p) {
    constexpr int kSeqs = 32 / G;
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

    // group pass: R1 pieces of kRows rows; own pass: R2 pieces of G rows
    const int32_t* info = p.info + ((size_t)(active ? s : 0) * p.Hkv + kvh) * kInfoWords;
    const int4 i0 = *reinterpret_cast<const int4*>(info);
    const int2 i1 = *reinterpret_cast<const int2*>(info + 4);
    const int R1 = has1 ? i0.z - i0.x + 1 : 0, R2 = has2 ? i1.y - i1.x + 1 : 0;
    const float* lse1 = p.sh_lse + (has1 ? (size_t)i0.x * kRows + i0.y + hh : 0);
    const float* po1 = p.sh_out + (has1 ? ((size_t)i0.x * D + d0) * kRows + i0.y + hh : 0);
    const float* lse2 = p.own_lse + (has2 ? (size_t)i1.x * G + hh : 0);
    const float* po2 = p.own_out + (has2 ? ((size_t)i1.x * G + hh) * D + d0 : 0);
    const int R = R1 + R2;
    float M = -INFINITY;
    for (int i = wp; i < R1; i += kWP) M = fmaxf(M, lse1[(size_t)i * kRows]);
    for (int i = wp; i < R2; i += kWP) M = fmaxf(M, lse2[(size_t)i * G]);
    if (kWP > 1) {
        s_max[warp][lane] = M;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWP; ++w) M = fmaxf(M, s_max[warp - wp + w][lane]);
    }
    float num[C], den = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) num[c] = 0.f;
    // (loads do not wait for the weight: a row that holds nothing, lse -inf, is selected away; a NaN is carried on)
#pragma unroll 2
    for (int i = wp; i < R1; i += kWP) {
        const float lw = lse1[(size_t)i * kRows];
        const float* x = po1 + (size_t)i * kRows * D;
        float y[C];
#pragma unroll
        for (int c = 0; c < C; ++c) y[c] = x[c * kRows];
        const bool holds = lw != -INFINITY;
        const float w = holds ? ex2((lw - M) * kLog2e) : 0.f;
        den += w;
#pragma unroll
        for (int c = 0; c < C; ++c) num[c] = fmaf(w, holds ? y[c] : 0.f, num[c]);
    }
#pragma unroll 2
    for (int i = wp; i < R2; i += kWP) {
        const float lw = lse2[(size_t)i * G];
        const float4* x = reinterpret_cast<const float4*>(po2 + (size_t)i * G * D);
        float4 y[C / 4];
#pragma unroll
        for (int c = 0; c < C / 4; ++c) y[c] = x[c];
        const bool holds = lw != -INFINITY;
        const float w = holds ? ex2((lw - M) * kLog2e) : 0.f;
        den += w;
#pragma unroll
        for (int c = 0; c < C / 4; ++c) {
            num[4 * c] = fmaf(w, holds ? y[c].x : 0.f, num[4 * c]);
            num[4 * c + 1] = fmaf(w, holds ? y[c].y : 0.f, num[4 * c + 1]);
            num[4 * c + 2] = fmaf(w, holds ? y[c].z : 0.f, num[4 * c + 2]);
            num[4 * c + 3] = fmaf(w, holds ? y[c].w : 0.f, num[4 * c + 3]);
        }
    }
    if constexpr (kWP > 1) {
        s_den[warp][lane] = den;
#pragma unroll
        for (int c = 0; c < C; ++c) s_num[warp][c][lane] = num[c];
        __syncthreads();
        if (wp != 0) return;
#pragma unroll
        for (int w = 1; w < kWP; ++w) {
            den += s_den[warp + w][lane];
#pragma unroll
            for (int c = 0; c < C; ++c) num[c] += s_num[warp + w][c][lane];
        }
    }
    if (!active) return;
    const float inv = R > 0 ? 1.f / den : 0.f;                  // an empty sequence gives a zero row
    uint4* o = reinterpret_cast<uint4*>(p.out + ((size_t)s * p.Hq + kvh * G + hh) * D + d0);
#pragma unroll
    for (int c = 0; c < C / 8; ++c)
        o[c] = make_uint4(pack2(num[8 * c] * inv, num[8 * c + 1] * inv), pack2(num[8 * c + 2] * inv, num[8 * c + 3] * inv),
                          pack2(num[8 * c + 4] * inv, num[8 * c + 5] * inv), pack2(num[8 * c + 6] * inv, num[8 * c + 7] * inv));
}

// ----------------------------------------------------------------------------- host
// q [B, Hq, D] as a 3-D tensor; a box is 64 dims x the G heads of a group x 128 / G sequences.
bool make_q_map(CUtensorMap* map, const void* q, int B, int Hq, int G, int D) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)Hq, (cuuint64_t)B};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)Hq * D * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)(kRows / G)};
    return make_bf16_map(map, q, 3, dims, strides, box);
}

// The cache as a 3-D tensor [64-dim halves, rows, 64]; a box is the bs token rows of a page, half after half.
bool make_slice_map(CUtensorMap* map, const void* cache, uint64_t rows, int D, int bs) {
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(D / 64)};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, 128};
    const cuuint32_t box[3] = {64, (cuuint32_t)bs, (cuuint32_t)(D / 64)};
    return make_bf16_map(map, cache, 3, dims, strides, box);
}

template <int D, int G>
int launch_pass(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const SharedParams& p, unsigned ctas,
                cudaStream_t stream) {
    static std::atomic<bool> configured[kMaxDevices];
    if (!ensure_smem_limit(decode_shared_kernel<D, G>, ShLayout<D>::kSmemBytes, configured, true)) return OPT_GQA_ERR_CUDA;
    return launch_dependent(decode_shared_kernel<D, G>, dim3(ctas), dim3(kThreads), ShLayout<D>::kSmemBytes, stream, mq, mk,
                            mv, p);
}

template <int D>
int launch_pass_g(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const SharedParams& p, int G,
                  unsigned ctas, cudaStream_t stream) {
    switch (G) {
        case 1: return launch_pass<D, 1>(mq, mk, mv, p, ctas, stream);
        case 2: return launch_pass<D, 2>(mq, mk, mv, p, ctas, stream);
        case 4: return launch_pass<D, 4>(mq, mk, mv, p, ctas, stream);
        case 8: return launch_pass<D, 8>(mq, mk, mv, p, ctas, stream);
    }
    return OPT_GQA_ERR_SHAPE;
}

template <int D, int G>
int launch_merge(const MergeParams& p, cudaStream_t stream) {
    const unsigned slabs = (unsigned)((p.B + 32 / G - 1) / (32 / G));
    auto launch = [&](auto kernel, unsigned z) {
        return launch_dependent(kernel, dim3(slabs, (unsigned)p.Hkv, z), dim3(kMergeWarps * 32), 0, stream, p);
    };
    // Few rows: eight warps share a row's pieces and a CTA takes 8 columns; many rows: a CTA takes all of a row.
    if ((long long)slabs * p.Hkv <= 128) return launch(merge_shared_kernel<D, G, 8, 8>, D / 8);
    return launch(merge_shared_kernel<D, G, 1, D / 8>, 1);
}

template <int D>
int launch_merge_g(const MergeParams& p, int G, cudaStream_t stream) {
    switch (G) {
        case 1: return launch_merge<D, 1>(p, stream);
        case 2: return launch_merge<D, 2>(p, stream);
        case 4: return launch_merge<D, 4>(p, stream);
        case 8: return launch_merge<D, 8>(p, stream);
    }
    return OPT_GQA_ERR_SHAPE;
}

}  // namespace

int launch_decode_shared(void* out, const void* q, const void* k_cache, const void* v_cache, const int32_t* block_tables,
                         int max_blocks_per_seq, const int32_t* context_lens, const SharedPrefix& shared,
                         const float* alibi_slopes, float scale, int B, int Hq, int Hkv, int D, int bs,
                         int64_t num_blocks, int partition_size, void* workspace, int max_partitions,
                         int* device_status, cudaStream_t stream) {
    const uint64_t rows = (uint64_t)num_blocks * (uint64_t)Hkv * (uint64_t)bs;
    if (rows == 0 || rows > 0x7fffffffull) return OPT_GQA_ERR_SHAPE;
    const int G = Hq / Hkv, N = shared.num_groups;
    const SharedLayout L = shared_layout(B, Hq, Hkv, D, N, max_partitions);
    if (L.own.rows > 0x7fffffffull || L.rows / kSharedRows > 0x7fffffffull) return OPT_GQA_ERR_SHAPE;
    const int sms = sm_count();
    if (sms <= 0) return OPT_GQA_ERR_CUDA;
    CUtensorMap mq, mk, mv;
    if (!make_q_map(&mq, q, B, Hq, G, D) || !make_cache_map(&mk, k_cache, rows, D, bs) ||
        !make_slice_map(&mv, v_cache, rows, D, bs))
        return OPT_GQA_ERR_CUDA;
    char* ws = static_cast<char*>(workspace);
    SharedParams p;
    p.block_tables = block_tables;
    p.context_lens = context_lens;
    p.prefix_lens = shared.prefix_lens;
    p.group_start = shared.group_start;
    p.slopes = alibi_slopes;
    p.partial_out = reinterpret_cast<float*>(ws + L.out);
    p.partial_lse = reinterpret_cast<float*>(ws + L.lse);
    p.info = reinterpret_cast<int32_t*>(ws + L.info);
    p.status = device_status;
    p.scale = scale;
    p.num_groups = N;
    p.B = B;
    p.max_blocks = max_blocks_per_seq;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.bs = bs;
    p.lanes_log2 = 0;           // lanes that scan one group's sequences: about the mean size of a group
    while (p.lanes_log2 < 5 && ((long long)N << p.lanes_log2) < B) ++p.lanes_log2;
    // one CTA per multiprocessor, beside one of the own pass
    const int ctas = sms < kSharedMaxWorkers ? sms : kSharedMaxWorkers;
    int rc = D == 128 ? launch_pass_g<128>(mq, mk, mv, p, G, (unsigned)ctas, stream)
                      : launch_pass_g<64>(mq, mk, mv, p, G, (unsigned)ctas, stream);
    if (rc != OPT_GQA_OK) return rc;
    SharedPrefix own = shared;
    own.info = p.info;
    rc = launch_decode_stream(q, k_cache, v_cache, block_tables, max_blocks_per_seq, context_lens, alibi_slopes, scale, B, Hq,
                              Hkv, D, bs, num_blocks, partition_size, workspace, max_partitions, 0, device_status, stream,
                              nullptr, &own);
    if (rc != OPT_GQA_OK) return rc;
    MergeParams m;
    m.out = static_cast<__nv_bfloat16*>(out);
    m.context_lens = context_lens;
    m.prefix_lens = shared.prefix_lens;
    m.group_start = shared.group_start;
    m.info = p.info;
    m.sh_lse = p.partial_lse;
    m.sh_out = p.partial_out;
    m.own_lse = reinterpret_cast<const float*>(ws + L.own.lse);
    m.own_out = reinterpret_cast<const float*>(ws + L.own.out);
    m.num_groups = N;
    m.B = B;
    m.Hq = Hq;
    m.Hkv = Hkv;
    return D == 128 ? launch_merge_g<128>(m, G, stream) : launch_merge_g<64>(m, G, stream);
}

}  // namespace optgqa
