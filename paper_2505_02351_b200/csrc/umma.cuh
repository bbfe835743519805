// Shared by the kernels on tcgen05 (prefill_umma.cu, decode_shared.cu, chunk.cu): instruction wrappers, descriptors, and the two
// passes of a row thread over a chunk of its scores.
#pragma once

#include "tma_mma.cuh"

namespace optgqa {

// ----------------------------------------------------------------------------- PTX wrappers
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Arrives on `bar` once every tcgen05.mma issued so far by this thread has completed.
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                 : "memory");
}

// Shared-memory matrix descriptor: 128-byte swizzle, descriptor version 1.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo_bytes >> 4) << 16) | ((uint64_t)(sbo_bytes >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

// Shared-memory matrix descriptor without swizzle (core matrices of 8 rows x 16 bytes): lbo = distance between the
// core matrices of one row group along K, sbo = distance between row groups.
__device__ __forceinline__ uint64_t smem_desc_plain(uint32_t addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo_bytes >> 4) << 16) | ((uint64_t)(sbo_bytes >> 4) << 32) |
           (1ull << 46);
}

// The descriptor of the same layout `bytes` further on in shared memory (a multiple of 16; the address field counts
// 16-byte units and shared memory ends below 2^18, so only the low word changes): one add where building a
// descriptor anew costs several instructions of the one thread that issues all tensor-core work.
__device__ __forceinline__ uint64_t desc_advance(uint64_t desc, uint32_t bytes) {
    return (desc & 0xFFFFFFFF00000000ull) | (uint32_t)((uint32_t)desc + (bytes >> 4));
}

// Instruction descriptor, kind::f16: bf16 x bf16 -> fp32, M = m, N = n, A K-major (optionally negated), B K-major
// or MN-major.
__host__ __device__ constexpr uint32_t instr_desc(bool b_mn_major, uint32_t n, bool negate_a = false, uint32_t m = 128) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((negate_a ? 1u : 0u) << 13) | ((b_mn_major ? 1u : 0u) << 16) |
           ((n >> 3) << 17) | ((m >> 4) << 24);
}

// D[tmem] (+)= A[smem] * B[smem]
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}

// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}

// Starts the load of 32 consecutive 32-bit columns of this thread's lane; the registers are valid only after
// tmem_wait_ld() (and tmem_pin(), which keeps the compiler from moving their uses above the wait).
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_pin(uint32_t* r) {     // 32 registers, no instruction
#pragma unroll
    for (int i = 0; i < 32; i += 16)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]),
                          "+r"(r[i + 6]), "+r"(r[i + 7]), "+r"(r[i + 8]), "+r"(r[i + 9]), "+r"(r[i + 10]), "+r"(r[i + 11]),
                          "+r"(r[i + 12]), "+r"(r[i + 13]), "+r"(r[i + 14]), "+r"(r[i + 15])
                     :
                     : "memory");
}

// 32 consecutive fp32 columns of this thread's lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
    uint32_t r[32];
    tmem_ld32_issue(taddr, r);
    tmem_wait_ld();
    tmem_pin(r);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
          "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
          "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}

__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// max of three (one instruction on sm_100)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// the same, NaN where one of them is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Pass 1 over one 32-key chunk of a row's raw scores s = q.k + (slope/scale)*(key index in the tile): running
// maxima.  The map to log2 units, t = s*qscale + (tile constant), is increasing, so it is applied to the maximum
// afterwards.  kMasked adds the select of the visible keys, lo < key <= pos (causal bound pos; lo = pos - window,
// or -1); tiles strictly inside that range skip it.  kNan: a score that is NaN makes its maximum NaN.
template <bool kMasked, bool kNan = false>
__device__ __forceinline__ void chunk_max(const float (&v)[32], int key0, int pos, int lo, float (&mx)[4]) {
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        float s0 = v[e], s1 = v[e + 1];
        if (kMasked) {
            s0 = (key0 + e <= pos && key0 + e > lo) ? s0 : -INFINITY;
            s1 = (key0 + e + 1 <= pos && key0 + e + 1 > lo) ? s1 : -INFINITY;
        }
        mx[(e >> 1) & 3] = kNan ? max3_nan(mx[(e >> 1) & 3], s0, s1) : max3(mx[(e >> 1) & 3], s0, s1);
    }
}

// mbar_wait with its waiting loop in one place: the kernels that work through a list of items wait at some twenty, their
// warps run all over them, and their time goes with the instruction cache's misses (the shared-prefix decode as inlined:
// 86 KB, the caches' shared port busy 74 % of the time).
inline __noinline__ __device__ bool wait_long(uint64_t* bar, uint32_t parity, int* status) { return mbar_wait(bar, parity, status); }
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, int* status) {
    return mbar_try_wait(bar, parity) || wait_long(bar, parity, status);
}

// Where the share of worker i of W begins in a list of `total`: rounded down, so that the shares follow one another.
__device__ __forceinline__ long long share_at(long long total, int i, int W) {
    return total < (1 << 22) ? (long long)((unsigned)total * (unsigned)i / (unsigned)W) : total * i / W;      // (W < 512)
}

// Two fp32 values in one 64-bit register, for the packed fp32 instructions of sm_100 (one issue slot for two lanes).
__device__ __forceinline__ uint64_t pack_f2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack_f2(uint64_t v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// Pass 2 over one chunk: p = 2^(s*qscale + bias) with the tile's ALiBi constant and the row maximum folded into
// bias; bf16 pairs for the tensor core; returns the chunk's sum of p (kRounded: of the bf16 values, so that numerator and
// denominator round alike).
template <bool kMasked, bool kRounded = false>
__device__ __forceinline__ float chunk_exp(const float (&v)[32], float qscale, float bias, int key0, int pos, int lo,
                                           uint32_t (&w)[16]) {
    if (kMasked) {
        float sm[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float t0 = fmaf(v[2 * e], qscale, bias);
            float t1 = fmaf(v[2 * e + 1], qscale, bias);
            t0 = (key0 + 2 * e <= pos && key0 + 2 * e > lo) ? t0 : -INFINITY;
            t1 = (key0 + 2 * e + 1 <= pos && key0 + 2 * e + 1 > lo) ? t1 : -INFINITY;
            const float p0 = ex2(t0), p1 = ex2(t1);
            w[e] = pack2(p0, p1);
            const float2 sum = kRounded ? bf16x2_to_float2(w[e]) : make_float2(p0, p1);
            sm[e & 3] += sum.x + sum.y;
        }
        return (sm[0] + sm[1]) + (sm[2] + sm[3]);
    }
    const uint64_t qs2 = pack_f2(qscale, qscale), b2 = pack_f2(bias, bias);
    uint64_t sm2[2] = {pack_f2(0.f, 0.f), pack_f2(0.f, 0.f)};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint64_t t2 = fma2(pack_f2(v[2 * e], v[2 * e + 1]), qs2, b2);
        float t0, t1;
        unpack_f2(t2, t0, t1);
        const float p0 = ex2(t0), p1 = ex2(t1);
        w[e] = pack2(p0, p1);
        const float2 sum = kRounded ? bf16x2_to_float2(w[e]) : make_float2(p0, p1);
        sm2[e & 1] = add2(sm2[e & 1], pack_f2(sum.x, sum.y));
    }
    float s0, s1;
    unpack_f2(add2(sm2[0], sm2[1]), s0, s1);
    return s0 + s1;
}

}  // namespace optgqa
