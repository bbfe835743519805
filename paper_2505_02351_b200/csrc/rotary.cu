// Rotary positions: the first R dims of every query and key head are rotated in pairs by angles that grow with the
// token's position, y = amplitude * R(pos * f_i) x, and -- in the append form -- the rotated keys and the values are
// written to their slots of the paged cache on the way (Algorithm 1, "Reshape and store K, V into C_K, C_V", for
// models whose positions are rotary instead of ALiBi).
//
// Angles.  The caller hands over f_i as a fraction of a turn in 64-bit fixed point, F_i = f_i / 2pi * 2^64 mod 2^64,
// so that pos * F_i mod 2^64 -- one wrapping integer product -- is the angle reduced to a turn, exactly, at any
// position: no 64-bit floating point, no argument reduction, no table over positions.  Its upper 32 bits go through
// one conversion (off by at most 2^-25 of half a turn, 9e-8 rad) and sincospi; cos, sin and the products are fp32,
// the result is rounded once when stored.
//
// Bound by memory: every element is read once and written once, about one flop per byte.  A CTA takes kTokens tokens;
// their cos/sin pairs are computed once into shared memory (before the wait for the preceding kernel) and used by all
// heads: computed per head they would cost as much as the copy itself (30 instructions against 6 per pair).
// A unit of work is P pairs of one row, two 16-byte vectors: vectors P u and R/2 + P u of the half layout, two
// adjacent ones of the interleaved layout and of the dims past R, which pass through unchanged.  A thread requests
// kBatch units before it uses the first; registers are held to five CTAs per multiprocessor (80 KB in flight; four
// units per thread at two CTAs took 40 us where this takes 29).  It asks for R / 2 to be whole vectors; for any other R
// the rows go through shared memory, where a pair's elements are read one by one (rotary_staged_kernel).
#include <math.h>

#include "common.cuh"

namespace optgqa {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotCtas = 5;            // resident CTAs per multiprocessor the registers are held to

struct RotaryParams {
    const void* q;
    const void* k;
    const void* v;                     // null: no values (the rotation alone)
    void* q_out;
    void* k_out;                       // may be null when there is a cache
    void* k_cache;                     // null: no cache
    void* v_cache;
    const int64_t* slots;
    const int32_t* positions;
    const uint64_t* freq;
    long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;   // elements from token to token
    long long num_slots;
    int T, Hq, Hk, Hv, R, bs_log2;
    float cos_amp, sin_amp;            // amplitude, and with the direction's sign
};

// P adjacent elements, 16 bytes, as fp32.
template <typename T, int P>
struct Chunk {
    uint4 raw;
    __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = raw; }
    __device__ __forceinline__ void get(float (&f)[P]) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2) {
                const float2 v = bf16x2_to_float2(w[i]);
                f[2 * i] = v.x;
                f[2 * i + 1] = v.y;
            } else {
                f[i] = __uint_as_float(w[i]);
            }
        }
    }
    __device__ __forceinline__ void set(const float (&f)[P]) {
        if constexpr (sizeof(T) == 2)
            raw = make_uint4(float2_to_bf16x2(f[0], f[1]), float2_to_bf16x2(f[2], f[3]), float2_to_bf16x2(f[4], f[5]),
                             float2_to_bf16x2(f[6], f[7]));
        else
            raw = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
// cos and sin of the pairs of `tokens` tokens from t0 on, [tokens][D / 2], by all threads of the CTA.
template <int D>
__device__ __forceinline__ void angles(const RotaryParams& p, long long t0, int tokens, float* s_cos, float* s_sin) {
    const int half = p.R / 2;
    for (int i = threadIdx.x; i < tokens * half; i += kRotThreads) {
        const int tok = i / half, pair = i - tok * half;
        const uint64_t turn = (uint64_t)(int64_t)__ldg(p.positions + t0 + tok) * __ldg(p.freq + pair);
        float s, c;
        sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &s, &c);     // half turns, in [-1, 1]
        s_cos[tok * (D / 2) + pair] = c * p.cos_amp;
        s_sin[tok * (D / 2) + pair] = s * p.sin_amp;
    }
}

// Row h of token t (queries, then keys, then values).
template <typename T, int D>
__device__ __forceinline__ const T* source_row(const RotaryParams& p, long long t, int h) {
    return h < p.Hq          ? static_cast<const T*>(p.q) + t * p.q_stride + (long long)h * D
           : h < p.Hq + p.Hk ? static_cast<const T*>(p.k) + t * p.k_stride + (long long)(h - p.Hq) * D
                             : static_cast<const T*>(p.v) + t * p.v_stride + (long long)(h - p.Hq - p.Hk) * D;
}

// Calls store(destination row) for every place row h of token t goes to.
template <typename T, int D, typename Store>
__device__ __forceinline__ void for_destinations(const RotaryParams& p, long long t, int h, Store store) {
    if (h < p.Hq) {
        store(static_cast<T*>(p.q_out) + t * p.q_out_stride + (long long)h * D);
        return;
    }
    const bool is_v = h >= p.Hq + p.Hk;
    const int kh = is_v ? h - p.Hq - p.Hk : h - p.Hq;
    if (!is_v && p.k_out) store(static_cast<T*>(p.k_out) + t * p.k_out_stride + (long long)kh * D);
    if (p.k_cache) {
        const long long slot = p.slots[t];
        if (slot >= 0 && slot < p.num_slots) {
            const long long page = slot >> p.bs_log2, off = slot & ((1 << p.bs_log2) - 1);
            store(static_cast<T*>(is_v ? p.v_cache : p.k_cache) + (((page * p.Hk + kh) << p.bs_log2) + off) * D);
        }
    }
}

template <typename T, int D, int P, bool kInterleaved, int kTokens, int kBatch>
__global__ void __launch_bounds__(kRotThreads, kRotCtas)
rotary_kernel(const RotaryParams p) {
    constexpr int U = D / (2 * P);                    // units per row
    __shared__ __align__(16) float s_cos[kTokens][D / 2], s_sin[kTokens][D / 2];
    grid_dependency_launch();
    const long long t0 = (long long)blockIdx.x * kTokens;
    const int tokens = (int)min((long long)kTokens, p.T - t0), half = p.R / 2;
    angles<D>(p, t0, tokens, &s_cos[0][0], &s_sin[0][0]);
    __syncthreads();
    grid_dependency_wait();     // q, k, v may come from the preceding kernel, which may also still read what is written here

    const int H = p.Hq + p.Hk + p.Hv, units = tokens * H * U;
    const int step = kRotThreads * gridDim.y;         // the CTAs of one token in y take its units in turns
    for (int base = threadIdx.x + kRotThreads * blockIdx.y; base < units; base += kBatch * step) {
        Chunk<T, P> a[kBatch], b[kBatch];
        // element offsets of a unit's two halves inside its row
        auto offsets = [&](int u, int& e0, int& e1) {
            const bool split = !kInterleaved && P * u < half;
            e0 = split ? P * u : 2 * P * u;
            e1 = split ? half + P * u : 2 * P * u + P;
        };
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
            const int i = base + n * step;
            if (i < units) {
                const int row = i / U, tok = row / H, h = row - tok * H;
                const long long t = t0 + tok;
                int e0, e1;
                offsets(i % U, e0, e1);
                const T* src = source_row<T, D>(p, t, h);
                a[n].load(src + e0);
                b[n].load(src + e1);
            }
        }
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
            const int i = base + n * step;
            if (i < units) {
                const int u = i % U, row = i / U, tok = row / H, h = row - tok * H;
                const long long t = t0 + tok;
                int e0, e1;
                offsets(u, e0, e1);
                if (h < p.Hq + p.Hk && P * u < half) {
                    const float* cs = &s_cos[tok][P * u];
                    const float* sn = &s_sin[tok][P * u];
                    float x[P], y[P];
                    a[n].get(x);
                    b[n].get(y);
                    if constexpr (kInterleaved) {
                        // the P pairs are (2i, 2i + 1) of the 2 P adjacent elements x, y
#pragma unroll
                        for (int e = 0; e < P / 2; ++e) {
                            const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
                            x[2 * e] = x0 * cs[e] - x1 * sn[e];
                            x[2 * e + 1] = x1 * cs[e] + x0 * sn[e];
                            y[2 * e] = y0 * cs[P / 2 + e] - y1 * sn[P / 2 + e];
                            y[2 * e + 1] = y1 * cs[P / 2 + e] + y0 * sn[P / 2 + e];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < P; ++e) {
                            const float x0 = x[e], y0 = y[e];
                            x[e] = x0 * cs[e] - y0 * sn[e];
                            y[e] = y0 * cs[e] + x0 * sn[e];
                        }
                    }
                    a[n].set(x);
                    b[n].set(y);
                }
                for_destinations<T, D>(p, t, h, [&](T* dst) {
                    a[n].store(dst + e0);
                    b[n].store(dst + e1);
                });
            }
        }
    }
}

// Any even R: a warp brings kBatch times 512 bytes of rows into shared memory, 16 bytes a lane, its lanes rotate pair by pair
// there, and the rows leave as they came; the next ones are requested before.  8192 tokens of 40 heads of 128, bf16, R 126:
// 47.6 us of a floor of 26.0 (R 50: 40.2); bound by the two-byte passes through shared memory.  One row at a time 57.7, four 47.4
// (R 50: 40.5, 64 wide 34.8 where two take 31.4); one pair per thread straight from memory 101.
template <typename T, int D, bool kInterleaved, int kTokens, int kBatch>
__global__ void __launch_bounds__(kRotThreads)
rotary_staged_kernel(const RotaryParams p) {
    constexpr int kVec = 16 / sizeof(T), kLanes = D / kVec, kRowsPer = 32 / kLanes, kWarps = kRotThreads / 32;
    __shared__ float s_cos[kTokens * D / 2], s_sin[kTokens * D / 2];
    __shared__ __align__(16) T s_rows[kWarps][kBatch * kRowsPer * D];
    grid_dependency_launch();
    const long long t0 = (long long)blockIdx.x * kTokens;
    const int tokens = (int)min((long long)kTokens, p.T - t0), half = p.R / 2;
    angles<D>(p, t0, tokens, s_cos, s_sin);
    __syncthreads();
    grid_dependency_wait();

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int H = p.Hq + p.Hk + p.Hv, rows = tokens * H, mine = lane / kLanes, e = lane % kLanes * kVec;
    const int step = kWarps * kBatch * kRowsPer * gridDim.y;        // rows all warps take at a time
    T* stage = s_rows[warp];
    uint4 next[kBatch];
    auto fetch = [&](int first) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int row = first + u * kRowsPer + mine;
            if (row < rows) next[u] = *reinterpret_cast<const uint4*>(source_row<T, D>(p, t0 + row / H, row % H) + e);
        }
    };
    int first = (blockIdx.y * kWarps + warp) * kBatch * kRowsPer;
    fetch(first);
    for (; first < rows; first += step) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) *reinterpret_cast<uint4*>(stage + (u * kRowsPer + mine) * D + e) = next[u];
        __syncwarp();
        fetch(first + step);
#pragma unroll
        for (int r = 0; r < kBatch * kRowsPer; ++r) {
            const int row = first + r, tok = row / H;
            if (row >= rows || row - tok * H >= p.Hq + p.Hk) continue;     // values are not rotated
            const float *cs = s_cos + tok * (D / 2), *sn = s_sin + tok * (D / 2);
            for (int i = lane; i < half; i += 32) {
                T *a = stage + r * D + (kInterleaved ? 2 * i : i), *b = kInterleaved ? a + 1 : a + half;
                const float x = static_cast<float>(*a), y = static_cast<float>(*b);
                *a = static_cast<T>(x * cs[i] - y * sn[i]);
                *b = static_cast<T>(y * cs[i] + x * sn[i]);
            }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int row = first + u * kRowsPer + mine;
            if (row < rows) {
                const uint4 out = *reinterpret_cast<const uint4*>(stage + (u * kRowsPer + mine) * D + e);
                for_destinations<T, D>(p, t0 + row / H, row % H, [&](T* dst) { *reinterpret_cast<uint4*>(dst + e) = out; });
            }
        }
        __syncwarp();
    }
}

template <typename T, int D, bool kInterleaved>
int launch_staged(const RotaryParams& p, cudaStream_t stream) {
    constexpr int kStep = kRotThreads * 16 / (D * (int)sizeof(T));        // rows a CTA takes at a time
    // as in launch_tokens: several CTAs per token of a few, four tokens per CTA of many (us with four against one, bf16 of 128,
    // R 50, 24 / 40 / 80 heads: 2048 tokens 11.6 18.3 34.8 against 9.7 14.7 22.1, 4096 15.5 22.3 41.5 against 17.5 25.8 41.4)
    const int rounds = (p.Hq + p.Hk + p.Hv + kStep - 1) / kStep;
    auto launch = [&](auto kernel, long long x, int y) {
        return launch_dependent(kernel, dim3((unsigned)x, (unsigned)y), dim3(kRotThreads), 0, stream, p);
    };
    if (p.T <= 512) return launch(rotary_staged_kernel<T, D, kInterleaved, 1, 1>, p.T, rounds);
    if (p.T >= 4096) return launch(rotary_staged_kernel<T, D, kInterleaved, 4, 2>, (p.T + 3ll) / 4, 1);
    return launch(rotary_staged_kernel<T, D, kInterleaved, 1, 2>, p.T, 1);
}

template <typename T, int D, int P, bool kInterleaved>
int launch_tokens(const RotaryParams& p, cudaStream_t stream) {
    constexpr int U = D / (2 * P);
    const int units = (p.Hq + p.Hk + p.Hv) * U;
    auto launch = [&](auto kernel, long long x, int y) {
        return launch_dependent(kernel, dim3((unsigned)x, (unsigned)y), dim3(kRotThreads), 0, stream, p);
    };
    // Few tokens (a decode batch): latency counts, every thread takes one unit and a token as many CTAs as that needs
    // (256 tokens of 80 heads, bf16: 3.2 us against 3.8 with two units per thread).
    if (p.T <= 512)
        return launch(rotary_kernel<T, D, P, kInterleaved, 1, 1>, p.T, (units + kRotThreads - 1) / kRotThreads);
    // Many tokens whose rows do not fill a CTA's two units per thread: four per CTA (8192 tokens of 40 heads, bf16: 28.7
    // us against 35 to 40 with one); but not where one token fills it (4095 tokens of 72 heads, fp32: 47 us against 63 with
    // four).  Below, few CTAs per multiprocessor are left of a quarter of the tokens (1024 of 24 heads of 128, bf16: 5.0 us
    // with four against 3.7, of 40: 8.0 against 5.5; 1999 of 24 of 64, fp32: 6.4 against 5.6).  The two cross near 2048 tokens
    // already (us with four against one, bf16, 2048 / 3000 / 4095 tokens: 24 heads of 128 6.6 9.5 11.2 against 7.4 10.8 14.3;
    // 40 of 128 9.8 14.1 16.4 against 10.3 14.4 18.8; 40 of 64 5.7 8.7 10.2 against 6.1 9.9 12.9).
    if (p.T >= 4096 && units <= 2 * kRotThreads)
        return launch(rotary_kernel<T, D, P, kInterleaved, 4, 2>, (p.T + 3ll) / 4, 1);
    return launch(rotary_kernel<T, D, P, kInterleaved, 1, 2>, p.T, 1);
}

template <typename T, int D>
int launch_typed(const RotaryParams& p, int layout, cudaStream_t stream) {
    constexpr int kVec = 16 / sizeof(T);
    // whole vectors on both sides of every pair: R / 2 elements are whole 16-byte vectors
    const bool wide = p.R % (2 * kVec) == 0;
    if (layout == OPT_GQA_ROTARY_INTERLEAVED)
        return wide ? launch_tokens<T, D, kVec, true>(p, stream) : launch_staged<T, D, true>(p, stream);
    return wide ? launch_tokens<T, D, kVec, false>(p, stream) : launch_staged<T, D, false>(p, stream);
}

}  // namespace

int launch_rotary(const RotaryArgs& a, cudaStream_t stream) {
    RotaryParams p;
    p.q = a.q;
    p.k = a.k;
    p.v = a.v;
    p.q_out = a.q_out;
    p.k_out = a.k_out;
    p.k_cache = a.k_cache;
    p.v_cache = a.v_cache;
    p.slots = a.slots;
    p.positions = a.positions;
    p.freq = a.freq;
    p.q_stride = a.q_stride;
    p.k_stride = a.k_stride;
    p.v_stride = a.v_stride;
    p.q_out_stride = a.q_out_stride;
    p.k_out_stride = a.k_out_stride;
    p.num_slots = a.num_blocks * a.bs;
    p.T = a.T;
    p.Hq = a.Hq;
    p.Hk = a.Hkv;
    p.Hv = a.v ? a.Hkv : 0;
    p.R = a.rot_dim;
    p.bs_log2 = a.bs == 32 ? 5 : 4;
    p.cos_amp = a.amplitude;
    p.sin_amp = a.inverse ? -a.amplitude : a.amplitude;
    if (a.dtype == OPT_GQA_BF16)
        return a.D == 128 ? launch_typed<__nv_bfloat16, 128>(p, a.layout, stream) : launch_typed<__nv_bfloat16, 64>(p, a.layout, stream);
    return a.D == 128 ? launch_typed<float, 128>(p, a.layout, stream) : launch_typed<float, 64>(p, a.layout, stream);
}

// ----------------------------------------------------------------------------- host arithmetic
// Radians per position of pair i, i < R / 2, in 64 bits.
int rotary_frequencies(double* f, int R, double base, int scaling, double factor, double original_len, double low_turns,
                       double high_turns) {
    constexpr double kTwoPi = 6.283185307179586476925;
    for (int i = 0; i < R / 2; ++i) {
        const double plain = pow(base, -2.0 * i / R);
        switch (scaling) {
            case OPT_GQA_ROTARY_NONE: f[i] = plain; break;
            case OPT_GQA_ROTARY_LINEAR: f[i] = plain / factor; break;
            case OPT_GQA_ROTARY_NTK: f[i] = pow(base * pow(factor, (double)R / (R - 2)), -2.0 * i / R); break;
            case OPT_GQA_ROTARY_PARTS: {
                const double turns = original_len * plain / kTwoPi;
                const double w = fmin(fmax((turns - low_turns) / (high_turns - low_turns), 0.0), 1.0);
                f[i] = plain * (w + (1.0 - w) / factor);
                break;
            }
            case OPT_GQA_ROTARY_RAMP: {
                // the (real) pair index at which a dimension makes `turns` turns over the original context
                const double lo_at = R * log(original_len / (kTwoPi * high_turns)) / (2.0 * log(base));
                const double hi_at = R * log(original_len / (kTwoPi * low_turns)) / (2.0 * log(base));
                const double lo = fmax(floor(lo_at), 0.0), hi = fmin(ceil(hi_at), R - 1.0);
                const double w = 1.0 - fmin(fmax((i - lo) / fmax(hi - lo, 0.001), 0.0), 1.0);
                f[i] = plain * (w + (1.0 - w) / factor);
                break;
            }
            default: return OPT_GQA_ERR_SHAPE;
        }
        if (!isfinite(f[i])) return OPT_GQA_ERR_SHAPE;
    }
    return OPT_GQA_OK;
}

// f radians per position -> the fraction of a turn in 64-bit fixed point (whole turns per position drop out: positions
// are whole numbers).
uint64_t rotary_turns(double f) {
    constexpr double kTwoPi = 6.283185307179586476925;
    const double turns = f / kTwoPi, frac = turns - floor(turns);      // [0, 1]
    const double hi = floor(ldexp(frac, 32));                          // two exact halves of the 64 bits
    const double lo = floor(ldexp(ldexp(frac, 32) - hi, 32));
    return ((uint64_t)hi << 32) + (uint64_t)lo;
}

}  // namespace optgqa
