// Rows of a residual block in registers: what the norms' forward and backward kernels share.
//
// A row belongs to a team of 8, 16 or 32 lanes of a warp, of two or four warps, or of all warps of a CTA, whose threads hold packs of eight elements of it.
#pragma once

#include "kge_eight.cuh"

namespace kge {

enum { NORM_PLAIN = 0, NORM_SIGMOID = 1, NORM_SILU = 2 };
constexpr int NORM_THREADS = 256;              // of a CTA of several teams
constexpr int NORM_MOST = 8192;                // widest row that a CTA's threads hold
constexpr int NORM_LOOP_THREADS = 1024;        // of a CTA that goes over wider rows again and again

// Threads of the team that holds a row of d columns; 0: a CTA's.
inline int norm_team(int d) {
    for (int lanes = 8; lanes <= 128; lanes *= 2)
        if (d <= 8 * lanes) return lanes;
    return 0;
}

#ifdef __CUDACC__
// Eight fp32 numbers as four pairs: an instruction adds or multiplies two, which leaves the issue slots to the conversions.
struct P8 { uint64_t v[4]; };
template <class F> __device__ __forceinline__ P8 make_pairs(F&& f) { P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = pair(f(2 * i), f(2 * i + 1));
    return r; }
__device__ __forceinline__ float element(const P8& a, int e) { const float2 f = unpair(a.v[e >> 1]); return e & 1 ? f.y : f.x; }
__device__ __forceinline__ P8 all8(float x) { const uint64_t p = pair(x, x); return P8{{p, p, p, p}}; }
__device__ __forceinline__ P8 operator*(const P8& a, const P8& b) { P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = mul2(a.v[i], b.v[i]);
    return r; }
__device__ __forceinline__ P8 operator+(const P8& a, const P8& b) { P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = add2(a.v[i], b.v[i]);
    return r; }
__device__ __forceinline__ P8 operator*(const P8& a, float b) { return a * all8(b); }
__device__ __forceinline__ P8 operator+(const P8& a, float b) { return a + all8(b); }
__device__ __forceinline__ P8 fma8(const P8& a, const P8& b, const P8& c) { P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = fma2(a.v[i], b.v[i], c.v[i]);
    return r; }
__device__ __forceinline__ P8 fma8(const P8& a, float b, const P8& c) { return fma8(a, all8(b), c); }
template <typename T> __device__ __forceinline__ P8 pairs_of(const Raw8<T>& r) {
    const F8 x = wide_of(r);
    return make_pairs([&](int e) { return x.v[e]; });
}
__device__ __forceinline__ F8 singles_of(const P8& a) { return make8([&](int e) { return element(a, e); }); }

// Where a thread's elements lie in its row, W neighbours moving as one access: all eight of them (and all or none are there), pairs, or each alone.  What lies beyond
// the row's end is zero when loaded (with W = 8: other elements of the row) and is left out of stores and sums.
template <int W> struct Place {
    static constexpr bool WIDE = W == 8;
    int first, step, d;
    bool any;
    Place() = default;
    __device__ __forceinline__ Place(int team, int t, int k, int width) : first(WIDE ? (k * team + t) * 8 : k * team * 8 + t * W), step(W * team), d(width), any(first < width) {
        if (WIDE && !any) first = 0;
    }
    __device__ __forceinline__ int at(int e) const { return first + e / W * step + e % W; }
    __device__ __forceinline__ bool holds(int e) const { return WIDE ? any : at(e / W * W) < d; }
    // (a row's address is the same for a warp, and a thread's place in it takes 32 bits: one access, no arithmetic of 64 bits in every thread)
    template <typename T> __device__ __forceinline__ T* mine(T* row, int e = 0) const {
        using Byte = typename std::conditional<std::is_const<T>::value, const char, char>::type;
        return reinterpret_cast<T*>(reinterpret_cast<Byte*>(row) + (uint32_t)at(e) * (uint32_t)sizeof(T));
    }
    template <typename T> __device__ __forceinline__ Raw8<T> load(const T* row) const {
        if constexpr (WIDE) return load_wide(mine(row));
        Raw8<T> r;
        if constexpr (W == 2) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                if constexpr (sizeof(T) == 4) {
                    const uint2 w = holds(e) ? *reinterpret_cast<const uint2*>(mine(row, e)) : make_uint2(0u, 0u);
                    r.w[e] = w.x; r.w[e + 1] = w.y;
                } else r.w[e / 2] = holds(e) ? *reinterpret_cast<const uint32_t*>(mine(row, e)) : 0u;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) set_element(r, e, holds(e) ? *mine(row, e) : from_float<T>(0.f));
        }
        return r;
    }
    template <typename T> __device__ __forceinline__ void store(T* row, const P8& x, bool live) const {
        const Raw8<T> r = narrow_of<T>(singles_of(x));
        if constexpr (WIDE) { if (any && live) store_wide(mine(row), r); }
        else if constexpr (W == 2) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                if (!holds(e) || !live) continue;
                if constexpr (sizeof(T) == 4) *reinterpret_cast<uint2*>(mine(row, e)) = make_uint2(r.w[e], r.w[e + 1]);
                else *reinterpret_cast<uint32_t*>(mine(row, e)) = r.w[e / 2];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (holds(e) && live) *mine(row, e) = element(r, e);
        }
    }
    // A vector of parameters.  (Loaded here, from the L1 cache: the compiler would keep all of them in registers, and spill others.)
    __device__ __forceinline__ P8 vector(const float* p) const {
        if constexpr (WIDE) {
            const Pack<float, 8> v = load_now<Pack<float, 8>>(mine(p));
            return make_pairs([&](int e) { return v.v[e]; });
        } else if constexpr (W == 2) {
            P8 r;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r.v[i] = 0;
                if (!holds(2 * i)) continue;
                const Pack<float, 2> v = load_now<Pack<float, 2>>(mine(p, 2 * i));
                r.v[i] = pair(v.v[0], v.v[1]);
            }
            return r;
        }
        return make_pairs([&](int e) { return holds(e) ? load_now<Pack<float, 1>>(mine(p, e)).v[0] : 0.f; });
    }
    // Zero beyond the row's end (W < 8).
    __device__ __forceinline__ P8 there(const P8& a) const { return WIDE ? a : make_pairs([&](int e) { return holds(e) ? element(a, e) : 0.f; }); }
    // Sums over the thread's elements; with W < 8 one factor is zero beyond the row's end.
    __device__ __forceinline__ float total(const P8& a) const {
        const float2 s = unpair(add2(add2(a.v[0], a.v[1]), add2(a.v[2], a.v[3])));
        return WIDE && !any ? 0.f : s.x + s.y;
    }
    __device__ __forceinline__ float dot(const P8& a, const P8& b) const {
        uint64_t s = mul2(a.v[0], b.v[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) s = fma2(a.v[i], b.v[i], s);
        const float2 f = unpair(s);
        return WIDE && !any ? 0.f : f.x + f.y;
    }
};

// Sums (or the largest) over a team of L threads, or of the CTA's (L = 0).  Teams of several warps take turns with two sets of places in shared memory, so
// that one barrier (the team's own) a sum is enough.
template <int L> struct Team {
    static constexpr int COUNT = L == 0 ? 1 : NORM_THREADS / (L == 0 ? 1 : L);        // teams of a CTA
    float (*parts)[2][32];
    const int thread, index;           // within the team; the team's in its CTA
    int turn = 0;
    static __device__ __forceinline__ int size() { return L == 0 ? (int)blockDim.x : L; }
    // (made by all threads of a CTA: the index is told to be the same for a warp, so that addresses of rows are made once for it)
    explicit __device__ __forceinline__ Team(float (*p)[2][32])
        : parts(p), thread(L == 0 ? (int)threadIdx.x : (int)threadIdx.x % (L == 0 ? 1 : L)), index(index_of()) {}
    static __device__ __forceinline__ int index_of() {
        if (L == 0) return 0;
        const int i = (int)threadIdx.x / (L == 0 ? 1 : L);
        return L >= 32 ? __shfl_sync(0xffffffffu, i, 0) : i;
    }
    // (the largest of magnitudes as integers, which order as they do, a NaN above all)
    template <bool MOST> static __device__ __forceinline__ float join(float a, float b) {
        return MOST ? __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))) : a + b;
    }
    template <bool MOST, int N> __device__ __forceinline__ void all(float (&v)[N]) {
        constexpr int LANES = L == 0 || L > 32 ? 32 : L;
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = join<MOST>(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
        }
        if constexpr (L == 0 || L > 32) {
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) parts[turn][i][warp] = v[i];
            }
            if constexpr (L == 0) {
                __syncthreads();
                const int warps = (int)blockDim.x >> 5;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    v[i] = lane < warps ? parts[turn][i][lane] : 0.f;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) v[i] = join<MOST>(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
                }
            } else {
                constexpr int WARPS = L / 32;
                asm volatile("bar.sync %0, %1;" ::"r"(1 + index), "n"(L) : "memory");
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float* at = parts[turn][i] + index * WARPS;
                    float x = at[0];
#pragma unroll
                    for (int w = 1; w < WARPS; ++w) x = join<MOST>(x, at[w]);
                    v[i] = x;
                }
            }
            turn ^= 1;
        }
    }
    __device__ __forceinline__ float sum(float x) { float v[1] = {x}; all<false>(v); return v[0]; }
    __device__ __forceinline__ void sum(float& x, float& y) { float v[2] = {x, y}; all<false>(v); x = v[0]; y = v[1]; }
    __device__ __forceinline__ float most(float x) { float v[1] = {x}; all<true>(v); return v[0]; }
};

// 1 / (1 + exp(-g)) within 8 units of 2^-24 of itself, and 2^-147.  Where |g| < 80 (neither the power nor its reciprocal leaves the normal numbers there) both are one
// instruction each: t = -g log2 e is rounded, so 2^t is off by exp(r) with r = -g - t ln 2, some 2^-17 at most; ln 2 in two parts gives r (Cody and Waite), and
// 2^t (1 + r) is off by the instruction's 4 units and one more.  (Without it gates far below zero were off by 1.5 |g| units.)
constexpr float LOG2_E = 1.44269504f, LN_2 = 0.693147182f, LN_2_REST = -1.90465430e-9f;
__device__ __forceinline__ float power_of_two(float t) { float x; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(t)); return x; }
__device__ __forceinline__ float one_over(float y) { float x; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(y)); return x; }
// (A call, rare in the kernels that hold a row and cheap beside the loops' loads: inline it takes registers from both, the fp32 gradients of 3,000 x 20,000 2,095 us, so 2,320.)
static __device__ __noinline__ float sigmoid_of(float g) {
    if (fabsf(g) < 80.f) {
        const float t = g * -LOG2_E, r = fmaf(t, -LN_2_REST, fmaf(t, -LN_2, -g)), power = power_of_two(t);
        return one_over(fmaf(power, r, power) + 1.f);
    }
    const float e = expf(-fabsf(g)), r = __fdiv_rn(1.f, 1.f + e);
    return g < 0.f ? e * r : r;
}
__device__ __forceinline__ float sigmoid_brief(float g) { return one_over(1.f + power_of_two(-LOG2_E * g)); }
// The same bits for a thread's gates: f(k, sigmoids of pack k), in pairs where all of them are near.
// BRIEF: without the remainder, and 0 below the normal numbers: within 6 + 1.5 |g| units of 2^-24 of itself (its share of |g| for g < 0 only), less than 2^-16.  Enough where
// all that is made of it is rounded to 16 bits (h and z of 16-bit rows and blocks; 32,768 x 4,096 bf16: 245 us, 255 with the remainder).
__device__ __forceinline__ float most_of(float a, float b, float c) { float m; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c)); return m; }
template <bool BRIEF, int K, typename T, class F> __device__ __forceinline__ void with_sigmoids(const Raw8<T> (&gate)[K], F&& f) {
    if constexpr (BRIEF) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const P8 g = pairs_of(gate[k]);
            f(k, make_pairs([&](int e) { return sigmoid_brief(element(g, e)); }));
        }
        return;
    }
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const F8 g = wide_of(gate[k]);
#pragma unroll
        for (int e = 0; e < 8; e += 2) most = most_of(most, fabsf(g.v[e]), fabsf(g.v[e + 1]));
    }
    if (!(most < 80.f)) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const F8 g = wide_of(gate[k]);
            f(k, make_pairs([&](int e) { return sigmoid_of(g.v[e]); }));
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const P8 g = pairs_of(gate[k]), t = g * -LOG2_E, r = fma8(t, -LN_2_REST, fma8(t, -LN_2, g * -1.f)), power = make_pairs([&](int e) { return power_of_two(element(t, e)); });
        const P8 sum = fma8(power, r, power) + 1.f;
        f(k, make_pairs([&](int e) { return one_over(element(sum, e)); }));
    }
}
template <bool BRIEF> __device__ __forceinline__ float act_of(float g, int act) {
    if (act == NORM_PLAIN) return g;
    const float s = BRIEF ? sigmoid_brief(g) : sigmoid_of(g);
    return act == NORM_SIGMOID ? s : g * s;
}
__device__ __forceinline__ float2 act_and_slope(float g, int act) {
    if (act == NORM_PLAIN) return make_float2(g, 1.f);
    const float s = sigmoid_of(g);
    return act == NORM_SIGMOID ? make_float2(s, s * (1.f - s)) : make_float2(g * s, s * (1.f + g * (1.f - s)));
}
#endif

}  // namespace kge
