// Rows of a residual block in registers: what the norms' forward and backward kernels share.
//
// A thread holds eight elements of a row; a row belongs to a team of 8, 16 or 32 lanes of a warp, of two or four warps, or of all warps of a CTA, the
// least that hold it.  Arithmetic is on pairs (two fp32 operations to an instruction): the kernels would be bound by their
// instructions otherwise, not by memory (32,768 x 4,096: 91 instructions an element before, a floor of 40 at the memory's pace).
#pragma once

#include <type_traits>

#include "kge_ops.cuh"

namespace kge {

enum { NORM_PLAIN = 0, NORM_SIGMOID = 1, NORM_SILU = 2 };
constexpr int NORM_THREADS = 256;              // of a CTA of several teams
constexpr int NORM_CTAS = 3;                   // of these on an SM
constexpr int NORM_MOST = 8192;                // widest row that a CTA's threads hold
constexpr int NORM_LOOP_THREADS = 1024;        // of a CTA that goes over wider rows again and again

// Threads of the team that holds a row of d columns; 0: a CTA's.
inline int norm_team(int d) {
    for (int lanes = 8; lanes <= 128; lanes *= 2)
        if (d <= 8 * lanes) return lanes;
    return 0;
}

#ifdef __CUDACC__
// Eight elements of a row in a thread: neighbours where rows allow wide accesses, the team's size apart where not.
template <typename T> struct alignas(8) Raw8 { T v[8]; };

template <typename T> __device__ __forceinline__ Raw8<T> load_wide(const T* p) {
    Raw8<T> r;
    uint32_t* w = reinterpret_cast<uint32_t*>(r.v);
    if constexpr (sizeof(T) == 4)
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    else
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    return r;
}
template <typename T> __device__ __forceinline__ void store_wide(T* p, const Raw8<T>& r) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(r.v);
    if constexpr (sizeof(T) == 4)
        asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p) : "memory");
    else
        asm volatile("st.global.v4.b32 [%4], {%0, %1, %2, %3};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "l"(p) : "memory");
}

// Eight fp32 numbers as four pairs.
struct F8 {
    uint64_t v[4];
    __device__ __forceinline__ float get(int e) const { const float2 f = unpair(v[e >> 1]); return e & 1 ? f.y : f.x; }
};
__device__ __forceinline__ F8 all8(float x) { const uint64_t p = pair(x, x); return F8{{p, p, p, p}}; }
__device__ __forceinline__ F8 operator*(const F8& a, const F8& b) { F8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = mul2(a.v[i], b.v[i]);
    return r; }
__device__ __forceinline__ F8 operator+(const F8& a, const F8& b) { F8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = add2(a.v[i], b.v[i]);
    return r; }
__device__ __forceinline__ F8 operator*(const F8& a, float b) { return a * all8(b); }
__device__ __forceinline__ F8 operator+(const F8& a, float b) { return a + all8(b); }
__device__ __forceinline__ F8 fma8(const F8& a, const F8& b, const F8& c) { F8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = fma2(a.v[i], b.v[i], c.v[i]);
    return r; }
__device__ __forceinline__ F8 fma8(const F8& a, float b, const F8& c) { return fma8(a, all8(b), c); }
__device__ __forceinline__ float total(const F8& a) { const float2 f = unpair(add2(add2(a.v[0], a.v[1]), add2(a.v[2], a.v[3]))); return f.x + f.y; }
__device__ __forceinline__ float dot(const F8& a, const F8& b) {
    uint64_t s = mul2(a.v[0], b.v[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) s = fma2(a.v[i], b.v[i], s);
    const float2 f = unpair(s);
    return f.x + f.y;
}
template <class F> __device__ __forceinline__ F8 each8(const F8& a, F&& f) { F8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 x = unpair(a.v[i]); r.v[i] = pair(f(x.x), f(x.y)); }
    return r; }

__device__ __forceinline__ F8 wide_of(const Raw8<float>& r) { F8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = pair(r.v[2 * i], r.v[2 * i + 1]);
    return x; }
__device__ __forceinline__ F8 wide_of(const Raw8<__nv_bfloat16>& r) { F8 x;
    const uint32_t* w = reinterpret_cast<const uint32_t*>(r.v);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    return x; }
__device__ __forceinline__ F8 wide_of(const Raw8<__half>& r) { F8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(r.v + 2 * i)); x.v[i] = pair(f.x, f.y); }
    return x; }
template <typename T> __device__ __forceinline__ Raw8<T> narrow_of(const F8& x) { Raw8<T> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpair(x.v[i]);
        if constexpr (std::is_same<T, float>::value) { r.v[2 * i] = f.x; r.v[2 * i + 1] = f.y; }
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) *reinterpret_cast<__nv_bfloat162*>(r.v + 2 * i) = __floats2bfloat162_rn(f.x, f.y);
        else *reinterpret_cast<__half2*>(r.v + 2 * i) = __floats2half2_rn(f.x, f.y);
    }
    return r; }

// Where a thread's elements lie in its row: WIDE rows let eight neighbours move as one access, and all of them or none are there.
template <bool WIDE> struct Place {
    int first, step, d;
    __device__ __forceinline__ Place(int team, int t, int width) : first(WIDE ? t * 8 : t), step(WIDE ? 1 : team), d(width) {}
    __device__ __forceinline__ int at(int e) const { return first + e * step; }
    __device__ __forceinline__ bool holds(int e) const { return WIDE ? first < d : at(e) < d; }
    __device__ __forceinline__ bool any() const { return first < d; }
    template <typename T> __device__ __forceinline__ Raw8<T> load(const T* row, bool there = true) const {
        Raw8<T> r = {};
        if constexpr (WIDE) { if (there && any()) r = load_wide(row + first); }
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (there && holds(e)) r.v[e] = row[at(e)];
        }
        return r;
    }
    template <typename T> __device__ __forceinline__ void store(T* row, const F8& x) const {
        const Raw8<T> r = narrow_of<T>(x);
        if constexpr (WIDE) { if (any()) store_wide(row + first, r); }
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (holds(e)) row[at(e)] = r.v[e];
        }
    }
    // A vector of parameters, zeros beyond the row.  (Loaded here, from the L1 cache: the compiler would keep all of them in registers, and spill others.)
    __device__ __forceinline__ F8 vector(const float* p) const {
        Raw8<float> r = {};
        if constexpr (WIDE) {
            if (any()) *reinterpret_cast<Pack<float, 8>*>(r.v) = load_now<Pack<float, 8>>(p + first);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (holds(e)) r.v[e] = __ldg(p + at(e));
        }
        return wide_of(r);
    }
    // x where the row is, zeros beyond it.
    __device__ __forceinline__ F8 spread(float x) const {
        if constexpr (WIDE) return all8(any() ? x : 0.f);
        Raw8<float> r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = holds(e) ? x : 0.f;
        return wide_of(r);
    }
};

// Sums (or the largest) over a team of L threads, or of the CTA's (L = 0).  Teams of several warps take turns with two sets of places in shared memory, so
// that one barrier (the team's own) a sum is enough.
template <int L> struct Team {
    static constexpr int COUNT = L == 0 ? 1 : NORM_THREADS / (L == 0 ? 1 : L);        // teams of a CTA
    float (*parts)[2][32];
    int turn = 0;
    static __device__ __forceinline__ int size() { return L == 0 ? (int)blockDim.x : L; }
    static __device__ __forceinline__ int thread() { return L == 0 ? (int)threadIdx.x : (int)threadIdx.x % (L == 0 ? 1 : L); }
    static __device__ __forceinline__ int index() {
        if (L == 0) return 0;
        const int i = (int)threadIdx.x / (L == 0 ? 1 : L);
        return L >= 32 ? __shfl_sync(0xffffffffu, i, 0) : i;          // (the same for a warp, so that addresses of rows are made once for it)
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
                asm volatile("bar.sync %0, %1;" ::"r"(1 + index()), "n"(L) : "memory");
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float* at = parts[turn][i] + index() * WARPS;
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

// 1 / (1 + exp(-g)).  The power of two is taken of the rounded product g log2 e, what the rounding and the constant's last bits left out joins it to first
// order: the exponential's instruction is within 3 units of 2^-24, its product with the rest, the sum and the reciprocal (2) another four.
__device__ __forceinline__ float sigmoid_of(float g) {
    constexpr float LOG2E = 1.44269502f, REST = 1.92596299e-8f;        // their sum is log2 e
    const float t = -LOG2E * g, left = fmaf(-REST, g, fmaf(-LOG2E, g, -t));
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    // (an exponent beyond the range: the quotient is 0, and inf - inf must not get into it)
    e = fabsf(t) < 126.f ? fmaf(e, 0.693147182f * left, e) : e;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}
__device__ __forceinline__ F8 act_of(const F8& g, int act) {
    if (act == NORM_PLAIN) return g;
    const F8 s = each8(g, sigmoid_of);
    return act == NORM_SIGMOID ? s : g * s;
}
// act(g) and its derivative, from g and its sigmoid.
__device__ __forceinline__ F8 act_with(const F8& g, const F8& sigmoid, int act) { return act == NORM_PLAIN ? g : (act == NORM_SIGMOID ? sigmoid : g * sigmoid); }
__device__ __forceinline__ F8 slope_with(const F8& g, const F8& sigmoid, int act) {
    if (act == NORM_PLAIN) return all8(1.f);
    const F8 rest = fma8(sigmoid, -1.f, all8(1.f));
    return sigmoid * (act == NORM_SIGMOID ? rest : fma8(g, rest, all8(1.f)));
}
__device__ __forceinline__ float act_of(float g, int act) { return act == NORM_PLAIN ? g : (act == NORM_SIGMOID ? sigmoid_of(g) : g * sigmoid_of(g)); }
__device__ __forceinline__ float2 act_and_slope(float g, int act) {
    if (act == NORM_PLAIN) return make_float2(g, 1.f);
    const float s = sigmoid_of(g);
    return act == NORM_SIGMOID ? make_float2(s, s * (1.f - s)) : make_float2(g * s, s * (1.f + g * (1.f - s)));
}
#endif

}  // namespace kge
