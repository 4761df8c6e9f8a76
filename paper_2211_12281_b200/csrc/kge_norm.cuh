// Rows of a residual block in registers: what the norms' forward and backward kernels share.
#pragma once

#include "kge_ops.cuh"

namespace kge {

enum { NORM_PLAIN = 0, NORM_SIGMOID = 1, NORM_SILU = 2 };
constexpr int NORM_THREADS = 256;              // of a CTA whose rows belong to lanes of one warp
constexpr int NORM_MOST = 8192;                // widest row that a CTA's threads hold, eight elements each
constexpr int NORM_LOOP_THREADS = 1024;        // of a CTA that goes over wider rows again and again

#ifdef __CUDACC__
// Eight elements of a row in a thread: neighbours where rows allow wide accesses, `lanes` apart where not.
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

// Where a thread's elements of pack k lie in its row.
struct Place {
    int first, step, d;
    Place() = default;
    __device__ __forceinline__ Place(bool wide, int lanes, int t, int k, int width)
        : first(wide ? (k * lanes + t) * 8 : k * lanes * 8 + t), step(wide ? 1 : lanes), d(width) {}
    __device__ __forceinline__ int at(int e) const { return first + e * step; }
    __device__ __forceinline__ bool holds(int e) const { return at(e) < d; }
    __device__ __forceinline__ bool any() const { return first < d; }
};
template <typename T> __device__ __forceinline__ Raw8<T> load_row(const T* row, const Place& w, bool wide) {
    if (wide && w.any()) return load_wide(row + w.first);
    Raw8<T> r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = !wide && w.holds(e) ? row[w.at(e)] : from_float<T>(0.f);
    return r;
}
template <typename T> __device__ __forceinline__ void store_row(T* row, const Place& w, bool wide, const float (&x)[8]) {
    Raw8<T> r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = from_float<T>(x[e]);
    if (wide) { if (w.any()) store_wide(row + w.first, r); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (w.holds(e)) row[w.at(e)] = r.v[e];
}
// A vector of parameters; `other` where it is not given or the row has ended.
__device__ __forceinline__ void load_vector(const float* p, const Place& w, bool wide, float other, float (&x)[8]) {
    if (p && wide && w.any()) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p + w.first)), b = __ldg(reinterpret_cast<const float4*>(p + w.first) + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p && !wide && w.holds(e) ? __ldg(p + w.at(e)) : other;
}

// Sums (or the largest) over the threads of a row: L lanes of a warp, or all of the CTA (L = 0), which takes turns with two sets of places
// in shared memory: one barrier each.
template <int L> struct Team {
    float (*parts)[2][32];
    int turn = 0;
    // (the largest of magnitudes as integers, which order as they do, a NaN above all)
    template <bool MOST> static __device__ __forceinline__ float join(float a, float b) {
        return MOST ? __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))) : a + b;
    }
    template <bool MOST, int N> __device__ __forceinline__ void all(float (&v)[N]) {
        constexpr int LANES = L == 0 ? 32 : L;
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = join<MOST>(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
        }
        if constexpr (L == 0) {
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) parts[turn][i][warp] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = lane < warps ? parts[turn][i][lane] : 0.f;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) v[i] = join<MOST>(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
            }
            turn ^= 1;
        }
    }
    __device__ __forceinline__ float sum(float x) { float v[1] = {x}; all<false>(v); return v[0]; }
    __device__ __forceinline__ void sum(float& x, float& y) { float v[2] = {x, y}; all<false>(v); x = v[0]; y = v[1]; }
    __device__ __forceinline__ float most(float x) { float v[1] = {x}; all<true>(v); return v[0]; }
};

__device__ __forceinline__ float sigmoid_of(float g) { return __fdividef(1.f, 1.f + expf(-g)); }
__device__ __forceinline__ float act_of(float g, int act) { return act == NORM_PLAIN ? g : (act == NORM_SIGMOID ? sigmoid_of(g) : g * sigmoid_of(g)); }
// act(g) and its derivative.
__device__ __forceinline__ float2 act_and_slope(float g, int act) {
    if (act == NORM_PLAIN) return make_float2(g, 1.f);
    const float s = sigmoid_of(g);
    return act == NORM_SIGMOID ? make_float2(s, s * (1.f - s)) : make_float2(g * s, s * (1.f + g * (1.f - s)));
}
#endif

}  // namespace kge
