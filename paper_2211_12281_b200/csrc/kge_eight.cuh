// Eight elements of a row or a tensor in a thread: how they are loaded, looked at in fp32, and stored (the norms' and the optimiser's kernels).
#pragma once

#include <type_traits>

#include "kge_ops.cuh"

namespace kge {

#ifdef __CUDACC__
// Eight elements in a thread, as the words they are loaded and stored in (as elements of 16 bits the compiler took the words apart and put them
// together again at every copy: the norms of 32,768 x 4,096 bf16 368 us, so 294).
template <typename T> struct Raw8 { uint32_t w[2 * sizeof(T)]; };

template <typename T> __device__ __forceinline__ Raw8<T> load_wide(const T* p) {
    Raw8<T> r;
    if constexpr (sizeof(T) == 4)
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "l"(p));
    else if constexpr (sizeof(T) == 2)
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p));
    else
        asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(p));
    return r;
}
template <typename T> __device__ __forceinline__ void store_wide(T* p, const Raw8<T>& r) {
    if constexpr (sizeof(T) == 4)
        asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     ::"r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]), "l"(p) : "memory");
    else if constexpr (sizeof(T) == 2)
        asm volatile("st.global.v4.b32 [%4], {%0, %1, %2, %3};" ::"r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "l"(p) : "memory");
    else
        asm volatile("st.global.v2.b32 [%2], {%0, %1};" ::"r"(r.w[0]), "r"(r.w[1]), "l"(p) : "memory");
}
// Element e of the eight, and back.
template <typename T> __device__ __forceinline__ T element(const Raw8<T>& r, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[e]);
    else if constexpr (sizeof(T) == 2) { const uint16_t h = (uint16_t)(r.w[e >> 1] >> (16 * (e & 1))); return *reinterpret_cast<const T*>(&h); }
    else return (T)(r.w[e >> 2] >> (8 * (e & 3)));
}
template <typename T> __device__ __forceinline__ void set_element(Raw8<T>& r, int e, T x) {
    if constexpr (sizeof(T) == 4) r.w[e] = __float_as_uint(x);
    else if constexpr (sizeof(T) == 2) {
        const uint32_t h = *reinterpret_cast<const uint16_t*>(&x);
        r.w[e >> 1] = e & 1 ? (r.w[e >> 1] & 0xFFFFu) | h << 16 : h;
    } else {
        r.w[e >> 2] = (e & 3 ? r.w[e >> 2] : 0u) | (uint32_t)(uint8_t)x << (8 * (e & 3));
    }
}

// Eight fp32 numbers.
struct F8 { float v[8]; };
template <class F> __device__ __forceinline__ F8 make8(F&& f) { F8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = f(e);
    return r; }


__device__ __forceinline__ F8 wide_of(const Raw8<float>& r) { return make8([&](int e) { return __uint_as_float(r.w[e]); }); }
__device__ __forceinline__ F8 wide_of(const Raw8<__nv_bfloat16>& r) { return make8([&](int e) { return __uint_as_float(e & 1 ? r.w[e >> 1] & 0xFFFF0000u : r.w[e >> 1] << 16); }); }
__device__ __forceinline__ F8 wide_of(const Raw8<__half>& r) { F8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r.w[i]));
        x.v[2 * i] = f.x;
        x.v[2 * i + 1] = f.y;
    }
    return x; }
template <typename T> __device__ __forceinline__ Raw8<T> narrow_of(const F8& x) { Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w[e] = __float_as_uint(x.v[e]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) { const __nv_bfloat162 h = __floats2bfloat162_rn(x.v[2 * i], x.v[2 * i + 1]); r.w[i] = *reinterpret_cast<const uint32_t*>(&h); }
            else { const __half2 h = __floats2half2_rn(x.v[2 * i], x.v[2 * i + 1]); r.w[i] = *reinterpret_cast<const uint32_t*>(&h); }
        }
    }
    return r; }
#endif

}  // namespace kge
