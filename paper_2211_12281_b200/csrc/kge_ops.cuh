// What the handle-less operators on rows share (lookup and its gradient, dropout, 8-bit quantisation and products): element
// types, packs of elements that move as one access, and host-side checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "kge_common.cuh"

namespace kge {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool is_float_type(int t) { return t == KGE_F32 || t == KGE_BF16 || t == KGE_F16; }
inline bool is_fp8_type(int t) { return t == KGE_E4M3 || t == KGE_E5M2; }
inline int type_bytes(int t) { return t == KGE_F32 ? 4 : (is_float_type(t) ? 2 : 1); }
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
// An error that an earlier, unrelated call left behind is not this launch's: the launch's own code is what is looked at.
inline int launch_status(cudaError_t e) { return e == cudaSuccess ? KGE_OK : KGE_ERR_CUDA; }

// Largest of `most`, most / 2, ..., 1 elements that divides a row of `dim` and starts at multiples of its bytes (of 16, if it has more)
// in every row of both matrices.
inline int vector_length(int most, int64_t dim, int64_t ld0, int bytes0, const void* p0, int64_t ld1, int bytes1, const void* p1) {
    auto fits = [](int v, int64_t ld, int bytes, const void* p) {
        const int64_t step = v * bytes < 16 ? v * bytes : 16;
        return ld * bytes % step == 0 && aligned_to(p, (size_t)step);
    };
    for (int v = most; v > 1; v >>= 1)
        if (dim % v == 0 && fits(v, ld0, bytes0, p0) && fits(v, ld1, bytes1, p1)) return v;
    return 1;
}

// n / d and n % d by a multiplication, for n < 2^31 (d >= 1): m = floor(2^(31 + l) / d) + 1 with l = ceil(log2 d) is exact there.
struct FastDiv {
    uint32_t d, m, s;
    FastDiv() = default;
    explicit FastDiv(uint32_t div) : d(div), m(0), s(0) {
        if (d > 1) {
            uint32_t l = 0;
            while ((1ull << l) < d) ++l;
            m = (uint32_t)(((1ull << (31 + l)) / d) + 1);
            s = l - 1;
        }
    }
#ifdef __CUDACC__
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return d == 1 ? n : __umulhi(n, m) >> s; }
#endif
};

// Streaming multiprocessors of the current device.
inline int sm_count(int* sms) {
    static std::atomic<int> known[kMaxDevices];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return KGE_ERR_CUDA;
    const bool tracked = dev >= 0 && dev < kMaxDevices;
    *sms = tracked ? known[dev].load(std::memory_order_relaxed) : 0;
    if (*sms == 0) {
        e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return KGE_ERR_CUDA;
        if (tracked) known[dev].store(*sms, std::memory_order_relaxed);
    }
    return KGE_OK;
}

#ifdef __CUDACC__
template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };
// fp32 in packs of eight are two 16-byte accesses
template <> struct alignas(16) Pack<float, 8> { float v[8]; };

// A pack of read-only memory, loaded here and not where the compiler would rather have it (it moves a load whose value is used under
// a condition to that condition, behind the loads and uses before it).
template <typename P> __device__ __forceinline__ P load_now(const void* p) {
    P r;
    if constexpr (sizeof(P) == 2) {
        uint16_t a;
        asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(a) : "l"(p));
        *reinterpret_cast<uint16_t*>(&r) = a;
    } else if constexpr (sizeof(P) == 4) {
        asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(*reinterpret_cast<uint32_t*>(&r)) : "l"(p));
    } else if constexpr (sizeof(P) == 8) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&r);
        asm volatile("ld.global.nc.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    } else {
        uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
        for (int i = 0; i < (int)sizeof(P) / 16; ++i)
            asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                         : "l"(static_cast<const char*>(p) + 16 * i));
    }
    return r;
}

// A pack that is read once, in 16-byte pieces past the L1 cache (it may be overwritten in place by its own thread afterwards).
template <typename P> __device__ __forceinline__ P load_stream(const void* p) {
    P r;
    uint4* w = reinterpret_cast<uint4*>(&r);
#pragma unroll
    for (int i = 0; i < (int)sizeof(P) / 16; ++i) w[i] = __ldcs(static_cast<const uint4*>(p) + i);
    return r;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// Two fp32 operations in one instruction, each rounded as a single one would be.
__device__ __forceinline__ uint64_t pair(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 unpair(uint64_t a) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a)); return r; }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }

__device__ __forceinline__ void note_status(int32_t* status, int code) { if (status) set_status(status, code); }

// Calls f with a value of the element type `t` names.
template <class F> inline int with_type(int t, F&& f) {
    if (t == KGE_F32) return f(float());
    if (t == KGE_BF16) return f(__nv_bfloat16());
    return f(__half());
}
#endif

}  // namespace kge
