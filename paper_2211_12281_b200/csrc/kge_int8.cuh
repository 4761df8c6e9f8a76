// Rounding to 8-bit integers with a scale for each row (the norm's and the quantiser's kernels).
#pragma once

#include "kge_eight.cuh"

namespace kge {

#ifdef __CUDACC__
// A row's scale, and what its values are multiplied by, from its largest magnitude a.  Zeros alone have scale 1; an infinity or a NaN makes
// it NaN, and all of the row stands for that.
struct RowScale { float s, inv; };
__device__ __forceinline__ RowScale row_scale(float a) {
    RowScale r;
    r.s = a < __int_as_float(0x7F800000) ? (a == 0.f ? 1.f : fmaxf(__fdiv_rn(a, 127.f), 1.17549435e-38f)) : __int_as_float(0x7FC00000);       // (false for a NaN)
    r.inv = __fdiv_rn(1.f, r.s);
    return r;
}

// |y| < 2^22 plus this has y rounded to an integer (ties to even) in its low bits; of a product and this, the exact product is rounded.
constexpr float ROUND_TO_INT = 12582912.f;

// The low bytes of eight such sums.
__device__ __forceinline__ uint2 low_bytes(const F8& t) {
    uint2 w;
    const uint32_t a = __byte_perm(__float_as_uint(t.v[0]), __float_as_uint(t.v[1]), 0x0040), b = __byte_perm(__float_as_uint(t.v[2]), __float_as_uint(t.v[3]), 0x0040);
    const uint32_t c = __byte_perm(__float_as_uint(t.v[4]), __float_as_uint(t.v[5]), 0x0040), d = __byte_perm(__float_as_uint(t.v[6]), __float_as_uint(t.v[7]), 0x0040);
    w.x = __byte_perm(a, b, 0x5410);
    w.y = __byte_perm(c, d, 0x5410);
    return w;
}
// Integers nearest to the fp32 values times 1 / s, the product exact: within 1/2 + 2^-17 of the true quotients.
__device__ __forceinline__ uint2 round_products(const F8& x, float inv) { return low_bytes(make8([&](int e) { return fmaf(x.v[e], inv, ROUND_TO_INT); })); }
#endif

}  // namespace kge
