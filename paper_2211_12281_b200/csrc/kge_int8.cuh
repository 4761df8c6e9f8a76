// Rounding to 8-bit integers with a scale for each row (the norm's and the quantiser's kernels).
#pragma once

#include "kge_ops.cuh"

namespace kge {

#ifdef __CUDACC__
// A row's scale and its reciprocal, from its largest magnitude a.  Zeros alone have scale 1; an infinity or a NaN makes the scale one, and
// the factor 0: the row's integers are 0 and stand for NaN, all of them.
struct RowScale { float s, inv; };
__device__ __forceinline__ RowScale row_scale(float a) {
    const bool finite = a < __int_as_float(0x7F800000);       // (false for a NaN)
    RowScale r{a, 0.f};
    if (finite) {
        r.s = a == 0.f ? 1.f : fmaxf(__fdiv_rn(a, 127.f), 1.17549435e-38f);
        r.inv = __fdiv_rn(1.f, r.s);
    }
    return r;
}
// The integer nearest to the true quotient x / s (ties to even), not to its rounded form: t = |x| (1 / s) is within 2^-23 of it, and the
// middles k + 1/2 are multiples of 16 units of their fp32 neighbours; m, such a multiple next to t, is compared with the quotient exactly (the sign of
// |x| - m s, one fused operation) and moved a unit to the side where that lies.
__device__ __forceinline__ int round_quotient(float x, const RowScale& r) {
    const float ax = r.inv == 0.f ? 0.f : fabsf(x);
    int m = (int)(__float_as_uint(ax * r.inv) + 8u) & ~15;
    const float d = fmaf(-__int_as_float(m), r.s, ax);
    m += d > 0.f ? 1 : (d < 0.f ? -1 : 0);
    const int q = __float2int_rn(__int_as_float(m));
    return x < 0.f ? -q : q;
}
__device__ __forceinline__ uint2 pack_bytes(const int (&q)[8]) {
    return make_uint2((q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | (uint32_t)q[3] << 24,
                      (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | (uint32_t)q[7] << 24);
}
#endif

}  // namespace kge
