// Dropout from a counter-based generator: which elements stay is a function of (seed, step, site, index), so the backward pass
// makes the mask again instead of reading it.
//   element i:  h = 16-bit half (i mod 8) of Philox4x32-10(key = seed, counter = (i div 8, step lo, step hi, 2^31 | site))
//               out = h >= cut ? x * 65536 / (65536 - cut) : 0,  cut = rint(65536 p)   (+ residual)
// Sixteen bits an element: one call of the generator, some eighty integer instructions, serves eight elements.
#include <cmath>

#include "kge_ops.cuh"
#include "kge_sample.cuh"

namespace kge {

namespace {

struct DropoutParams {
    const void *x, *residual;
    void* out;
    int64_t n;
    uint32_t cut, site;
    float scale;
    uint64_t seed, step;
    const int64_t* step_dev;      // added to step, or NULL
    int vec;                      // all arrays start at multiples of 16 bytes
};

template <typename TX, typename TO, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutParams p) {
    const int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x, i0 = g * 8;
    if (i0 >= p.n) return;
    const uint64_t step = p.step + (p.step_dev ? (uint64_t)*p.step_dev : 0ull);
    const TX* x = static_cast<const TX*>(p.x) + i0;
    const TO* res = static_cast<const TO*>(p.residual) + (RES ? i0 : 0);
    TO* out = static_cast<TO*>(p.out) + i0;
    const int m = (int)min((int64_t)8, p.n - i0);
    Pack<TX, 8> a;
    Pack<TO, 8> r;
    const bool whole = p.vec && m == 8;
    if (whole) {
        a = *reinterpret_cast<const Pack<TX, 8>*>(x);
        if (RES) r = *reinterpret_cast<const Pack<TO, 8>*>(res);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < m) { a.v[i] = x[i]; if (RES) r.v[i] = res[i]; }
    }
    const Philox4 w = philox4x32_10((uint32_t)g, (uint32_t)step, (uint32_t)(step >> 32), p.site, (uint32_t)p.seed, (uint32_t)(p.seed >> 32));
    const uint32_t words[4] = {w.x, w.y, w.z, w.w};
    Pack<TO, 8> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t h = i & 1 ? words[i >> 1] >> 16 : words[i >> 1] & 0xFFFFu;
        const bool keep = h >= p.cut;          // a dropped infinity or NaN leaves nothing: selected, not multiplied
        const float v = keep ? to_float(a.v[i]) : 0.f;
        o.v[i] = from_float<TO>(RES ? fmaf(v, p.scale, to_float(r.v[i])) : v * p.scale);
    }
    if (whole) *reinterpret_cast<Pack<TO, 8>*>(out) = o;
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < m) out[i] = o.v[i];
    }
}

}  // namespace
}  // namespace kge

using namespace kge;

extern "C" int kge_dropout(const void* x, int32_t x_type, const void* residual, void* out, int32_t out_type, int64_t n, double p,
                           uint64_t seed, uint64_t step, const int64_t* step_dev, int32_t site, void* stream) {
    if (!is_float_type(x_type) || !is_float_type(out_type) || n < 0 || n > (1ll << 34) || !(p >= 0.0 && p <= 1.0) || site < 0) return KGE_ERR_BAD_ARG;
    if (n == 0) return KGE_OK;
    if (!x || !out || !aligned_to(x, type_bytes(x_type)) || !aligned_to(out, type_bytes(out_type)) ||
        (residual && !aligned_to(residual, type_bytes(out_type))) || (step_dev && !aligned_to(step_dev, 8))) return KGE_ERR_BAD_ARG;
    DropoutParams q{};
    q.x = x; q.residual = residual; q.out = out; q.n = n;
    q.cut = (uint32_t)std::nearbyint(p * 65536.0);
    q.scale = q.cut < 65536u ? (float)(65536.0 / (65536.0 - q.cut)) : 0.f;
    q.seed = seed; q.step = step; q.step_dev = step_dev; q.site = 0x80000000u | (uint32_t)site;
    q.vec = aligned_to(x, 16) && aligned_to(out, 16) && (!residual || aligned_to(residual, 16));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid((unsigned)ceil_div(n, 8 * 256));
    return with_type(x_type, [&](auto tx) {
        return with_type(out_type, [&](auto to) {
            using TX = decltype(tx); using TO = decltype(to);
            if (residual) dropout_kernel<TX, TO, true><<<grid, 256, 0, s>>>(q);
            else dropout_kernel<TX, TO, false><<<grid, 256, 0, s>>>(q);
            return launch_status(cudaGetLastError());
        });
    });
}
