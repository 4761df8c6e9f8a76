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
    uint32_t key[20];             // the generator's round keys: k0 + r w0, k1 + r w1
    uint64_t step;
    const int64_t* step_dev;      // added to step, or NULL
    int vec;                      // all arrays start at multiples of 16 bytes
};

// Philox4x32 with 10 rounds; the round keys come with the launch, and 32 x 32 -> 64-bit products are one instruction each.
__device__ __forceinline__ Philox4 dropout_words(const DropoutParams& p, uint32_t group, uint64_t step) {
    uint32_t c0 = group, c1 = (uint32_t)step, c2 = (uint32_t)(step >> 32), c3 = p.site;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ p.key[2 * r]; c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ p.key[2 * r + 1]; c3 = (uint32_t)a;
    }
    return Philox4{c0, c1, c2, c3};
}

// Two groups of eight elements a thread, 256 groups apart: their loads are under way while the generator runs.  Bound by memory: 76.8 M
// bf16 with a residual in 70 us (6.6 TB/s; one group 73, four 71), issue slots 60 % busy.
constexpr int DROPOUT_GROUPS = 2;
template <typename TX, typename TO, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropoutParams p) {
    grid_dependency_wait();
    allow_dependents();
    const TX* x = static_cast<const TX*>(p.x);
    const TO* res = static_cast<const TO*>(p.residual);
    TO* out = static_cast<TO*>(p.out);
    const int64_t g0 = (int64_t)blockIdx.x * (256 * DROPOUT_GROUPS) + threadIdx.x;
    Pack<TX, 8> a[DROPOUT_GROUPS];
    Pack<TO, 8> r[DROPOUT_GROUPS];
    if (p.vec && (g0 + 256 * (DROPOUT_GROUPS - 1)) * 8 + 8 <= p.n) {
#pragma unroll
        for (int u = 0; u < DROPOUT_GROUPS; ++u) {
            a[u] = load_stream<Pack<TX, 8>>(x + (g0 + 256 * u) * 8);
            if (RES) r[u] = load_stream<Pack<TO, 8>>(res + (g0 + 256 * u) * 8);
        }
        const uint64_t step = p.step + (p.step_dev ? (uint64_t)*p.step_dev : 0ull);
#pragma unroll
        for (int u = 0; u < DROPOUT_GROUPS; ++u) {
            const Philox4 w = dropout_words(p, (uint32_t)(g0 + 256 * u), step);
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
            Pack<TO, 8> o;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool keep = (i & 1 ? words[i >> 1] >> 16 : words[i >> 1] & 0xFFFFu) >= p.cut;
                const float v = keep ? to_float(a[u].v[i]) : 0.f;          // a dropped infinity or NaN leaves nothing: selected, not multiplied
                o.v[i] = from_float<TO>(RES ? fmaf(v, p.scale, to_float(r[u].v[i])) : v * p.scale);
            }
            *reinterpret_cast<Pack<TO, 8>*>(out + (g0 + 256 * u) * 8) = o;
        }
        return;
    }
    // the end of the list, and arrays that start between multiples of 16 bytes
    const uint64_t step = p.step + (p.step_dev ? (uint64_t)*p.step_dev : 0ull);
#pragma unroll 1
    for (int u = 0; u < DROPOUT_GROUPS; ++u) {
        const int64_t g = g0 + 256 * u;
        const int m = (int)max((int64_t)0, min((int64_t)8, p.n - g * 8));
        if (m == 0) return;
        const Philox4 w = dropout_words(p, (uint32_t)g, step);
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < m) {
                const int64_t at = g * 8 + i;
                const bool keep = (i & 1 ? words[i >> 1] >> 16 : words[i >> 1] & 0xFFFFu) >= p.cut;
                const float v = keep ? to_float(x[at]) : 0.f;
                out[at] = from_float<TO>(RES ? fmaf(v, p.scale, to_float(res[at])) : v * p.scale);
            }
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
    for (uint32_t r = 0; r < 10; ++r) { q.key[2 * r] = (uint32_t)seed + r * 0x9E3779B9u; q.key[2 * r + 1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u; }
    q.step = step; q.step_dev = step_dev; q.site = 0x80000000u | (uint32_t)site;
    q.vec = aligned_to(x, 16) && aligned_to(out, 16) && (!residual || aligned_to(residual, 16));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid((unsigned)ceil_div(n, 8 * 256 * DROPOUT_GROUPS));
    return with_type(x_type, [&](auto tx) {
        return with_type(out_type, [&](auto to) {
            using TX = decltype(tx); using TO = decltype(to);
            return launch_status(residual ? launch_dependent(dropout_kernel<TX, TO, true>, grid, dim3(256), 0, s, q)
                                          : launch_dependent(dropout_kernel<TX, TO, false>, grid, dim3(256), 0, s, q));
        });
    });
}
