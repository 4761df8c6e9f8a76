// The norms after and before a block, fused with its gate and residual scale:
//   a = N1(y) (or y),  h = x + s act(g) a,  z = N2(h);   N(u) = (u - mu) r w + b,  r = 1 / sqrt(mean((u - mu)^2) + eps),  mu = mean(u), or 0
// h is rounded once, when it is stored; z is made of the unrounded one.  z may leave as 8-bit integers with a scale for each row.
#include <cmath>

#include "kge_int8.cuh"
#include "kge_norm.cuh"

namespace kge {

namespace {

struct NormParams {
    const void *x, *y, *gate;
    void *h, *z;
    const float *w1, *b1, *scale, *w2, *b2;
    float *stats, *z_scales;
    int64_t ldx, ldy, ldg, ldh, ldz;
    int n, d;
    int post, layer, act, z8;          // act is looked at where a gate is given
    int wide;                          // every array's rows start at multiples of eight elements, vectors at multiples of four
    float eps, inv_d;
};

__device__ __forceinline__ float deviation(const NormParams& p, float squares) { return rsqrtf(fmaf(squares, p.inv_d, p.eps)); }

// Mean and reciprocal deviation of a row, in two passes over the registers (a mean far from zero does not eat the deviation's digits).
template <class T, int K>
__device__ __forceinline__ float2 row_stats(const NormParams& p, T& team, const float (&u)[K][8], const Place (&at)[K]) {
    float mu = 0.f, sq = 0.f;
    if (p.layer) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) mu += u[k][e];          // (zeros beyond the row)
        mu = team.sum(mu) * p.inv_d;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float c = at[k].holds(e) ? u[k][e] - mu : 0.f;
            sq = fmaf(c, c, sq);
        }
    return make_float2(mu, deviation(p, team.sum(sq)));
}

template <typename TB>
__device__ __forceinline__ void store_z8(const NormParams& p, int64_t row, const Place& at, const float (&z)[8], const RowScale& s) {
    int8_t* out = static_cast<int8_t*>(p.z) + row * p.ldz;
    int q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = round_quotient(z[e], s);
    if (p.wide) {
        if (!at.any()) return;
        uint2 w;
        w.x = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | (uint32_t)q[3] << 24;
        w.y = (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | (uint32_t)q[7] << 24;
        *reinterpret_cast<uint2*>(out + at.first) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (at.holds(e)) out[at.at(e)] = (int8_t)q[e];
    }
}

// L lanes hold a row (L = 0: the CTA's threads), K packs of eight elements each.
template <typename TX, typename TB, int L, int K>
__global__ void __launch_bounds__(L == 0 ? NORM_MOST / 8 : NORM_THREADS) norm_kernel(const __grid_constant__ NormParams p) {
    __shared__ float parts[2][2][32];
    Team<L> team{parts};
    const int lanes = L == 0 ? (int)blockDim.x : L, t = L == 0 ? (int)threadIdx.x : (int)threadIdx.x % L;
    const int64_t r = L == 0 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (NORM_THREADS / (L == 0 ? 1 : L)) + threadIdx.x / (L == 0 ? 1 : L);
    const bool live = r < p.n;
    const bool wide = p.wide;
    Place at[K];
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] = Place(wide, lanes, t, k, live ? p.d : 0);
    grid_dependency_wait();
    allow_dependents();
    float u[K][8];
    {
        Raw8<TX> x[K];
        Raw8<TB> y[K], g[K];
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] = load_row(static_cast<const TX*>(p.x) + r * p.ldx, at[k], wide);
        if (p.y) {
#pragma unroll
            for (int k = 0; k < K; ++k) y[k] = load_row(static_cast<const TB*>(p.y) + r * p.ldy, at[k], wide);
            if (p.gate) {
#pragma unroll
                for (int k = 0; k < K; ++k) g[k] = load_row(static_cast<const TB*>(p.gate) + r * p.ldg, at[k], wide);
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) u[k][e] = to_float(y[k].v[e]);
            if (p.post) {
                const float2 s = row_stats(p, team, u, at);
                if (p.stats && live && t == 0) *reinterpret_cast<float2*>(p.stats + 4 * r) = s;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    float w[8], b[8];
                    load_vector(p.w1, at[k], wide, 0.f, w);
                    load_vector(p.b1, at[k], wide, 0.f, b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[k][e] = fmaf((u[k][e] - s.x) * s.y, w[e], b[e]);
                }
            }
            if (p.gate) {
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[k][e] *= act_of(to_float(g[k].v[e]), p.act);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float w[8];
                load_vector(p.scale, at[k], wide, 1.f, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[k][e] = at[k].holds(e) ? fmaf(u[k][e], w[e], to_float(x[k].v[e])) : 0.f;
                if (p.h) store_row(static_cast<TX*>(p.h) + r * p.ldh, at[k], wide, u[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) u[k][e] = to_float(x[k].v[e]);
        }
    }
    if (p.stats && !p.post && live && t == 0) *reinterpret_cast<float2*>(p.stats + 4 * r) = make_float2(0.f, 0.f);
    if (!p.z) {
        if (p.stats && live && t == 0) *reinterpret_cast<float2*>(p.stats + 4 * r + 2) = make_float2(0.f, 0.f);
        return;
    }
    const float2 s = row_stats(p, team, u, at);
    if (p.stats && live && t == 0) *reinterpret_cast<float2*>(p.stats + 4 * r + 2) = s;
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float w[8], b[8];
        load_vector(p.w2, at[k], wide, 0.f, w);
        load_vector(p.b2, at[k], wide, 0.f, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[k][e] = fmaf((u[k][e] - s.x) * s.y, w[e], b[e]);
            if (at[k].holds(e)) most = Team<L>::template join<true>(most, fabsf(u[k][e]));
        }
        if (!p.z8) store_row(static_cast<TB*>(p.z) + r * p.ldz, at[k], wide, u[k]);
    }
    if (p.z8) {
        const RowScale q = row_scale(team.most(most));
        if (live && t == 0) p.z_scales[r] = q.s;
#pragma unroll
        for (int k = 0; k < K; ++k) store_z8<TB>(p, r, at[k], u[k], q);
    }
}

// Rows wider than a CTA's registers: the row is gone over again for every sum, from cache.  (An element's thread is the same in every
// pass, and only the last one stores: a result may take an operand's place.)
template <typename TX, typename TB>
__global__ void __launch_bounds__(NORM_LOOP_THREADS) norm_loop_kernel(const __grid_constant__ NormParams p) {
    __shared__ float parts[2][2][32];
    Team<0> team{parts};
    const int64_t r = blockIdx.x;
    grid_dependency_wait();
    allow_dependents();
    const TX* x = static_cast<const TX*>(p.x) + r * p.ldx;
    const TB* y = static_cast<const TB*>(p.y) + (p.y ? r * p.ldy : 0);
    const TB* gate = static_cast<const TB*>(p.gate) + (p.gate ? r * p.ldg : 0);
    auto sum = [&](auto&& f) {
        float v = 0.f;
        for (int i = threadIdx.x; i < p.d; i += NORM_LOOP_THREADS) v += f(i);
        return team.sum(v);
    };
    auto stats_of = [&](auto&& f) {
        float2 s = make_float2(0.f, 0.f);
        if (p.layer) s.x = sum(f) * p.inv_d;
        s.y = deviation(p, sum([&](int i) { const float c = f(i) - s.x; return c * c; }));
        return s;
    };
    float2 s1 = make_float2(0.f, 0.f), s2 = make_float2(0.f, 0.f);
    if (p.post) s1 = stats_of([&](int i) { return to_float(y[i]); });
    auto stream = [&](int i) {
        float u = to_float(x[i]);
        if (p.y) {
            float a = to_float(y[i]);
            if (p.post) a = fmaf((a - s1.x) * s1.y, p.w1[i], p.b1 ? p.b1[i] : 0.f);
            if (p.gate) a *= act_of(to_float(gate[i]), p.act);
            u = fmaf(a, p.scale ? p.scale[i] : 1.f, u);
        }
        return u;
    };
    if (p.z) s2 = stats_of(stream);
    auto normed = [&](float u, int i) { return fmaf((u - s2.x) * s2.y, p.w2[i], p.b2 ? p.b2[i] : 0.f); };
    RowScale q{1.f, 0.f};
    if (p.z && p.z8) {
        float most = 0.f;
        for (int i = threadIdx.x; i < p.d; i += NORM_LOOP_THREADS) most = Team<0>::join<true>(most, fabsf(normed(stream(i), i)));
        q = row_scale(team.most(most));
        if (threadIdx.x == 0) p.z_scales[r] = q.s;
    }
    for (int i = threadIdx.x; i < p.d; i += NORM_LOOP_THREADS) {
        const float u = stream(i);
        if (p.h) static_cast<TX*>(p.h)[r * p.ldh + i] = from_float<TX>(u);
        if (p.z && p.z8) static_cast<int8_t*>(p.z)[r * p.ldz + i] = (int8_t)round_quotient(normed(u, i), q);
        else if (p.z) static_cast<TB*>(p.z)[r * p.ldz + i] = from_float<TB>(normed(u, i));
    }
    if (p.stats && threadIdx.x == 0) *reinterpret_cast<float4*>(p.stats + 4 * r) = make_float4(s1.x, s1.y, s2.x, s2.y);
}

template <typename TX, typename TB>
int launch_norm(const NormParams& p, cudaStream_t s) {
    auto lanes = [&](auto kernel, int per) { return launch_status(launch_dependent(kernel, dim3((unsigned)ceil_div(p.n, NORM_THREADS / per)), dim3(NORM_THREADS), 0, s, p)); };
    if (p.d <= 64) return lanes(norm_kernel<TX, TB, 8, 1>, 8);
    if (p.d <= 128) return lanes(norm_kernel<TX, TB, 16, 1>, 16);
    if (p.d <= 256) return lanes(norm_kernel<TX, TB, 32, 1>, 32);
    if (p.d <= 512) return lanes(norm_kernel<TX, TB, 32, 2>, 32);
    if (p.d <= 1024) return lanes(norm_kernel<TX, TB, 32, 4>, 32);
    if (p.d <= NORM_MOST) return launch_status(launch_dependent(norm_kernel<TX, TB, 0, 1>, dim3((unsigned)p.n), dim3((unsigned)(ceil_div(p.d, 256) * 32)), 0, s, p));
    return launch_status(launch_dependent(norm_loop_kernel<TX, TB>, dim3((unsigned)p.n), dim3(NORM_LOOP_THREADS), 0, s, p));
}

}  // namespace
}  // namespace kge

using namespace kge;

extern "C" int kge_block_norm(const kge_norm_block* b, int64_t n, int32_t d, void* h, int64_t ldh, void* z, int32_t z_int8, int64_t ldz, float* z_scales,
                              float eps, float* stats, void* stream) {
    if (!b || !is_float_type(b->x_type) || !is_float_type(b->block_type) || n < 0 || n > INT32_MAX || d < 1 || d > INT32_MAX - 65536 || (b->layer != 0 && b->layer != 1) ||
        (b->gate && (b->gate_act < 0 || b->gate_act > 2)) || (z_int8 != 0 && z_int8 != 1) || !(eps >= 0.f) || std::isinf(eps)) return KGE_ERR_BAD_ARG;
    if (n == 0) return KGE_OK;
    if ((!h && !z) || (!b->y && (h || b->gate || b->post_weight || b->post_bias || b->scale))) return KGE_ERR_BAD_ARG;
    if ((b->post_bias && !b->post_weight) || (z && !b->pre_weight) || (z && z_int8 && !z_scales)) return KGE_ERR_BAD_ARG;
    const int xs = type_bytes(b->x_type), bs = type_bytes(b->block_type), zs = z_int8 ? 1 : bs;
    auto ok = [&](const void* p, int64_t ld, int size) { return !p || (ld >= d && aligned_to(p, (size_t)size)); };
    if (!b->x || !ok(b->x, b->ldx, xs) || !ok(b->y, b->ldy, bs) || !ok(b->gate, b->ld_gate, bs) || !ok(h, ldh, xs) || !ok(z, ldz, zs)) return KGE_ERR_BAD_ARG;
    const float* vectors[5] = {b->post_weight, b->post_bias, b->scale, b->pre_weight, b->pre_bias};
    bool wide = d % 8 == 0;
    for (const float* v : vectors) {
        if (!aligned_to(v, 4)) return KGE_ERR_BAD_ARG;
        wide = wide && aligned_to(v, 16);
    }
    if (!aligned_to(z_scales, 4) || !aligned_to(stats, 16)) return KGE_ERR_BAD_ARG;
    auto packs = [&](const void* p, int64_t ld, int size) { return !p || (ld % 8 == 0 && aligned_to(p, (size_t)(8 * size))); };
    wide = wide && packs(b->x, b->ldx, xs) && packs(b->y, b->ldy, bs) && packs(b->gate, b->ld_gate, bs) && packs(h, ldh, xs) && packs(z, ldz, zs);
    NormParams p{};
    p.x = b->x; p.y = b->y; p.gate = b->gate; p.h = h; p.z = z;
    p.w1 = b->post_weight; p.b1 = b->post_bias; p.scale = b->scale; p.w2 = b->pre_weight; p.b2 = b->pre_bias;
    p.stats = stats; p.z_scales = z_scales;
    p.ldx = b->ldx; p.ldy = b->ldy; p.ldg = b->ld_gate; p.ldh = ldh; p.ldz = ldz;
    p.n = (int)n; p.d = d; p.post = b->post_weight != nullptr; p.layer = b->layer; p.act = b->gate_act; p.z8 = z_int8; p.wide = wide;
    p.eps = eps; p.inv_d = 1.f / (float)d;
    return with_type(b->x_type, [&](auto tx) {
        return with_type(b->block_type, [&](auto tb) { return launch_norm<decltype(tx), decltype(tb)>(p, static_cast<cudaStream_t>(stream)); });
    });
}
