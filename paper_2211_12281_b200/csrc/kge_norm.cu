// The norms after and before a block, fused with its gate and residual scale:
//   a = N1(y) (or y),  h = x + s act(g) a,  z = N2(h);   N(u) = (u - mu) r w + b,  r = 1 / sqrt(mean((u - mu)^2) + eps),  mu = mean(u), or 0
// h is rounded once, when it is stored; z is made of the unrounded one.  z may leave as 8-bit integers with a scale for each row.
#include <algorithm>
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

// Takes the mean out of a team's row; returns it and the reciprocal deviation.  Two passes over the registers: a mean far from zero does not eat the deviation's digits.
template <int L, bool WIDE>
__device__ __forceinline__ float2 centre(const NormParams& p, Team<L>& team, F8& u, const Place<WIDE>& at) {
    float mu = 0.f;
    if (p.layer) {
        mu = team.sum(at.total(u)) * p.inv_d;
        u = u + -mu;
    }
    return make_float2(mu, deviation(p, team.sum(at.dot(u, u))));
}

// (z is off by its own roundings: what the product with 1 / s adds to them moves an integer only where they do)
template <bool WIDE>
__device__ __forceinline__ void store_z8(const NormParams& p, int64_t row, const Place<WIDE>& at, const F8& z, const RowScale& s) {
    int8_t* out = static_cast<int8_t*>(p.z) + row * p.ldz;
    const uint2 w = round_products(z, s.inv);
    if constexpr (WIDE) {
        if (at.any) *reinterpret_cast<uint2*>(at.mine(out)) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (at.holds(e)) out[at.at(e)] = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
    }
}

template <typename TX, typename TB> struct NormRow { Raw8<TX> x; Raw8<TB> y, gate; };
template <typename TX, typename TB, bool WIDE>
__device__ __forceinline__ void load_norm_row(const NormParams& p, int64_t r, const Place<WIDE>& at, NormRow<TX, TB>& v) {
    v.x = at.load(static_cast<const TX*>(p.x) + r * p.ldx);
    if (p.y) v.y = at.load(static_cast<const TB*>(p.y) + r * p.ldy);
    if (p.gate) v.gate = at.load(static_cast<const TB*>(p.gate) + r * p.ldg);
}

// Teams of L threads (L = 0: the CTA) take rows in turn, the next one's loads under way.  (Teams that have run out of rows go along with the last one.)
template <typename TX, typename TB, int L, bool WIDE>
__global__ void __launch_bounds__(L == 0 ? NORM_MOST / 8 : NORM_THREADS, L == 0 ? 1 : NORM_CTAS) norm_kernel(const __grid_constant__ NormParams p) {
    __shared__ float parts[2][2][32];
    Team<L> team(parts);
    const int t = team.thread, last = p.n - 1;
    const Place<WIDE> at(Team<L>::size(), t, p.d);
    const int64_t step = (int64_t)gridDim.x * Team<L>::COUNT;
    grid_dependency_wait();
    allow_dependents();
    NormRow<TX, TB> next;
    load_norm_row<TX, TB>(p, min((int64_t)blockIdx.x * Team<L>::COUNT + team.index, (int64_t)last), at, next);
    for (int64_t r0 = (int64_t)blockIdx.x * Team<L>::COUNT; r0 < p.n; r0 += step) {
        const int64_t mine = r0 + team.index, r = L == 0 ? mine : min(mine, (int64_t)last);
        const bool live = L == 0 || mine <= last;
        const NormRow<TX, TB> now = next;
        if (r0 + step < p.n) load_norm_row<TX, TB>(p, min(mine + step, (int64_t)last), at, next);
        float* const stats = p.stats && live && t == 0 ? p.stats + 4 * r : nullptr;
        F8 u = wide_of(now.x);
        float2 s = make_float2(0.f, 0.f);
        if (p.y) {
            F8 a = wide_of(now.y);
            if (p.post) {
                s = centre(p, team, a, at);
                a = a * s.y * at.vector(p.w1);
                if (p.b1) a = a + at.vector(p.b1);
            }
            if (p.gate) {
                const F8 g = wide_of(now.gate);
                a = a * (p.act == NORM_PLAIN ? g : act_with(g, sigmoid_of(g), p.act));
            }
            u = p.scale ? fma8(a, at.vector(p.scale), u) : a + u;
            if (p.h) at.store(static_cast<TX*>(p.h) + r * p.ldh, u, live);
        }
        if (stats) *reinterpret_cast<float2*>(stats) = s;
        s = make_float2(0.f, 0.f);
        if (p.z) {
            s = centre(p, team, u, at);
            u = u * s.y * at.vector(p.w2);
            if (p.b2) u = u + at.vector(p.b2);
            if (p.z8) {
                float most = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) if (at.holds(e)) most = Team<L>::template join<true>(most, fabsf(u.v[e]));
                const RowScale q = row_scale(team.most(most));
                if (live && t == 0) p.z_scales[r] = q.s;
                if (live) store_z8(p, r, at, u, q);
            } else {
                at.store(static_cast<TB*>(p.z) + r * p.ldz, u, live);
            }
        }
        if (stats) *reinterpret_cast<float2*>(stats + 2) = s;
    }
}

// Rows wider than a CTA's registers: the row is gone over again for every sum, from cache.  (An element's thread is the same in every
// pass, and only the last one stores: a result may take an operand's place.)
template <typename TX, typename TB>
__global__ void __launch_bounds__(NORM_LOOP_THREADS) norm_loop_kernel(const __grid_constant__ NormParams p) {
    __shared__ float parts[2][2][32];
    Team<0> team(parts);
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
        if (p.z && p.z8) static_cast<int8_t*>(p.z)[r * p.ldz + i] = (int8_t)__float_as_int(fmaf(normed(u, i), q.inv, ROUND_TO_INT));
        else if (p.z) static_cast<TB*>(p.z)[r * p.ldz + i] = from_float<TB>(normed(u, i));
    }
    if (p.stats && threadIdx.x == 0) *reinterpret_cast<float4*>(p.stats + 4 * r) = make_float4(s1.x, s1.y, s2.x, s2.y);
}

// As many CTAs as run at a time, or fewer, so that each has as many rows as the others.
template <typename TX, typename TB, int L, bool WIDE>
int launch_rows(const NormParams& p, int sms, cudaStream_t s) {
    const int threads = L == 0 ? (int)ceil_div(p.d, 256) * 32 : NORM_THREADS;
    const int64_t all = ceil_div(p.n, Team<L>::COUNT), room = (int64_t)sms * (L == 0 ? std::max(1, 1024 / threads) : NORM_CTAS), turns = ceil_div(all, room);
    return launch_status(launch_dependent(norm_kernel<TX, TB, L, WIDE>, dim3((unsigned)ceil_div(all, turns)), dim3((unsigned)threads), 0, s, p));
}

template <typename TX, typename TB>
int launch_norm(const NormParams& p, cudaStream_t s) {
    int sms = 0;
    const int rc = sm_count(&sms);
    if (rc != KGE_OK) return rc;
    if (p.d > NORM_MOST) return launch_status(launch_dependent(norm_loop_kernel<TX, TB>, dim3((unsigned)p.n), dim3(NORM_LOOP_THREADS), 0, s, p));
    const int team = norm_team(p.d);
    if (!p.wide) return team == 0 ? launch_rows<TX, TB, 0, false>(p, sms, s) : (team > 32 ? launch_rows<TX, TB, 128, false>(p, sms, s) : launch_rows<TX, TB, 32, false>(p, sms, s));
    switch (team) {
        case 8: return launch_rows<TX, TB, 8, true>(p, sms, s);
        case 16: return launch_rows<TX, TB, 16, true>(p, sms, s);
        case 32: return launch_rows<TX, TB, 32, true>(p, sms, s);
        case 64: return launch_rows<TX, TB, 64, true>(p, sms, s);
        case 128: return launch_rows<TX, TB, 128, true>(p, sms, s);
        default: return launch_rows<TX, TB, 0, true>(p, sms, s);
    }
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
