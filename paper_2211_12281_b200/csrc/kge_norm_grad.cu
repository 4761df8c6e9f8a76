// Gradients of a residual block's norms, gate and scale (kge_norm.cu), from the gradients dz of z and dh of h.  With the rows' statistics as the
// forward pass left them, yn = (y - mu1) r1 (or y), a = yn w1 + b1, h = x + s act a, hn = (h - mu2) r2, c = w2 dz:
//   dh' = dh + r2 (c - mean(c) - hn mean(c hn))        dx = dh'
//   e = s dh',  dgate = act' a e,  f = w1 act e        dy = r1 (f - mean(f) - yn mean(f yn))
// and over the rows  T1 = sum dz hn,  T0 = sum dz,  S1 = sum act dh' yn,  S0 = sum act dh':
//   dw2 = T1,  db2 = T0,  dw1 = s S1,  db1 = s S0,  ds = w1 S1 + b1 S0       (mean(c) and mean(f) only where the norm takes a mean)
// x, y and the gate are read again rather than h: it is made from what the other gradients need anyway, and not rounded.
#include <algorithm>
#include <cmath>

#include "kge_norm.cuh"

namespace kge {

namespace {

struct NormGradParams {
    const void *x, *y, *gate, *dz, *dh;
    void *dx, *dy, *dgate;
    const float *w1, *b1, *scale, *w2;
    const float* stats;
    float* part;                       // [CTAs][sums][d]
    int64_t ldx, ldy, ldg, ldz, ldh, ldox, ldoy, ldog;
    int n, d;
    int post, layer, act, wide;
    int sums;                          // 0: no gradients of vectors; 2: T1, S1; 4: T0 and S0 too
    float inv_d;
};

constexpr int GRAD_CTAS = 592;                 // at most, each with sums of its own; a constant, so that the order of additions is the sizes' alone
constexpr int GRAD_HELD = 4096;                // widest row that a CTA's threads hold with its sums

// CTAs that share n rows, `per` at a time.
inline int grad_ctas(int64_t n, int per) { return (int)std::min<int64_t>(GRAD_CTAS, ceil_div(n, per)); }
inline int grad_lanes(int d) { return d <= 64 ? 8 : (d <= 128 ? 16 : 32); }
inline int grad_ctas_of(int64_t n, int d) { return grad_ctas(n, d <= 512 ? NORM_THREADS / grad_lanes(d) : 1); }

struct Sums { float t1[8], t0[8], s1[8], s0[8]; };

// One row: L lanes of a warp, or the CTA's threads.
template <typename TX, typename TB, int L, int K>
__device__ __forceinline__ void grad_row(const NormGradParams& p, Team<L>& team, int64_t r, const Place (&at)[K], Sums (&sums)[K]) {
    const bool wide = p.wide, live = at[0].d > 0;
    float dh[K][8], yn[K][8], gate[K][8];
    const float4 st = live ? __ldg(reinterpret_cast<const float4*>(p.stats + 4 * r)) : make_float4(0.f, 0.f, 0.f, 0.f);
    {
        Raw8<TX> x[K], dhr[K];
        Raw8<TB> y[K], g[K], dz[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (p.dh) dhr[k] = load_row(static_cast<const TX*>(p.dh) + r * p.ldh, at[k], wide);
            if (p.dz) {
                x[k] = load_row(static_cast<const TX*>(p.x) + r * p.ldx, at[k], wide);
                dz[k] = load_row(static_cast<const TB*>(p.dz) + r * p.ldz, at[k], wide);
            }
            if (p.y) y[k] = load_row(static_cast<const TB*>(p.y) + r * p.ldy, at[k], wide);
            if (p.gate) g[k] = load_row(static_cast<const TB*>(p.gate) + r * p.ldg, at[k], wide);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dh[k][e] = p.dh ? to_float(dhr[k].v[e]) : 0.f;
                yn[k][e] = p.y && at[k].holds(e) ? (to_float(y[k].v[e]) - st.x) * (p.post ? st.y : 1.f) : 0.f;
                gate[k][e] = p.gate ? to_float(g[k].v[e]) : 0.f;
            }
        if (p.dz) {
            float hn[K][8], c[K][8], mean = 0.f, dot = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float w1[8], b1[8], s[8], w2[8];
                load_vector(p.w1, at[k], wide, 1.f, w1);
                load_vector(p.b1, at[k], wide, 0.f, b1);
                load_vector(p.scale, at[k], wide, 1.f, s);
                load_vector(p.w2, at[k], wide, 0.f, w2);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float h = to_float(x[k].v[e]);
                    if (p.y) h = fmaf(fmaf(yn[k][e], w1[e], b1[e]) * (p.gate ? act_of(gate[k][e], p.act) : 1.f), s[e], h);
                    const float z = to_float(dz[k].v[e]);
                    hn[k][e] = at[k].holds(e) ? (h - st.z) * st.w : 0.f;
                    c[k][e] = z * w2[e];
                    mean += c[k][e];
                    dot = fmaf(c[k][e], hn[k][e], dot);
                    sums[k].t1[e] = fmaf(z, hn[k][e], sums[k].t1[e]);
                    sums[k].t0[e] += z;
                }
            }
            if (p.layer) team.sum(mean, dot);
            else { dot = team.sum(dot); mean = 0.f; }
            mean *= p.inv_d; dot *= p.inv_d;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) dh[k][e] = fmaf(st.w, c[k][e] - mean - hn[k][e] * dot, dh[k][e]);
        }
    }
    if (p.dx) {
#pragma unroll
        for (int k = 0; k < K; ++k) store_row(static_cast<TX*>(p.dx) + r * p.ldox, at[k], wide, dh[k]);
    }
    if (!p.y) return;
    float f[K][8], mean = 0.f, dot = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float w1[8], b1[8], s[8], dg[8];
        load_vector(p.w1, at[k], wide, 1.f, w1);
        load_vector(p.b1, at[k], wide, 0.f, b1);
        load_vector(p.scale, at[k], wide, 1.f, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 act = p.gate ? act_and_slope(gate[k][e], p.act) : make_float2(1.f, 0.f);
            const float u = at[k].holds(e) ? act.x * dh[k][e] : 0.f, ee = s[e] * dh[k][e];
            dg[e] = act.y * fmaf(yn[k][e], w1[e], b1[e]) * ee;
            sums[k].s1[e] = fmaf(u, yn[k][e], sums[k].s1[e]);
            sums[k].s0[e] += u;
            f[k][e] = u * s[e] * w1[e];
            mean += f[k][e];
            dot = fmaf(f[k][e], yn[k][e], dot);
        }
        if (p.dgate) store_row(static_cast<TB*>(p.dgate) + r * p.ldog, at[k], wide, dg);
    }
    if (!p.dy) return;
    if (p.post) {
        if (p.layer) team.sum(mean, dot);
        else { dot = team.sum(dot); mean = 0.f; }
        mean *= p.inv_d; dot *= p.inv_d;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[k][e] = st.y * (f[k][e] - mean - yn[k][e] * dot);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) store_row(static_cast<TB*>(p.dy) + r * p.ldoy, at[k], wide, f[k]);
}

template <typename TX, typename TB, int L, int K>
__global__ void __launch_bounds__(L == 0 ? GRAD_HELD / 8 : NORM_THREADS) norm_grad_kernel(const __grid_constant__ NormGradParams p) {
    __shared__ float parts[2][2][32];
    __shared__ float joined[L == 0 ? 1 : NORM_THREADS * 8 * K];
    Team<L> team{parts};
    constexpr int TEAMS = L == 0 ? 1 : NORM_THREADS / (L == 0 ? 1 : L);
    const int lanes = L == 0 ? (int)blockDim.x : L, t = L == 0 ? (int)threadIdx.x : (int)threadIdx.x % L, mine = L == 0 ? 0 : threadIdx.x / (L == 0 ? 1 : L);
    grid_dependency_wait();
    allow_dependents();
    Sums sums[K] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * TEAMS; r0 < p.n; r0 += (int64_t)gridDim.x * TEAMS) {
        const int64_t r = r0 + mine;
        Place at[K];
#pragma unroll
        for (int k = 0; k < K; ++k) at[k] = Place(p.wide, lanes, t, k, r < p.n ? p.d : 0);
        grad_row<TX, TB, L, K>(p, team, r, at, sums);
    }
    if (p.sums == 0) return;
    float* part = p.part + (int64_t)blockIdx.x * p.sums * p.d;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= p.sums) break;
        // (order: T1, S1, T0, S0)
        if constexpr (L == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const Place at(p.wide, lanes, t, k, p.d);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at.holds(e)) part[(int64_t)q * p.d + at.at(e)] = q == 0 ? sums[k].t1[e] : (q == 1 ? sums[k].s1[e] : (q == 2 ? sums[k].t0[e] : sums[k].s0[e]));
            }
        } else {
            constexpr int WIDTH = L * 8 * K;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const Place at(p.wide, lanes, t, k, WIDTH);
#pragma unroll
                for (int e = 0; e < 8; ++e) joined[mine * WIDTH + at.at(e)] = q == 0 ? sums[k].t1[e] : (q == 1 ? sums[k].s1[e] : (q == 2 ? sums[k].t0[e] : sums[k].s0[e]));
            }
            __syncthreads();
            for (int i = threadIdx.x; i < p.d; i += NORM_THREADS) {
                float v = joined[i];
                for (int m = 1; m < TEAMS; ++m) v += joined[m * WIDTH + i];
                part[(int64_t)q * p.d + i] = v;
            }
        }
    }
}

// Rows wider than that: gone over again for every sum, from cache; the sums over rows are added up in the CTA's own part.  (An element's
// thread is the same in every pass, and only a row's last one stores: a result may take an operand's place.)
template <typename TX, typename TB>
__global__ void __launch_bounds__(NORM_LOOP_THREADS) norm_grad_loop_kernel(const __grid_constant__ NormGradParams p) {
    __shared__ float parts[2][2][32];
    Team<0> team{parts};
    grid_dependency_wait();
    allow_dependents();
    float* part = p.part + (int64_t)blockIdx.x * p.sums * p.d;
    bool first = true;
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x, first = false) {
        const TX* x = static_cast<const TX*>(p.x) + r * p.ldx;
        const TX* dhr = p.dh ? static_cast<const TX*>(p.dh) + r * p.ldh : nullptr;
        const TB* dz = p.dz ? static_cast<const TB*>(p.dz) + r * p.ldz : nullptr;
        const TB* y = p.y ? static_cast<const TB*>(p.y) + r * p.ldy : nullptr;
        const TB* gate = p.gate ? static_cast<const TB*>(p.gate) + r * p.ldg : nullptr;
        const float4 st = *reinterpret_cast<const float4*>(p.stats + 4 * r);
        float mean_c = 0.f, dot_c = 0.f, mean_f = 0.f, dot_f = 0.f;
        struct Element { float yn, a, act, slope, s, w1, hn, z, dh; };
        auto element = [&](int i) {
            Element v{0.f, 0.f, 1.f, 0.f, p.scale ? p.scale[i] : 1.f, p.w1 ? p.w1[i] : 1.f, 0.f, 0.f, dhr ? to_float(dhr[i]) : 0.f};
            if (y) {
                v.yn = (to_float(y[i]) - st.x) * (p.post ? st.y : 1.f);
                v.a = fmaf(v.yn, v.w1, p.b1 ? p.b1[i] : 0.f);
                if (gate) { const float2 g = act_and_slope(to_float(gate[i]), p.act); v.act = g.x; v.slope = g.y; }
            }
            if (dz) {
                v.z = to_float(dz[i]);
                v.hn = (fmaf(v.a * v.act, v.s, to_float(x[i])) - st.z) * st.w;
                v.dh = fmaf(st.w, v.z * p.w2[i] - mean_c - v.hn * dot_c, v.dh);
            }
            return v;
        };
        auto sums_of = [&](float& mean, float& dot, auto&& f) {
            float m = 0.f, o = 0.f;
            for (int i = threadIdx.x; i < p.d; i += NORM_LOOP_THREADS) {
                const float2 v = f(i);
                m += v.x;
                o = fmaf(v.x, v.y, o);
            }
            team.sum(m, o);
            mean = p.layer ? m * p.inv_d : 0.f;
            dot = o * p.inv_d;
        };
        if (dz) {
            float m, o;
            sums_of(m, o, [&](int i) { const Element v = element(i); return make_float2(v.z * p.w2[i], v.hn); });
            mean_c = m; dot_c = o;
        }
        if (y && p.post && p.dy) {
            float m, o;
            sums_of(m, o, [&](int i) { const Element v = element(i); return make_float2(v.act * v.dh * v.s * v.w1, v.yn); });
            mean_f = m; dot_f = o;
        }
        for (int i = threadIdx.x; i < p.d; i += NORM_LOOP_THREADS) {
            const Element v = element(i);
            const float u = v.act * v.dh, f = u * v.s * v.w1;
            if (p.dx) static_cast<TX*>(p.dx)[r * p.ldox + i] = from_float<TX>(v.dh);
            if (p.dgate) static_cast<TB*>(p.dgate)[r * p.ldog + i] = from_float<TB>(v.slope * v.a * (v.s * v.dh));
            if (p.dy) static_cast<TB*>(p.dy)[r * p.ldoy + i] = from_float<TB>(p.post ? st.y * (f - mean_f - v.yn * dot_f) : f);
            if (p.sums) {
                const float add[4] = {v.z * v.hn, u * v.yn, v.z, u};
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < p.sums) part[(int64_t)q * p.d + i] = first ? add[q] : part[(int64_t)q * p.d + i] + add[q];
            }
        }
    }
}

// The CTAs' sums, added in their order; then what the vectors' gradients are.
struct NormJoinParams {
    const float* part;
    const float *w1, *b1, *scale;
    float *dw1, *db1, *dscale, *dw2, *db2;
    int ctas, sums, d, accumulate;
};
constexpr int JOIN_COLS = 32, JOIN_ROWS = 8;
__global__ void __launch_bounds__(JOIN_COLS * JOIN_ROWS) norm_join_kernel(const __grid_constant__ NormJoinParams p) {
    __shared__ float part[4][JOIN_ROWS][JOIN_COLS];
    grid_dependency_wait();
    allow_dependents();
    const int c = blockIdx.x * JOIN_COLS + threadIdx.x % JOIN_COLS, row = threadIdx.x / JOIN_COLS;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < p.d) {
        for (int g = row; g < p.ctas; g += JOIN_ROWS) {
#pragma unroll
            for (int q = 0; q < 4; ++q) if (q < p.sums) v[q] += p.part[((int64_t)g * p.sums + q) * p.d + c];
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) part[q][row][threadIdx.x % JOIN_COLS] = v[q];
    __syncthreads();
    if (row > 0 || c >= p.d) return;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        for (int i = 1; i < JOIN_ROWS; ++i) v[q] += part[q][i][threadIdx.x];
    auto give = [&](float* to, float x) { if (to) to[c] = p.accumulate ? to[c] + x : x; };
    const float s = p.scale ? p.scale[c] : 1.f, w1 = p.w1 ? p.w1[c] : 1.f, b1 = p.b1 ? p.b1[c] : 0.f;
    give(p.dw2, v[0]);
    give(p.db2, v[2]);
    give(p.dw1, s * v[1]);
    give(p.db1, s * v[3]);
    give(p.dscale, p.b1 ? fmaf(w1, v[1], b1 * v[3]) : w1 * v[1]);
}

template <typename TX, typename TB>
int launch_norm_grad(const NormGradParams& p, int ctas, cudaStream_t s) {
    auto launch = [&](auto kernel, int threads) { return launch_status(launch_dependent(kernel, dim3((unsigned)ctas), dim3((unsigned)threads), 0, s, p)); };
    if (p.d <= 64) return launch(norm_grad_kernel<TX, TB, 8, 1>, NORM_THREADS);
    if (p.d <= 128) return launch(norm_grad_kernel<TX, TB, 16, 1>, NORM_THREADS);
    if (p.d <= 256) return launch(norm_grad_kernel<TX, TB, 32, 1>, NORM_THREADS);
    if (p.d <= 512) return launch(norm_grad_kernel<TX, TB, 32, 2>, NORM_THREADS);
    if (p.d <= GRAD_HELD) return launch(norm_grad_kernel<TX, TB, 0, 1>, (int)ceil_div(p.d, 256) * 32);
    return launch(norm_grad_loop_kernel<TX, TB>, NORM_LOOP_THREADS);
}

}  // namespace
}  // namespace kge

using namespace kge;

extern "C" {

size_t kge_block_norm_grad_scratch_bytes(int64_t n, int32_t d) {
    if (n < 1 || n > INT32_MAX || d < 1 || d > INT32_MAX - 65536) return 0;
    return (size_t)grad_ctas_of(n, d) * 4 * (size_t)d * sizeof(float);
}

int kge_block_norm_grad(const kge_norm_block* b, int64_t n, int32_t d, const float* stats, const void* dz, int64_t ld_dz, const void* dh, int64_t ld_dh,
                        const kge_norm_grads* o, int32_t accumulate, void* scratch, size_t scratch_bytes, void* stream) {
    if (!b || !o || !is_float_type(b->x_type) || !is_float_type(b->block_type) || n < 0 || n > INT32_MAX || d < 1 || d > INT32_MAX - 65536 ||
        (b->layer != 0 && b->layer != 1) || (b->gate && (b->gate_act < 0 || b->gate_act > 2)) || (accumulate != 0 && accumulate != 1)) return KGE_ERR_BAD_ARG;
    // (arrays of no rows may have no address: without rows only the vectors are looked at)
    if (n > 0 && ((!dz && !dh) || (!b->y && (b->gate || b->post_weight || b->post_bias || b->scale || o->dy || o->dgate || o->dpost_weight || o->dpost_bias || o->dscale))))
        return KGE_ERR_BAD_ARG;
    if ((b->post_bias && !b->post_weight) || (dz && !b->pre_weight)) return KGE_ERR_BAD_ARG;
    if (n > 0 && ((o->dgate && !b->gate) || (o->dpost_weight && !b->post_weight) || (o->dpost_bias && !b->post_weight) || (o->dscale && !b->scale) ||
                  ((o->dpre_weight || o->dpre_bias) && !dz))) return KGE_ERR_BAD_ARG;
    const float* vectors[9] = {b->post_weight, b->post_bias, b->scale, b->pre_weight, o->dpost_weight, o->dpost_bias, o->dscale, o->dpre_weight, o->dpre_bias};
    for (const float* v : vectors) if (!aligned_to(v, 4)) return KGE_ERR_BAD_ARG;
    const int xs = type_bytes(b->x_type), bs = type_bytes(b->block_type);
    const bool wanted = o->dpost_weight || o->dpost_bias || o->dscale || o->dpre_weight || o->dpre_bias;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    NormJoinParams j{};
    j.w1 = b->post_weight; j.b1 = b->post_bias; j.scale = b->scale;
    j.dw1 = o->dpost_weight; j.db1 = o->dpost_bias; j.dscale = o->dscale; j.dw2 = o->dpre_weight; j.db2 = o->dpre_bias;
    j.d = d; j.accumulate = accumulate;
    j.sums = o->dpost_bias || o->dpre_bias || (o->dscale && b->post_bias) ? 4 : 2;
    if (n > 0) {
        auto ok = [&](const void* p, int64_t ld, int size) { return !p || (ld >= d && aligned_to(p, (size_t)size)); };
        if (!stats || !aligned_to(stats, 16) || !b->x || !ok(b->x, b->ldx, xs) || !ok(b->y, b->ldy, bs) || !ok(b->gate, b->ld_gate, bs) || !ok(dz, ld_dz, bs) ||
            !ok(dh, ld_dh, xs) || !ok(o->dx, o->ld_dx, xs) || !ok(o->dy, o->ld_dy, bs) || !ok(o->dgate, o->ld_dgate, bs)) return KGE_ERR_BAD_ARG;
        auto packs = [&](const void* p, int64_t ld, int size) { return !p || (ld % 8 == 0 && aligned_to(p, (size_t)(8 * size))); };
        NormGradParams p{};
        p.wide = d % 8 == 0 && packs(b->x, b->ldx, xs) && packs(b->y, b->ldy, bs) && packs(b->gate, b->ld_gate, bs) && packs(dz, ld_dz, bs) && packs(dh, ld_dh, xs) &&
                 packs(o->dx, o->ld_dx, xs) && packs(o->dy, o->ld_dy, bs) && packs(o->dgate, o->ld_dgate, bs);
        for (int i = 0; i < 4; ++i) p.wide = p.wide && aligned_to(vectors[i], 16);
        p.x = b->x; p.y = b->y; p.gate = b->gate; p.dz = dz; p.dh = dh; p.dx = o->dx; p.dy = o->dy; p.dgate = o->dgate;
        p.w1 = b->post_weight; p.b1 = b->post_bias; p.scale = b->scale; p.w2 = b->pre_weight; p.stats = stats;
        p.ldx = b->ldx; p.ldy = b->ldy; p.ldg = b->ld_gate; p.ldz = ld_dz; p.ldh = ld_dh; p.ldox = o->ld_dx; p.ldoy = o->ld_dy; p.ldog = o->ld_dgate;
        p.n = (int)n; p.d = d; p.post = b->post_weight != nullptr; p.layer = b->layer; p.act = b->gate_act; p.inv_d = 1.f / (float)d;
        const int ctas = grad_ctas_of(n, d);
        if (wanted) {
            if (!scratch || !aligned_to(scratch, 256) || scratch_bytes < kge_block_norm_grad_scratch_bytes(n, d)) return KGE_ERR_WORKSPACE;
            p.sums = j.sums;
            p.part = static_cast<float*>(scratch);
        }
        const int rc = with_type(b->x_type, [&](auto tx) { return with_type(b->block_type, [&](auto tb) { return launch_norm_grad<decltype(tx), decltype(tb)>(p, ctas, s); }); });
        if (rc != KGE_OK) return rc;
        j.part = p.part; j.ctas = ctas;
    }
    if (!wanted || (n == 0 && accumulate)) return KGE_OK;
    return launch_status(launch_dependent(norm_join_kernel, dim3((unsigned)ceil_div(d, JOIN_COLS)), dim3(JOIN_COLS * JOIN_ROWS), 0, s, j));
}

}  // extern "C"
