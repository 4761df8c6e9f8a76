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

constexpr int GRAD_HELD = 4096;                // widest row that a CTA's threads hold with its sums
constexpr int GRAD_SMS = 148;                  // CTAs are as many as this many SMs run, each with sums of its own: a constant, so that the order of additions is the sizes' alone

// CTAs that share n rows, each as many as the others.
inline int grad_ctas_of(int64_t n, int d) {
    const int team = norm_team(d), threads = (int)std::min<int64_t>(ceil_div(d, 256) * 32, 512);
    const int64_t all = team == 0 ? n : ceil_div(n, NORM_THREADS / team), room = GRAD_SMS * (team == 0 ? std::max(1, 512 / threads) : 2);
    return (int)ceil_div(all, ceil_div(all, room));
}

template <typename TX, typename TB> struct GradRow { Raw8<TX> x, dh; Raw8<TB> y, gate, dz; float4 stats; };
template <typename TX, typename TB, bool WIDE>
__device__ __forceinline__ void load_grad_row(const NormGradParams& p, int64_t r, const Place<WIDE>& at, GradRow<TX, TB>& v) {
    if (p.dh) v.dh = at.load(static_cast<const TX*>(p.dh) + r * p.ldh);
    if (p.dz) {
        v.dz = at.load(static_cast<const TB*>(p.dz) + r * p.ldz);
        v.x = at.load(static_cast<const TX*>(p.x) + r * p.ldx);
    }
    if (p.y) v.y = at.load(static_cast<const TB*>(p.y) + r * p.ldy);
    if (p.gate) v.gate = at.load(static_cast<const TB*>(p.gate) + r * p.ldg);
    v.stats = __ldg(reinterpret_cast<const float4*>(p.stats + 4 * r));
}

struct Sums { F8 t1, s1, t0, s0; };
__device__ __forceinline__ const F8& sum_of(const Sums& s, int q) { return q == 0 ? s.t1 : (q == 1 ? s.s1 : (q == 2 ? s.t0 : s.s0)); }

// One row of a team (live: it is the team's own).
template <typename TX, typename TB, int L, bool WIDE>
__device__ __forceinline__ void grad_row(const NormGradParams& p, Team<L>& team, int64_t r, bool live, const Place<WIDE>& at, const GradRow<TX, TB>& v, Sums& sums) {
    F8 dh = p.dh ? wide_of(v.dh) : all8(0.f), yn = all8(0.f), gate = all8(0.f), act = all8(1.f);
    if (p.y) {
        yn = wide_of(v.y);
        if (p.post) yn = (yn + -v.stats.x) * v.stats.y;
    }
    if (p.gate) {
        gate = wide_of(v.gate);
        act = p.act == NORM_PLAIN ? gate : sigmoid_of(gate);          // (its sigmoid, where there is one)
    }
    float mean = 0.f, along = 0.f;
    if (p.dz) {
        F8 h = wide_of(v.x);
        if (p.y) {
            F8 a = yn;
            if (p.w1) a = a * at.vector(p.w1);
            if (p.b1) a = a + at.vector(p.b1);
            if (p.gate) a = a * act_with(gate, act, p.act);
            h = p.scale ? fma8(a, at.vector(p.scale), h) : a + h;
        }
        const F8 hn = (h + -v.stats.z) * v.stats.w, dz = wide_of(v.dz), c = dz * at.vector(p.w2);
        if (live) {
            sums.t1 = fma8(dz, hn, sums.t1);
            if (p.sums > 2) sums.t0 = sums.t0 + dz;
        }
        along = at.dot(c, hn);
        if (p.layer) { mean = at.total(c); team.sum(mean, along); }
        else along = team.sum(along);
        dh = fma8(fma8(hn, -along * p.inv_d, p.layer ? c + -mean * p.inv_d : c), v.stats.w, dh);
    }
    if (p.dx) at.store(static_cast<TX*>(p.dx) + r * p.ldox, dh, live);
    if (!p.y) return;
    F8 f = dh;
    if (p.gate) f = f * act_with(gate, act, p.act);
    if (live) {
        sums.s1 = fma8(f, yn, sums.s1);
        if (p.sums > 2) sums.s0 = sums.s0 + f;
    }
    if (p.scale) {
        const F8 s = at.vector(p.scale);
        f = f * s;
        dh = dh * s;
    }
    const F8 w1 = p.w1 ? at.vector(p.w1) : all8(1.f);
    if (p.dgate) {
        F8 a = yn;
        if (p.w1) a = a * w1;
        if (p.b1) a = a + at.vector(p.b1);
        at.store(static_cast<TB*>(p.dgate) + r * p.ldog, slope_with(gate, act, p.act) * a * dh, live);
    }
    if (!p.dy) return;
    if (p.post) {
        f = f * w1;
        along = at.dot(f, yn);
        if (p.layer) { mean = at.total(f); team.sum(mean, along); }
        else along = team.sum(along);
        f = fma8(yn, -along * p.inv_d, p.layer ? f + -mean * p.inv_d : f) * v.stats.y;
    }
    at.store(static_cast<TB*>(p.dy) + r * p.ldoy, f, live);
}

// Teams take rows in turn, the next one's loads under way, and add up the columns' sums of theirs in registers.  (Teams that have run out of rows go along with
// the last one.)
template <typename TX, typename TB, int L, bool WIDE>
__global__ void __launch_bounds__(L == 0 ? GRAD_HELD / 8 : NORM_THREADS, L == 0 ? 1 : 2) norm_grad_kernel(const __grid_constant__ NormGradParams p) {
    __shared__ float parts[2][2][32];
    __shared__ float joined[L == 0 ? 1 : NORM_THREADS * 8];
    Team<L> team(parts);
    const int t = team.thread, last = p.n - 1;
    const Place<WIDE> at(Team<L>::size(), t, 0, p.d);
    const int64_t step = (int64_t)gridDim.x * Team<L>::COUNT;
    grid_dependency_wait();
    allow_dependents();
    Sums sums{all8(0.f), all8(0.f), all8(0.f), all8(0.f)};
    GradRow<TX, TB> next;
    load_grad_row<TX, TB>(p, min((int64_t)blockIdx.x * Team<L>::COUNT + team.index, (int64_t)last), at, next);
    for (int64_t r0 = (int64_t)blockIdx.x * Team<L>::COUNT; r0 < p.n; r0 += step) {
        const int64_t mine = r0 + team.index;
        const GradRow<TX, TB> now = next;
        if (r0 + step < p.n) load_grad_row<TX, TB>(p, min(mine + step, (int64_t)last), at, next);
        grad_row<TX, TB, L, WIDE>(p, team, min(mine, (int64_t)last), mine <= last, at, now, sums);
    }
    if (p.sums == 0) return;
    float* part = p.part + (int64_t)blockIdx.x * p.sums * p.d;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q >= p.sums) break;
        if constexpr (L == 0) {
            at.store(part + (int64_t)q * p.d, sum_of(sums, q), true);
        } else {
            constexpr int WIDTH = L * 8;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) if (at.holds(e)) joined[team.index * WIDTH + at.at(e)] = sum_of(sums, q).v[e];
            __syncthreads();
            for (int i = threadIdx.x; i < p.d; i += NORM_THREADS) {
                float v = joined[i];
                for (int m = 1; m < Team<L>::COUNT; ++m) v += joined[m * WIDTH + i];
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
    Team<0> team(parts);
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
constexpr int JOIN_COLS = 32, JOIN_ROWS = 32;
__global__ void __launch_bounds__(JOIN_COLS * JOIN_ROWS) norm_join_kernel(const __grid_constant__ NormJoinParams p) {
    __shared__ float part[4][JOIN_ROWS][JOIN_COLS];
    grid_dependency_wait();
    allow_dependents();
    const int col = threadIdx.x % JOIN_COLS, c = blockIdx.x * JOIN_COLS + col, row = threadIdx.x / JOIN_COLS;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < p.d) {
#pragma unroll 4
        for (int g = row; g < p.ctas; g += JOIN_ROWS) {
#pragma unroll
            for (int q = 0; q < 4; ++q) if (q < p.sums) v[q] += p.part[((int64_t)g * p.sums + q) * p.d + c];
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) part[q][row][col] = v[q];
    __syncthreads();
    if (row > 0 || c >= p.d) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll 8
        for (int i = 1; i < JOIN_ROWS; ++i) v[q] += part[q][i][col];
    }
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
    if (p.d > GRAD_HELD) return launch(norm_grad_loop_kernel<TX, TB>, NORM_LOOP_THREADS);
    const int team = norm_team(p.d), threads = (int)ceil_div(p.d, 256) * 32;
    if (!p.wide) {
        // (teams as for wide rows, so that the columns' sums are the same)
        switch (team) {
            case 8: return launch(norm_grad_kernel<TX, TB, 8, false>, NORM_THREADS);
            case 16: return launch(norm_grad_kernel<TX, TB, 16, false>, NORM_THREADS);
            case 32: return launch(norm_grad_kernel<TX, TB, 32, false>, NORM_THREADS);
            case 64: return launch(norm_grad_kernel<TX, TB, 64, false>, NORM_THREADS);
            case 128: return launch(norm_grad_kernel<TX, TB, 128, false>, NORM_THREADS);
            default: return launch(norm_grad_kernel<TX, TB, 0, false>, threads);
        }
    }
    switch (team) {
        case 8: return launch(norm_grad_kernel<TX, TB, 8, true>, NORM_THREADS);
        case 16: return launch(norm_grad_kernel<TX, TB, 16, true>, NORM_THREADS);
        case 32: return launch(norm_grad_kernel<TX, TB, 32, true>, NORM_THREADS);
        case 64: return launch(norm_grad_kernel<TX, TB, 64, true>, NORM_THREADS);
        case 128: return launch(norm_grad_kernel<TX, TB, 128, true>, NORM_THREADS);
        default: return launch(norm_grad_kernel<TX, TB, 0, true>, threads);
    }
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
