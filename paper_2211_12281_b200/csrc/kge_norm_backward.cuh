// Gradients of a residual block's norms, gate and scale (kge_norm_forward.cuh), from the gradients dz of z and dh of h.  With the rows' statistics as the
// forward pass left them, yn = (y - mu1) r1 (or y), a = yn w1 + b1, h = x + s act a, hn = (h - mu2) r2, c = w2 dz:
//   dh' = dh + r2 (c - mean(c) - hn mean(c hn))        dx = dh'
//   e = s dh',  dgate = act' a e,  f = w1 act e        dy = r1 (f - mean(f) - yn mean(f yn))
// and over the rows  T1 = sum dz hn,  T0 = sum dz,  S1 = sum act dh' yn,  S0 = sum act dh':
//   dw2 = T1,  db2 = T0,  dw1 = s S1,  db1 = s S0,  ds = w1 S1 + b1 S0       (mean(c) and mean(f) only where the norm takes a mean)
// x, y and the gate are read again rather than h: it is made from what the other gradients need anyway, and not rounded.
#pragma once

#include <algorithm>

#include "kge_norm.cuh"

namespace kge {

struct NormGradParams {
    const void *x, *y, *gate, *dz, *dh;
    void *dx, *dy, *dgate;
    const float *w1, *b1, *scale, *w2;
    const float* stats;
    float* part;                       // [CTAs][sums][d]
    int64_t ldx, ldy, ldg, ldz, ldh, ldox, ldoy, ldog;
    int n, d;
    int post, layer, act, access;         // access: elements that move as one in every array, 8, 2 or 1
    int sums;                          // 0: no gradients of vectors; 2: T1, S1; 4: T0 and S0 too
    float inv_d;
};

constexpr int GRAD_HELD = 4096;                // widest row that a CTA's threads hold with the vectors and the columns' sums
constexpr int GRAD_SMS = 148;                  // CTAs are as many as this many SMs run, each with sums of its own: a constant, so that the order of additions is the sizes' alone

// CTAs that share n rows, each as many as the others.
inline int grad_ctas_of(int64_t n, int d) {
    const int team = norm_team(d), threads = (int)std::min<int64_t>(ceil_div(d, 256) * 32, 512);
    const int64_t all = team == 0 ? n : ceil_div(n, NORM_THREADS / team), room = GRAD_SMS * (team == 0 ? std::max(1, 512 / threads) : 2);
    return (int)ceil_div(all, ceil_div(all, room));
}

// Launches the kernel for fp32, bf16 or fp16 rows of x (each in a source of its own, so that they are compiled side by side).
int launch_norm_grad_f32(const NormGradParams& p, int block_type, int ctas, cudaStream_t s);
int launch_norm_grad_bf16(const NormGradParams& p, int block_type, int ctas, cudaStream_t s);
int launch_norm_grad_f16(const NormGradParams& p, int block_type, int ctas, cudaStream_t s);

namespace {

template <typename TX, typename TB> struct GradRow { Raw8<TX> x, dh; Raw8<TB> y, gate[1], dz; float4 stats; };

// Teams take rows in turn, the next one's loads under way, and add up the columns' sums of theirs in registers.  (Teams that have run out of rows go along with
// the last one.)  The vectors enter as sw = s w1, sb = s b1 and w2, which a thread keeps: with q = yn sw + sb
//   h = x + act q,  dgate = act' q dh',  f = act dh' sw
// FULL: norms that take a mean, or biases; without them sb, T0 and S0 are not there.
// AHEAD: the next row's loads are under way where registers hold it too: with FULL only in teams of 32 to 128 threads, not where a CTA holds a row (16,384 x 4,096 bf16,
// layer norms: 350 us, root-mean-square norms 231).  (Two or three rows ahead, copied into shared memory asynchronously: 16,384 x 4,096 bf16 229
// instead of 234 us, 8,192 x 4,096 fp32 330 instead of 204, 24,576 x 256 46 instead of 38: it is not memory that they wait for.)
// SHARED: a CTA of up to 1,024 threads for a row of up to 8,192 columns, whose registers hold neither: the sums are in shared memory, a thread's own places, and the
// vectors are loaded where they are used (8,192 x 8,192 bf16: 390 us; gone over in three passes 2,284).
template <typename TX, typename TB, int L, int W, bool FULL, bool SHARED>
__global__ void __launch_bounds__(SHARED ? NORM_MOST / 8 : (L == 0 ? GRAD_HELD / 8 : NORM_THREADS), L == 0 ? 1 : 2) norm_grad_kernel(const __grid_constant__ NormGradParams p) {
    constexpr bool AHEAD = !SHARED && (!FULL || L >= 32) && (!FULL || sizeof(TX) + sizeof(TB) <= 6);
    __shared__ float parts[2][2][32];
    __shared__ float joined[L == 0 ? 1 : NORM_THREADS * 8];
    Team<L> team(parts);
    const int t = team.thread, last = p.n - 1;
    const Place<W> at(Team<L>::size(), t, 0, p.d);
    const int64_t step = (int64_t)gridDim.x * Team<L>::COUNT;
    grid_dependency_wait();
    allow_dependents();
    extern __shared__ float4 sums_in_shared[];
    auto scaled = [&](const float* v) { return p.scale ? at.vector(v) * at.vector(p.scale) : at.vector(v); };
    auto make_sw = [&] { return p.w1 ? scaled(p.w1) : (p.scale ? at.vector(p.scale) : all8(1.f)); };
    auto make_sb = [&] { return FULL && p.b1 ? scaled(p.b1) : all8(0.f); };
    P8 sw_held, sb_held, w2_held;
    if (!SHARED) { sw_held = make_sw(); sb_held = make_sb(); w2_held = p.w2 ? at.vector(p.w2) : all8(0.f); }
    // T1, S1, T0, S0
    P8 held[4] = {all8(0.f), all8(0.f), all8(0.f), all8(0.f)};
    auto place = [&](int q, int half) { return sums_in_shared + (2 * q + half) * (int)blockDim.x + t; };
    auto add = [&](int q, const P8& x, const P8& y) {
        if (!SHARED) { held[q] = fma8(x, y, held[q]); return; }
        if (q >= p.sums) return;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float4 s = *place(q, half);
            const float2 a = unpair(fma2(x.v[2 * half], y.v[2 * half], pair(s.x, s.y))), b = unpair(fma2(x.v[2 * half + 1], y.v[2 * half + 1], pair(s.z, s.w)));
            *place(q, half) = make_float4(a.x, a.y, b.x, b.y);
        }
    };
    if (SHARED) {
        for (int q = 0; q < p.sums; ++q) *place(q, 0) = *place(q, 1) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    GradRow<TX, TB> next;
    auto load = [&](int64_t row, GradRow<TX, TB>& v) {
        const int64_t r = L == 0 ? row : min(row, (int64_t)last);
        if (p.dh) v.dh = at.load(static_cast<const TX*>(p.dh) + r * p.ldh);
        if (p.dz) {
            v.dz = at.load(static_cast<const TB*>(p.dz) + r * p.ldz);
            v.x = at.load(static_cast<const TX*>(p.x) + r * p.ldx);
        }
        if (p.y) v.y = at.load(static_cast<const TB*>(p.y) + r * p.ldy);
        if (p.gate) v.gate[0] = at.load(static_cast<const TB*>(p.gate) + r * p.ldg);
        v.stats = __ldg(reinterpret_cast<const float4*>(p.stats + 4 * r));
    };
    if (AHEAD) load((int64_t)blockIdx.x * Team<L>::COUNT + team.index, next);
    for (int64_t r0 = (int64_t)blockIdx.x * Team<L>::COUNT; r0 < p.n; r0 += step) {
        const int64_t mine = r0 + team.index, r = L == 0 ? mine : min(mine, (int64_t)last);
        const bool live = L == 0 || mine <= last;
        GradRow<TX, TB> v;
        if (AHEAD) {
            v = next;
            if (r0 + step < p.n) load(mine + step, next);
        } else load(mine, v);

        P8 dh = p.dh ? pairs_of(v.dh) : all8(0.f), yn = all8(0.f), act = all8(1.f);
        if (p.y) {
            yn = pairs_of(v.y);
            if (p.post) yn = FULL ? fma8(yn, v.stats.y, all8(-v.stats.x * v.stats.y)) : yn * v.stats.y;
        }
        // act: the gate, or its sigmoid (of which a silu gate takes the gate's multiple wherever it is used)
        if (p.gate && p.act == NORM_PLAIN) act = pairs_of(v.gate[0]);
        else if (p.gate) with_sigmoids<false>(v.gate, [&](int, const P8& s) { act = s; });
        float mean = 0.f, along = 0.f;
        if (p.dz) {
            P8 h = pairs_of(v.x);
            if (p.y) {
                const P8 sw = SHARED ? make_sw() : sw_held;
                P8 q = FULL ? fma8(yn, sw, SHARED ? make_sb() : sb_held) : yn * sw;
                if (p.gate && p.act == NORM_SILU) q = q * pairs_of(v.gate[0]);
                h = fma8(q, act, h);
            }
            const P8 hn = FULL ? fma8(h, v.stats.w, all8(-v.stats.z * v.stats.w)) : h * v.stats.w, dz = pairs_of(v.dz), c = dz * (SHARED ? at.vector(p.w2) : w2_held);
            if (live) {
                add(0, dz, hn);
                if (FULL) add(2, dz, all8(1.f));
            }
            along = at.dot(c, hn);
            if (FULL) { mean = at.total(c); team.sum(mean, along); }
            else along = team.sum(along);
            mean = FULL && p.layer ? mean * p.inv_d : 0.f;
            dh = fma8(FULL ? fma8(hn, -along * p.inv_d, c + -mean) : fma8(hn, -along * p.inv_d, c), v.stats.w, dh);
        }
        if (p.dx) at.store(static_cast<TX*>(p.dx) + r * p.ldox, dh, live);
        if (!p.y) continue;
        const P8 sw = SHARED ? make_sw() : sw_held;
        if (p.dgate) {
            P8 q = (FULL ? fma8(yn, sw, SHARED ? make_sb() : sb_held) : yn * sw) * dh;
            if (p.act != NORM_PLAIN) {
                P8 slope = act * fma8(act, -1.f, all8(1.f));          // s (1 - s), and s + g s (1 - s)
                if (p.act == NORM_SILU) slope = fma8(pairs_of(v.gate[0]), slope, act);
                q = q * slope;
            }
            at.store(static_cast<TB*>(p.dgate) + r * p.ldog, q, live);
        }
        P8 f = dh;
        if (p.gate) {
            f = f * act;
            if (p.act == NORM_SILU) f = f * pairs_of(v.gate[0]);
        }
        if (live) {
            add(1, f, yn);
            if (FULL) add(3, f, all8(1.f));
        }
        if (!p.dy) continue;
        f = f * sw;
        if (p.post) {
            along = at.dot(f, yn);
            if (FULL) { mean = at.total(f); team.sum(mean, along); }
            else along = team.sum(along);
            mean = FULL && p.layer ? mean * p.inv_d : 0.f;
            f = (FULL ? fma8(yn, -along * p.inv_d, f + -mean) : fma8(yn, -along * p.inv_d, f)) * v.stats.y;
        }
        at.store(static_cast<TB*>(p.dy) + r * p.ldoy, f, live);
    }
    if (p.sums == 0) return;
    float* part = p.part + (int64_t)blockIdx.x * p.sums * p.d;
#pragma unroll
    for (int q = 0; q < (FULL ? 4 : 2); ++q) {
        if (q >= p.sums) break;
        P8 sum = held[q];
        if (SHARED) {
            const float4 a = *place(q, 0), b = *place(q, 1);
            sum = P8{{pair(a.x, a.y), pair(a.z, a.w), pair(b.x, b.y), pair(b.z, b.w)}};
        }
        if constexpr (L == 0) {
            at.store(part + (int64_t)q * p.d, sum, true);
        } else {
            constexpr int WIDTH = L * 8;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) if (at.holds(e)) joined[team.index * WIDTH + at.at(e)] = element(sum, e);
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

template <typename TX, typename TB, int W, bool FULL>
int launch_held(const NormGradParams& p, int ctas, cudaStream_t s) {
    auto launch = [&](auto kernel, int threads) { return launch_status(launch_dependent(kernel, dim3((unsigned)ctas), dim3((unsigned)threads), 0, s, p)); };
    const int threads = (int)ceil_div(p.d, 256) * 32;
    if constexpr (W != 2) {
        if (p.d > GRAD_HELD) {
            auto kernel = norm_grad_kernel<TX, TB, 0, W, FULL, true>;
            static DeviceOnce configured;
            constexpr int most = (FULL ? 4 : 2) * NORM_MOST * (int)sizeof(float);
            if (once_per_device(configured, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most); }) != cudaSuccess) return KGE_ERR_CUDA;
            return launch_status(launch_dependent(kernel, dim3((unsigned)ctas), dim3((unsigned)threads), (size_t)p.sums * threads * 8 * sizeof(float), s, p));
        }
    }
    switch (norm_team(p.d)) {
        case 8: return launch(norm_grad_kernel<TX, TB, 8, W, FULL, false>, NORM_THREADS);
        case 16: return launch(norm_grad_kernel<TX, TB, 16, W, FULL, false>, NORM_THREADS);
        case 32: return launch(norm_grad_kernel<TX, TB, 32, W, FULL, false>, NORM_THREADS);
        case 64: return launch(norm_grad_kernel<TX, TB, 64, W, FULL, false>, NORM_THREADS);
        case 128: return launch(norm_grad_kernel<TX, TB, 128, W, FULL, false>, NORM_THREADS);
        default: return launch(norm_grad_kernel<TX, TB, 0, W, FULL, false>, threads);
    }
}

// (rows that are not wide take the same teams, in the same order: the columns' sums are the same)
template <typename TX, typename TB>
int launch_norm_grad(const NormGradParams& p, int ctas, cudaStream_t s) {
    if (p.d > NORM_MOST)
        return launch_status(launch_dependent(norm_grad_loop_kernel<TX, TB>, dim3((unsigned)ctas), dim3(NORM_LOOP_THREADS), 0, s, p));
    // (pairs: 60,000 x 998 bf16 280 us, one by one 526; where the sums are in shared memory 64 registers do not hold them: 5,000 x 6,002 456 us, one by one 359)
    if (p.access == 2 && p.d <= GRAD_HELD) return launch_held<TX, TB, 2, true>(p, ctas, s);
    if (p.access < 8) return launch_held<TX, TB, 1, true>(p, ctas, s);
    return p.layer || p.b1 || p.sums > 2 ? launch_held<TX, TB, 8, true>(p, ctas, s) : launch_held<TX, TB, 8, false>(p, ctas, s);
}

}  // namespace
}  // namespace kge
