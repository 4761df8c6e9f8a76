// The norms after and before a block, fused with its gate and residual scale:
//   a = N1(y) (or y),  h = x + s act(g) a,  z = N2(h);   N(u) = (u - mu) r w + b,  r = 1 / sqrt(mean((u - mu)^2) + eps),  mu = mean(u), or 0
// h is rounded once, when it is stored; z is made of the unrounded one.  z may leave as 8-bit integers with a scale for each row.
#pragma once

#include <algorithm>

#include "kge_int8.cuh"
#include "kge_norm.cuh"

namespace kge {

struct NormParams {
    const void *x, *y, *gate;
    void *h, *z;
    const float *w1, *b1, *scale, *w2, *b2;
    float *stats, *z_scales;
    int64_t ldx, ldy, ldg, ldh, ldz;
    int n, d;
    int post, layer, act, z8;          // act is looked at where a gate is given
    int access;                        // elements that move as one access in every array: 8 (rows start at multiples of eight, vectors at multiples of four), 2 or 1
    float eps, inv_d;
};

// Launches the kernel for fp32, bf16 or fp16 rows of x (each in a source of its own, so that they are compiled side by side).
int launch_norm_f32(const NormParams& p, int block_type, cudaStream_t s);
int launch_norm_bf16(const NormParams& p, int block_type, cudaStream_t s);
int launch_norm_f16(const NormParams& p, int block_type, cudaStream_t s);

namespace {

__device__ __forceinline__ float deviation(const NormParams& p, float squares) { return rsqrtf(fmaf(squares, p.inv_d, p.eps)); }

// Takes the mean out of a team's row; returns it and the reciprocal deviation.  Two passes over the registers: a mean far from zero does not eat the deviation's digits.
template <bool LAYER, int L, int K, int W>
__device__ __forceinline__ float2 centre(const NormParams& p, Team<L>& team, P8 (&u)[K], const Place<W> (&at)[K]) {
    float mu = 0.f, sq = 0.f;
    if (LAYER) {
#pragma unroll
        for (int k = 0; k < K; ++k) mu += at[k].total(u[k]);
        mu = team.sum(mu) * p.inv_d;
#pragma unroll
        for (int k = 0; k < K; ++k) u[k] = at[k].there(u[k] + -mu);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) sq += at[k].dot(u[k], u[k]);
    return make_float2(mu, deviation(p, team.sum(sq)));
}

// (z is off by its own roundings: what the product with 1 / s adds to them moves an integer only where they do)
template <int W>
__device__ __forceinline__ void store_z8(int8_t* out, const Place<W>& at, const P8& z, const RowScale& s) {
    const uint2 w = round_products(singles_of(z), s.inv);
    if constexpr (W == 8) {
        if (at.any) *reinterpret_cast<uint2*>(at.mine(out)) = w;
    } else if constexpr (W == 2) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) if (at.holds(e)) *reinterpret_cast<uint16_t*>(at.mine(out, e)) = (uint16_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (at.holds(e)) *at.mine(out, e) = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
    }
}

// A team of L threads (L = 0: the CTA) holds a row, K packs of eight elements to a thread: the row's addresses, sums and scalars are shared out over up to 32
// elements a thread (32,768 x 4,096 bf16 with a thread for eight elements: 53 instructions an element, so 26).  Narrow rows take one pack a thread instead, the next row's
// loads under way: few rows are in an SM's hands then, and it waits for them (24,576 x 200: 16.3 us with two packs, 14.2).
constexpr int norm_threads(int l, int k, bool wide) { return l == 0 && !wide && k > 1 ? 2 * NORM_THREADS : NORM_THREADS; }
// CTAs on an SM, and so registers a thread; rows that are only normalised (Y = false) need few.
constexpr int norm_ctas(int l, int k, bool wide, int x_bytes, int block_bytes, bool y) {
    if (!y && (wide || l > 0 || k == 1)) return k == 1 || (x_bytes == 2 && wide) ? 4 : (k == 2 ? 3 : 2);
    if (l == 0 && !wide && k > 1) return 1;
    return (k == 1 || (k == 2 && wide && x_bytes + block_bytes <= 6) ? 3 : (k > 2 && x_bytes + block_bytes > 6 ? 1 : 2));
}
// Threads that the registers are made out for: where one CTA's are 64 to 256, 384, for 168 registers a thread and as many CTAs as that allows (16,384 x 4,096 fp32 with a
// gate: 205 us, with 200 registers 281).
constexpr int norm_bound(int l, int k, bool wide, int x_bytes, int block_bytes, bool y) {
    return l == 0 && wide && norm_ctas(l, k, wide, x_bytes, block_bytes, y) == 1 ? NORM_THREADS * 3 / 2 : norm_threads(l, k, wide);
}
template <typename TX, typename TB, int L, int K, int W, bool LAYER, bool Y>
__global__ void __launch_bounds__(norm_bound(L, K, W == 8, sizeof(TX), sizeof(TB), Y), norm_ctas(L, K, W == 8, sizeof(TX), sizeof(TB), Y)) norm_kernel(const __grid_constant__ NormParams p) {
    constexpr bool AHEAD = K == 1, BRIEF = sizeof(TX) + sizeof(TB) == 4;
    __shared__ float parts[2][2][32];
    Team<L> team(parts);
    const int t = team.thread;
    Place<W> at[K];
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] = Place<W>(Team<L>::size(), t, k, p.d);
    grid_dependency_wait();
    allow_dependents();
    struct Row { Raw8<TX> x[K]; Raw8<TB> y[K], gate[K]; };
    auto load = [&](int64_t row, Row& v) {
        // (a team that has run out of rows goes along with the last one)
        const int64_t r = L == 0 ? row : min(row, (int64_t)p.n - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) v.x[k] = at[k].load(static_cast<const TX*>(p.x) + r * p.ldx);
        if (Y) {
#pragma unroll
            for (int k = 0; k < K; ++k) v.y[k] = at[k].load(static_cast<const TB*>(p.y) + r * p.ldy);
            if (p.gate) {
#pragma unroll
                for (int k = 0; k < K; ++k) v.gate[k] = at[k].load(static_cast<const TB*>(p.gate) + r * p.ldg);
            }
        }
    };
    const int64_t step = (int64_t)gridDim.x * Team<L>::COUNT;
    Row next;
    if (AHEAD) load((int64_t)blockIdx.x * Team<L>::COUNT + team.index, next);
    for (int64_t r0 = (int64_t)blockIdx.x * Team<L>::COUNT; r0 < p.n; r0 += step) {
        const int64_t mine = r0 + team.index, r = L == 0 ? mine : min(mine, (int64_t)p.n - 1);
        const bool live = L == 0 || mine < p.n;
        float* const stats = p.stats && live && t == 0 ? p.stats + 4 * r : nullptr;
        P8 u[K];
        float2 s = make_float2(0.f, 0.f);
        {
            Row now;
            if (AHEAD) {
                now = next;
                if (r0 + step < p.n) load(mine + step, next);
            } else load(mine, now);
            if (Y) {
#pragma unroll
                for (int k = 0; k < K; ++k) u[k] = pairs_of(now.y[k]);
                if (p.post) {
                    s = centre<LAYER>(p, team, u, at);
#pragma unroll
                    for (int k = 0; k < K; ++k) u[k] = u[k] * s.y * at[k].vector(p.w1);
                    if (p.b1) {
#pragma unroll
                        for (int k = 0; k < K; ++k) u[k] = u[k] + at[k].vector(p.b1);
                    }
                }
                if (p.gate) {
                    if (p.act == NORM_PLAIN) {
#pragma unroll
                        for (int k = 0; k < K; ++k) u[k] = u[k] * pairs_of(now.gate[k]);
                    } else {
                        with_sigmoids<BRIEF>(now.gate, [&](int k, const P8& act) { u[k] = u[k] * act; });
                        if (p.act == NORM_SILU) {
#pragma unroll
                            for (int k = 0; k < K; ++k) u[k] = u[k] * pairs_of(now.gate[k]);
                        }
                    }
                }
                if (p.scale) {
#pragma unroll
                    for (int k = 0; k < K; ++k) u[k] = fma8(u[k], at[k].vector(p.scale), pairs_of(now.x[k]));
                } else {
#pragma unroll
                    for (int k = 0; k < K; ++k) u[k] = u[k] + pairs_of(now.x[k]);
                }
                if (p.h) {
                    TX* const hs = static_cast<TX*>(p.h) + r * p.ldh;
#pragma unroll
                    for (int k = 0; k < K; ++k) at[k].store(hs, u[k], live);
                }
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) u[k] = pairs_of(now.x[k]);
            }
        }
        if (stats) *reinterpret_cast<float2*>(stats) = s;
        s = make_float2(0.f, 0.f);
        if (p.z) {
            s = centre<LAYER>(p, team, u, at);
#pragma unroll
            for (int k = 0; k < K; ++k) u[k] = u[k] * s.y * at[k].vector(p.w2);
            if (p.b2) {
#pragma unroll
                for (int k = 0; k < K; ++k) u[k] = u[k] + at[k].vector(p.b2);
            }
            if (p.z8) {
                float most = 0.f;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (W < 8 || at[k].any) most = Team<L>::template join<true>(most, fabsf(element(u[k], e)));
                const RowScale q = row_scale(team.most(most));
                if (live) {
                    if (t == 0) p.z_scales[r] = q.s;
#pragma unroll
                    for (int k = 0; k < K; ++k) store_z8(static_cast<int8_t*>(p.z) + r * p.ldz, at[k], u[k], q);
                }
            } else {
                TB* const zs = static_cast<TB*>(p.z) + r * p.ldz;
#pragma unroll
                for (int k = 0; k < K; ++k) at[k].store(zs, u[k], live);
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
            if (p.gate) a *= act_of<sizeof(TX) + sizeof(TB) == 4>(to_float(gate[i]), p.act);
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
template <typename TX, typename TB, int L, int K, int W, bool Y>
int launch_rows(const NormParams& p, int threads, int sms, cudaStream_t s) {
    constexpr bool WIDE = W == 8;
    constexpr int ctas = norm_ctas(L, K, WIDE, sizeof(TX), sizeof(TB), Y), regs = ctas == 1 ? (WIDE ? (L == 0 ? 168 : 240) : 128) : 65536 / (ctas * NORM_THREADS) / 8 * 8;          // (at most)
    const int64_t all = ceil_div(p.n, Team<L>::COUNT), room = (int64_t)sms * std::max(1, 65536 / (regs * threads)), turns = ceil_div(all, room);
    const dim3 grid((unsigned)ceil_div(all, turns)), block((unsigned)threads);
    return launch_status(p.layer ? launch_dependent(norm_kernel<TX, TB, L, K, W, true, Y>, grid, block, 0, s, p)
                                 : launch_dependent(norm_kernel<TX, TB, L, K, W, false, Y>, grid, block, 0, s, p));
}

template <typename TX, typename TB, bool Y>
int launch_wide(const NormParams& p, int sms, cudaStream_t s) {
    const int d = p.d, cta = (int)ceil_div(d, 1024) * 32;          // threads of a CTA that holds a row, 32 elements each
    if (d <= 64) return launch_rows<TX, TB, 8, 1, 8, Y>(p, NORM_THREADS, sms, s);
    if (d <= 128) return launch_rows<TX, TB, 16, 1, 8, Y>(p, NORM_THREADS, sms, s);
    if (d <= 256) return launch_rows<TX, TB, 32, 1, 8, Y>(p, NORM_THREADS, sms, s);
    if (d <= 512) return launch_rows<TX, TB, 32, 2, 8, Y>(p, NORM_THREADS, sms, s);
    if (d <= 768) return launch_rows<TX, TB, 32, 3, 8, Y>(p, NORM_THREADS, sms, s);
    if (d <= 1024) return launch_rows<TX, TB, 32, 4, 8, Y>(p, NORM_THREADS, sms, s);
    return d <= 24 * cta ? launch_rows<TX, TB, 0, 3, 8, Y>(p, cta, sms, s) : launch_rows<TX, TB, 0, 4, 8, Y>(p, cta, sms, s);
}

template <typename TX, typename TB>
int launch_norm(const NormParams& p, cudaStream_t s) {
    int sms = 0;
    const int rc = sm_count(&sms), d = p.d;
    if (rc != KGE_OK) return rc;
    if (d > NORM_MOST) return launch_status(launch_dependent(norm_loop_kernel<TX, TB>, dim3((unsigned)p.n), dim3(NORM_LOOP_THREADS), 0, s, p));
    if (p.access == 8) return p.y ? launch_wide<TX, TB, true>(p, sms, s) : launch_wide<TX, TB, false>(p, sms, s);
    auto rows = [&](auto y, auto access) {
        constexpr bool Y = decltype(y)::value;
        constexpr int W = decltype(access)::value;
        if (d <= 64) return launch_rows<TX, TB, 8, 1, W, Y>(p, NORM_THREADS, sms, s);
        if (d <= 256) return launch_rows<TX, TB, 32, 1, W, Y>(p, NORM_THREADS, sms, s);
        if (d <= 2048) return launch_rows<TX, TB, 0, 1, W, Y>(p, (int)ceil_div(d, 256) * 32, sms, s);
        return launch_rows<TX, TB, 0, 2, W, Y>(p, (int)ceil_div(d, 512) * 32, sms, s);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    // (60,000 x 998 bf16 136 us, one by one 227; 9,811 x 7,694 256 and 430)
    if (p.access == 2) return p.y ? rows(std::true_type(), Two()) : rows(std::false_type(), Two());
    return p.y ? rows(std::true_type(), One()) : rows(std::false_type(), One());
}

}  // namespace
}  // namespace kge
