// One AdamW step over a list of tensors.
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps),  t = step + 1
// States in 32 bits, or in 8: m as e4m3, v as e5m2, with a power of two for each 128 elements of a tensor.  v moves by a thousandth of
// itself in a step, less than half the distance of two 8-bit values: rounded to nearest it would stand still.  Both states are
// rounded up or down with the probability that keeps them right on average, by counter-based numbers (four elements to a call of the
// generator, sixteen bits for each state), so a step is reproducible.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kge_eight.cuh"

namespace kge {

namespace {

constexpr int ADAM_THREADS = 256, ADAM_PER = 8;                        // elements per thread and turn
constexpr int ADAM_TURN = ADAM_THREADS * ADAM_PER;                     // elements of a CTA at a time
// Five CTAs an SM (48 registers); each takes one or two turns of one tensor, two where the CTAs of one turn each would not all run at a time (64 M elements with
// 8-bit states: 193 us with two turns, 198 with two on four CTAs an SM, 190 with one; a hundred tensors of 20 M, whose search for the tensor costs a CTA more: 71, 73, 80).
constexpr int ADAM_CTAS = 5, ADAM_SMS = 148;
constexpr int ADAM_BLOCK = 128;                                        // elements to a scale: the sixteen lanes of half a warp
static_assert(ADAM_BLOCK == 16 * ADAM_PER, "a block is half a warp's");

struct AdamTensor {
    void* p; const void* g; void *m, *v; float *ms, *vs; void* copy;
    int64_t n;
    float keep, decay;                // 1 - lr wd, and wd for a learning rate that is known on the device only
    uint8_t p_type, g_type, copy_type, vec;
    int32_t index;                    // its place in the caller's list
};

struct AdamCommon {
    float b1, o1, b2, o2, eps, grad_scale;
    float size, root;                 // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    double lr, log_b1, log_b2;
    uint64_t step;
    const int64_t* step_dev;
    const float *lr_dev, *grad_scale_dev;
    uint32_t key[20];
    int count, turns;
};

// A launch's tensors travel with its parameters: few with little to copy, many with what a launch may carry (13 small tensors: 5.7 us a step with room for 40, 9.2 with
// room for 340).
constexpr int ADAM_FEW = 12, ADAM_SOME = 40, ADAM_MANY = 340;
template <int CAP> struct AdamParams {
    AdamCommon c;
    uint32_t first[CAP + 1];          // first chunk of each tensor
    AdamTensor t[CAP];
};
static_assert(sizeof(AdamParams<ADAM_MANY>) <= 32764, "parameters of a launch");

struct AdamScalars { float size, root, keep, grad_scale; uint32_t c2, c3; };

// Four words for elements 4 group .. + 3 of the tensor.
__device__ __forceinline__ uint4 adam_words(const AdamCommon& c, uint64_t group, int index, const AdamScalars& s) {
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)index * 64u + (uint32_t)(group >> 32), c2 = s.c2, c3 = s.c3;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ c.key[2 * r]; c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ c.key[2 * r + 1]; c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}

template <typename T> __device__ __forceinline__ Raw8<T> get(const void* base, int64_t at, int valid, bool vec) {
    const T* p = static_cast<const T*>(base) + at;
    if (vec && valid == 8) return load_wide(p);
    Raw8<T> r = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < valid) set_element(r, e, p[e]);
    return r;
}
template <typename T> __device__ __forceinline__ void put(void* base, int64_t at, int valid, bool vec, const Raw8<T>& r) {
    T* p = static_cast<T*>(base) + at;
    if (vec && valid == 8) { store_wide(p, r); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < valid) p[e] = element(r, e);
}

// An e4m3 value is the half that the conversion instruction gives; an e5m2 value is a half without its low byte.
__device__ __forceinline__ F8 decode_m(const Raw8<uint8_t>& q, float scale) {
    F8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(q.w[i >> 1] >> (16 * (i & 1)))));
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        x.v[2 * i] = f.x * scale;
        x.v[2 * i + 1] = f.y * scale;
    }
    return x;
}
__device__ __forceinline__ F8 decode_v(const Raw8<uint8_t>& q, float scale) {
    F8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t h = __byte_perm(q.w[i >> 1], 0, i & 1 ? 0x3424 : 0x1404);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        x.v[2 * i] = f.x * scale;
        x.v[2 * i + 1] = f.y * scale;
    }
    return x;
}

// The scale of a block whose largest magnitude has the bits `most`: the power of two that puts it into the binade of exponent `top`,
// one below the type's last (a value rounded up may reach that).  1 for a block of zeros, NaN for one that holds an infinity or a
// NaN; `inv` is its reciprocal (0 for NaN: the block stands for NaN whatever its codes are).
struct BlockScale { float s, inv; };
__device__ __forceinline__ BlockScale block_scale(float largest, int top) {
    const uint32_t most = __float_as_uint(largest);
    const int e = max((int)(most >> 23) - top, 1);
    BlockScale b{__int_as_float(e << 23), __int_as_float((254 - e) << 23)};
    if (most == 0) b = {1.f, 1.f};
    if (most >= 0x7F800000u) b = {__int_as_float(0x7FC00000), 0.f};
    return b;
}
// |x| / scale times 2^(bias - 127) has the 8-bit type's exponent in the fp32 exponent field, its subnormal values being fp32's own; the
// bits below the type's last one are added to and cut off.  The code is the result's low byte.
template <int BITS, int BIAS> __device__ __forceinline__ uint32_t code_of(float x, float inv, uint32_t noise) {
    return (__float_as_uint((fabsf(x) * inv) * __int_as_float(BIAS << 23)) + noise) >> (23 - BITS);
}
// A half of a random word, and half a unit of it, below the last bit that stays.
template <int BITS, bool HIGH> __device__ __forceinline__ uint32_t noise_of(uint32_t word) {
    constexpr int UP = 23 - BITS - 16;
    return (HIGH ? (word >> (16 - UP)) & (0xFFFFu << UP) : (word << UP) & (0xFFFFu << UP)) | (1u << (UP - 1));
}
// Byte B of four words.
template <int B> __device__ __forceinline__ uint32_t four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    constexpr uint32_t PICK = B | (4 + B) << 4;
    return __byte_perm(__byte_perm(a, b, PICK), __byte_perm(c, d, PICK), 0x5410);
}
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float half_warp_max(float x) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
// Square root and reciprocal as one instruction each: within 2 units of 2^-24 both.
__device__ __forceinline__ float root_of(float x) { float r; asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float over(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

template <int BITS, typename TP, typename TG>
__device__ __forceinline__ void adam_chunk(const AdamCommon& c, const AdamTensor& t, const AdamScalars& s, int64_t from) {
    using TS = typename std::conditional<BITS == 32, float, uint8_t>::type;
#pragma unroll 1
    for (int turn = 0; turn < c.turns; ++turn) {
        const int64_t at = from + (turn * ADAM_THREADS + threadIdx.x) * ADAM_PER;
        const int valid = (int)max((int64_t)0, min((int64_t)8, t.n - at));
        if (BITS == 32 && valid == 0) return;
        if (BITS == 8 && from + turn * ADAM_THREADS * ADAM_PER + (int64_t)(threadIdx.x & ~31u) * ADAM_PER >= t.n) return;       // (a warp's lanes stay together)
        const bool vec = t.vec;
        const Raw8<TG> g8 = get<TG>(t.g, at, valid, vec);
        const Raw8<TS> m8 = get<TS>(t.m, at, valid, vec);
        const Raw8<TS> v8 = get<TS>(t.v, at, valid, vec);
        const Raw8<TP> p8 = get<TP>(t.p, at, valid, vec);
        F8 m, v;
        const int64_t block = at / ADAM_BLOCK;
        if constexpr (BITS == 8) {
            const float ms = valid ? t.ms[block] : 0.f, vs = valid ? t.vs[block] : 0.f;
            m = decode_m(m8, ms);
            v = decode_v(v8, vs);
        } else {
            m = wide_of(m8);
            v = wide_of(v8);
        }
        const F8 g = wide_of(g8);
        F8 p = wide_of(p8);
        // products and sums of the moments are rounded one by one: the 8-bit rounding below is a function of their last bits
        float most_m = 0.f, most_v = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = __fmul_rn(g.v[e], s.grad_scale);
            m.v[e] = __fadd_rn(__fmul_rn(m.v[e], c.b1), __fmul_rn(x, c.o1));
            v.v[e] = __fadd_rn(__fmul_rn(v.v[e], c.b2), __fmul_rn(__fmul_rn(x, x), c.o2));
            const float change = m.v[e] * over(fmaf(root_of(v.v[e]), s.root, c.eps));
            p.v[e] = fmaf(-s.size, change, p.v[e] * s.keep);
            if (BITS == 8) {
                most_m = max_nan(most_m, fabsf(m.v[e]));
                most_v = max_nan(most_v, fabsf(v.v[e]));
            }
        }
        if (valid) {
            put(t.p, at, valid, vec, narrow_of<TP>(p));
            if (t.copy && t.copy_type == KGE_BF16) put(t.copy, at, valid, vec, narrow_of<__nv_bfloat16>(p));
            if (t.copy && t.copy_type == KGE_F16) put(t.copy, at, valid, vec, narrow_of<__half>(p));
        }
        Raw8<TS> mn, vn;
        if constexpr (BITS == 32) {
            mn = narrow_of<float>(m);
            vn = narrow_of<float>(v);
        } else {
            const BlockScale sm = block_scale(half_warp_max(most_m), 7), sv = block_scale(half_warp_max(most_v), 14);
            if ((threadIdx.x & 15) == 0 && valid) { t.ms[block] = sm.s; t.vs[block] = sv.s; }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint4 words = adam_words(c, (uint64_t)at / 4 + k, t.index, s);
                const uint32_t w[4] = {words.x, words.y, words.z, words.w};
                uint32_t a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[i] = code_of<3, 7>(m.v[4 * k + i], sm.inv, noise_of<3, false>(w[i]));
                    // A positive v stays positive: with v = 0 beside an m that was rounded up the next step would be m / eps.
                    b[i] = max(code_of<2, 15>(v.v[4 * k + i], sv.inv, noise_of<2, true>(w[i])), min(__float_as_uint(v.v[4 * k + i]), 1u));
                }
                const uint32_t signs = four_bytes<3>(__float_as_uint(m.v[4 * k]), __float_as_uint(m.v[4 * k + 1]), __float_as_uint(m.v[4 * k + 2]), __float_as_uint(m.v[4 * k + 3]));
                mn.w[k] = (four_bytes<0>(a[0], a[1], a[2], a[3]) & 0x7F7F7F7Fu) | (signs & 0x80808080u);
                vn.w[k] = four_bytes<0>(b[0], b[1], b[2], b[3]);
            }
        }
        if (valid) {
            put(t.m, at, valid, vec, mn);
            put(t.v, at, valid, vec, vn);
        }
    }
}

template <int BITS, int CAP>
__global__ void __launch_bounds__(ADAM_THREADS, ADAM_CTAS) adamw_kernel(const __grid_constant__ AdamParams<CAP> q) {
    __shared__ AdamScalars shared;
    const AdamCommon& c = q.c;
    int i = 0;
    for (int hi = c.count; hi - i > 1;) {          // the tensor whose chunks hold this CTA's
        const int mid = (i + hi) / 2;
        if (q.first[mid] <= blockIdx.x) i = mid; else hi = mid;
    }
    const AdamTensor& t = q.t[i];
    AdamScalars s{c.size, c.root, t.keep, c.grad_scale, (uint32_t)c.step, (1u << 30) + (uint32_t)(c.step >> 32)};
    grid_dependency_wait();
    allow_dependents();
    if (c.step_dev || c.lr_dev || c.grad_scale_dev) {
        if (threadIdx.x == 0) {
            const uint64_t step = c.step + (c.step_dev ? (uint64_t)*c.step_dev : 0ull);
            const double lr = c.lr * (c.lr_dev ? (double)*c.lr_dev : 1.0), n = (double)step + 1.0;
            s.size = (float)(lr / -expm1(n * c.log_b1));
            s.root = (float)(1.0 / sqrt(-expm1(n * c.log_b2)));
            s.keep = (float)(1.0 - lr * (double)t.decay);
            if (c.grad_scale_dev) s.grad_scale *= *c.grad_scale_dev;
            s.c2 = (uint32_t)step;
            s.c3 = (1u << 30) + (uint32_t)(step >> 32);
            shared = s;
        }
        __syncthreads();
        s = shared;
    }
    const int64_t from = (int64_t)(blockIdx.x - q.first[i]) * (ADAM_TURN * c.turns);
    auto with_grad = [&](auto tp) {
        using TP = decltype(tp);
        if (t.g_type == KGE_F32) adam_chunk<BITS, TP, float>(c, t, s, from);
        else if (t.g_type == KGE_BF16) adam_chunk<BITS, TP, __nv_bfloat16>(c, t, s, from);
        else adam_chunk<BITS, TP, __half>(c, t, s, from);
    };
    if (t.p_type == KGE_F32) with_grad(float());
    else if (t.p_type == KGE_BF16) with_grad(__nv_bfloat16());
    else with_grad(__half());
}

bool fits(const void* p, int type_size) { return aligned_to(p, (size_t)std::min(32, 8 * type_size)); }

template <int BITS, int CAP>
int launch_adamw(AdamParams<CAP>& q, uint32_t chunks, cudaStream_t s) {
    return launch_status(launch_dependent(adamw_kernel<BITS, CAP>, dim3(chunks), dim3(ADAM_THREADS), 0, s, q));
}

// Launches for all tensors from *at on that one launch carries.
template <int CAP>
int adamw_part(const kge_adamw_tensor* tensors, int32_t count, int32_t* at, int32_t bits, double lr, const AdamCommon& common, cudaStream_t s) {
    AdamParams<CAP> q;
    q.c = common;
    int64_t chunks = 0;
    int k = 0;
    for (; *at < count && k < CAP; ++*at) {
        const kge_adamw_tensor& t = tensors[*at];
        if (t.n == 0 || !t.grad) continue;
        const int64_t more = ceil_div(t.n, ADAM_TURN * common.turns);
        if (chunks + more > INT32_MAX) break;
        AdamTensor& d = q.t[k];
        const int ps = type_bytes(t.param_type), gs = type_bytes(t.grad_type), ss = bits == 32 ? 4 : 1;
        d.p = t.param; d.g = t.grad; d.m = t.m; d.v = t.v; d.ms = t.m_scales; d.vs = t.v_scales; d.copy = t.copy; d.n = t.n;
        d.keep = (float)(1.0 - lr * (double)t.weight_decay); d.decay = t.weight_decay;
        d.p_type = (uint8_t)t.param_type; d.g_type = (uint8_t)t.grad_type; d.copy_type = (uint8_t)t.copy_type; d.index = *at;
        d.vec = fits(t.param, ps) && fits(t.grad, gs) && fits(t.m, ss) && fits(t.v, ss) && (!t.copy || fits(t.copy, 2));
        q.first[k++] = (uint32_t)chunks;
        chunks += more;
    }
    if (k == 0) return KGE_OK;
    q.first[k] = (uint32_t)chunks;
    q.c.count = k;
    return bits == 32 ? launch_adamw<32, CAP>(q, (uint32_t)chunks, s) : launch_adamw<8, CAP>(q, (uint32_t)chunks, s);
}

}  // namespace
}  // namespace kge

using namespace kge;

extern "C" int kge_adamw(const kge_adamw_tensor* tensors, int32_t count, int32_t state_bits, double lr, double beta1, double beta2, double eps,
                         double grad_scale, uint64_t step, const int64_t* step_dev, const float* lr_dev, const float* grad_scale_dev, uint64_t seed,
                         void* stream) {
    if (count < 0 || count > (1 << 26) || (count && !tensors) || (state_bits != 32 && state_bits != 8) || !std::isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) ||
        !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps >= 1.17549435e-38f) || !std::isfinite((float)eps) || !std::isfinite((float)grad_scale) || step >= 1ull << 62 || !aligned_to(step_dev, 8) ||
        !aligned_to(lr_dev, 4) || !aligned_to(grad_scale_dev, 4)) return KGE_ERR_BAD_ARG;
    int live = 0;
    int64_t turns = 0;
    for (int32_t i = 0; i < count; ++i) {
        const kge_adamw_tensor& t = tensors[i];
        if (t.n < 0 || !is_float_type(t.param_type) || !is_float_type(t.grad_type) || !std::isfinite(t.weight_decay)) return KGE_ERR_BAD_ARG;
        if (t.copy && t.copy_type != KGE_BF16 && t.copy_type != KGE_F16) return KGE_ERR_BAD_ARG;
        if (t.n > (1ll << 40)) return KGE_ERR_UNSUPPORTED;
        if (t.n == 0 || !t.grad) continue;
        const int ss = state_bits == 32 ? 4 : 1;
        if (!t.param || !t.m || !t.v || !aligned_to(t.param, type_bytes(t.param_type)) || !aligned_to(t.grad, type_bytes(t.grad_type)) || !aligned_to(t.m, ss) ||
            !aligned_to(t.v, ss) || (t.copy && !aligned_to(t.copy, 2))) return KGE_ERR_BAD_ARG;
        if (state_bits == 8 && (!t.m_scales || !t.v_scales || !aligned_to(t.m_scales, 4) || !aligned_to(t.v_scales, 4))) return KGE_ERR_BAD_ARG;
        ++live;
        turns += ceil_div(t.n, ADAM_TURN);
    }
    AdamCommon c{};
    c.b1 = (float)beta1; c.o1 = (float)(1.0 - beta1); c.b2 = (float)beta2; c.o2 = (float)(1.0 - beta2);
    c.eps = (float)eps; c.grad_scale = (float)grad_scale;
    c.lr = lr; c.log_b1 = std::log(beta1); c.log_b2 = std::log(beta2);
    const double n = (double)step + 1.0;
    c.size = (float)(lr / -std::expm1(n * c.log_b1));
    c.root = (float)(1.0 / std::sqrt(-std::expm1(n * c.log_b2)));
    c.turns = turns > ADAM_SMS * ADAM_CTAS ? 2 : 1;
    c.step = step; c.step_dev = step_dev; c.lr_dev = lr_dev; c.grad_scale_dev = grad_scale_dev;
    for (uint32_t r = 0; r < 10; ++r) { c.key[2 * r] = (uint32_t)seed + r * 0x9E3779B9u; c.key[2 * r + 1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u; }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    for (int32_t at = 0; at < count && live > 0;) {
        const int rc = live <= ADAM_FEW    ? adamw_part<ADAM_FEW>(tensors, count, &at, state_bits, lr, c, s)
                       : live <= ADAM_SOME ? adamw_part<ADAM_SOME>(tensors, count, &at, state_bits, lr, c, s)
                                           : adamw_part<ADAM_MANY>(tensors, count, &at, state_bits, lr, c, s);
        if (rc != KGE_OK) return rc;
    }
    return KGE_OK;
}
