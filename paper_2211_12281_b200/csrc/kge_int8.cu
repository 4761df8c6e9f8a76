// 8-bit integers with a scale for each row: making such operands, and their product.
//   quantise   s = amax / 127, q = the integer nearest to x / s
//   product    C[m, n] = sA[m] sB[n] sum_k A[m, k] B[n, k]   (+ C0[m, n])
// The sum is exact: 32-bit integers hold 131,071 products of 8-bit ones, so neither the order of k nor how many CTAs share it matters.
#include <algorithm>

#include "kge_int8.cuh"
#include "kge_product.cuh"

namespace kge {

namespace {

// ---- quantisation ----------------------------------------------------------------------------------------------------

struct QuantParams {
    const void* x; int64_t ldx;
    int8_t* q; int64_t ldq;
    float* scales;
    int rows, cols;
    int wide;                        // rows of x start at multiples of eight elements and have a whole number of eights
};

// Magnitudes as integers, which order as they do (a NaN above all).
__device__ __forceinline__ uint32_t most_of(const Raw8<float>& r) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, r.w[e] & 0x7FFFFFFFu);
    return m;
}
template <typename T> __device__ __forceinline__ uint32_t most_of(const Raw8<T>& r) {
    uint32_t m = r.w[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __vmaxu2(m, r.w[i] & 0x7FFF7FFFu);
    return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ float magnitude(uint32_t m, float) { return __uint_as_float(m); }
__device__ __forceinline__ float magnitude(uint32_t m, __nv_bfloat16) { return __uint_as_float(m << 16); }
__device__ __forceinline__ float magnitude(uint32_t m, __half) { return __half2float(__ushort_as_half((unsigned short)m)); }

// The integer stored is the one nearest to the true quotient x / s, ties to even, not to what x (1 / s) rounds to, which is within 2^-23 of it.
//   16-bit x    with a the row's largest value, x / a times 127 is k + 1/2 exactly, or off it by 2^-19 at least (254 x and (2 k + 1) a differ by
//               one unit then, of numbers of 19 bits).  In the first case the true quotient lies on the side that the rounding of s = a / 127
//               says: `inv` leans by 2^-21 to it.  Where s is exact the quotient is the middle itself: right if 1 / s is exact too, else decided
//               one by one.
//   fp32 x      products beside a middle (within 2^-12) are decided one by one.
// One by one: m, the multiple of 16 units next to |x| (1 / s) (all middles are such), is compared with the quotient exactly, by the sign of |x| - m s.
struct QuantScale { float s, inv; bool each; };
template <typename T> __device__ __forceinline__ QuantScale quant_scale(float a) {
    const RowScale r = row_scale(a);
    QuantScale q{r.s, r.inv, false};
    if (sizeof(T) == 2 && r.s > 1.17549435e-38f && a > 0.f) {          // (the smallest scale is a power of two and not a / 127)
        const float e = fmaf(-r.s, 127.f, a);
        q.each = e == 0.f && fmaf(r.s, r.inv, -1.f) != 0.f;
        q.inv = e == 0.f ? r.inv : fmaf(r.inv, e > 0.f ? 4.76837158e-7f : -4.76837158e-7f, r.inv);
    }
    return q;
}
__device__ __noinline__ uint32_t quotient_bits(float x, float s) {
    int m = (int)(__float_as_uint(fabsf(x) * __fdiv_rn(1.f, s)) + 8u) & ~15;
    const float up = s < 2.35098870e-38f ? 2.f : 1.f;          // (half a unit of 2^-149, of scales below 2^-125, is none)
    const float d = fmaf(-__int_as_float(m), up * s, up * fabsf(x));
    m += d > 0.f ? 1 : (d < 0.f ? -1 : 0);
    return __float_as_uint(copysignf(__int_as_float(m), x) + ROUND_TO_INT);
}
template <typename T> __device__ __forceinline__ uint2 quantized(const Raw8<T>& r, const QuantScale& s) {
    const F8 x = wide_of(r);
    F8 t = make8([&](int e) { return fmaf(x.v[e], s.inv, ROUND_TO_INT); });
    bool each = s.each;
    if (sizeof(T) == 4) {
        float far = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) far = fmaxf(far, fabsf(fmaf(x.v[e], s.inv, ROUND_TO_INT - t.v[e])));          // how far the product is from its integer
        each = far > 0.5f - 0.000244140625f;
    }
    if (each) t = make8([&](int e) { return __uint_as_float(quotient_bits(x.v[e], s.s)); });
    return low_bytes(t);
}

// A row to a warp (L = 32) or to a CTA (L = 0); a thread holds K packs of eight of it.
constexpr int QUANT_THREADS = 256;
template <typename T, int L, int K, bool WIDE>
__global__ void __launch_bounds__(QUANT_THREADS) int8_rows_kernel(const __grid_constant__ QuantParams p) {
    __shared__ uint32_t part[QUANT_THREADS / 32];
    const int team = L == 32 ? 32 : QUANT_THREADS, t = (int)threadIdx.x % (L == 32 ? 32 : QUANT_THREADS);
    const int64_t r = L == 32 ? (int64_t)blockIdx.x * (QUANT_THREADS / 32) + __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0) : (int64_t)blockIdx.x;
    grid_dependency_wait();
    allow_dependents();
    if (r >= p.rows) return;
    const T* const x = static_cast<const T*>(p.x) + r * p.ldx;
    int8_t* const out = p.q + r * p.ldq;
    auto load = [&](int64_t c) {
        Raw8<T> v = {};
        if (WIDE) { if (c < p.cols) v = load_wide(x + c); }
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < p.cols) set_element(v, e, x[c + e]);
        }
        return v;
    };
    auto store = [&](int64_t c, const Raw8<T>& v, const QuantScale& s) {
        if (c >= p.cols) return;
        const uint2 w = quantized(v, s);
        if (WIDE || c + 8 <= p.cols) *reinterpret_cast<uint2*>(out + c) = w;
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < p.cols) out[c + e] = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
        }
    };
    Raw8<T> held[K];
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) held[k] = load((k * team + t) * 8);
#pragma unroll
    for (int k = 0; k < K; ++k) m = max(m, most_of(held[k]));
    for (int64_t c = (int64_t)K * team * 8 + t * 8; c < p.cols; c += team * 8) m = max(m, most_of(load(c)));
    m = __reduce_max_sync(0xffffffffu, m);
    if (L == 0) {
        if ((t & 31) == 0) part[t >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < QUANT_THREADS / 32; ++w) m = max(m, part[w]);
    }
    const QuantScale s = quant_scale<T>(magnitude(m, T()));
    if (t == 0) p.scales[r] = s.s;
#pragma unroll
    for (int k = 0; k < K; ++k) store((k * team + t) * 8, held[k], s);
    for (int64_t c = (int64_t)K * team * 8 + t * 8; c < p.cols; c += team * 8) store(c, load(c), s);
}

template <typename T, bool WIDE>
int launch_quantize(const QuantParams& p, cudaStream_t s) {
    auto launch = [&](auto kernel, int64_t ctas) { return launch_status(launch_dependent(kernel, dim3((unsigned)ctas), dim3(QUANT_THREADS), 0, s, p)); };
    const int64_t by_eight = ceil_div(p.rows, QUANT_THREADS / 32);
    if (p.cols <= 256) return launch(int8_rows_kernel<T, 32, 1, WIDE>, by_eight);
    if (p.cols <= 512) return launch(int8_rows_kernel<T, 32, 2, WIDE>, by_eight);
    if (p.cols <= 768) return launch(int8_rows_kernel<T, 32, 3, WIDE>, by_eight);
    if (p.cols <= 1024) return launch(int8_rows_kernel<T, 32, 4, WIDE>, by_eight);
    if (p.cols <= 2048) return launch(int8_rows_kernel<T, 0, 1, WIDE>, p.rows);
    if (p.cols <= 4096) return launch(int8_rows_kernel<T, 0, 2, WIDE>, p.rows);
    return launch(int8_rows_kernel<T, 0, 4, WIDE>, p.rows);          // (what is beyond 8,192 columns is read again)
}

// ---- product ---------------------------------------------------------------------------------------------------------

constexpr int I8_BM = 128;
constexpr uint32_t I8_BOX_BYTES = 128 * OPERAND_BK;
constexpr int I8_NACC = 2;                                // accumulators in tensor memory: one is stored while the other is summed up
// Five forms of the kernel: tiles of 256 x 256 that a pair of CTAs shares, 128 rows and half of B's rows each; tiles of 128 x 128, two CTAs an SM (one loads and
// multiplies while the other stores) or one with three times the copies under way; tiles of 128 x 64, three CTAs an SM; tiles of 128 x 128 whose K a cluster shares,
// where tiles are few.
enum { I8_TWO = 0, I8_PAIR = 1, I8_NARROW = 2, I8_SPLIT = 3, I8_DEEP = 4 };
constexpr int I8_MAX_SPLIT = 8;           // CTAs that share a tile's K
__host__ __device__ constexpr int i8_bn(int form) { return form == I8_TWO ? 256 : (form == I8_NARROW ? 64 : 128); }
__host__ __device__ constexpr int i8_box_rows(int form) { return form == I8_NARROW ? 64 : 128; }             // of B per copy and CTA
__host__ __device__ constexpr int i8_stages(int form) { return form == I8_PAIR || form == I8_NARROW ? 2 : 6; }
__host__ __device__ constexpr int i8_epi_warps(int form) { return form == I8_NARROW ? 4 : 8; }
__host__ __device__ constexpr int i8_groups(int form) { return i8_bn(form) / OUT_COLS * 4 / i8_epi_warps(form); }     // of 64 columns per epilogue warp
__host__ __device__ constexpr int i8_threads(int form) { return 32 * (4 + i8_epi_warps(form)); }     // (four more: copies, MMAs, two idle)
__host__ __device__ constexpr int i8_ctas_per_sm(int form) { return form == I8_PAIR ? 2 : (form == I8_NARROW ? 3 : 1); }
__host__ __device__ constexpr uint32_t i8_stage_bytes(int form) { return I8_BOX_BYTES + (uint32_t)i8_box_rows(form) * OPERAND_BK; }
constexpr uint32_t I8_STORE_ROW = 128;                    // bytes of a row on their way to memory, per epilogue warp and turn
__host__ __device__ constexpr size_t i8_smem_bytes(int form) {
    return (size_t)i8_stages(form) * i8_stage_bytes(form) + i8_epi_warps(form) * (32 * I8_STORE_ROW + OUT_COLS * 4) + 256;
}

struct IntProductParams : ProductOut {
    int kblocks, kper;                    // blocks of K in all, and per CTA of a cluster
    int tiles_n, items;
    const float *sa, *sb;
    int32_t* status; int wait_limit;
    uint32_t idesc;
};

// Instruction descriptor: D int32, A and B signed 8-bit integers, both K-major.
constexpr uint32_t i8_idesc(int m, int n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }
__device__ __forceinline__ void i8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void i8_mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// A sum times its two scales (the sum's own rounding to fp32 is half a step of 24 bits), and the addend with the second of them, in an order that the two scales alone
// decide and in operations that the compiler may not join, so that an element has the same bits in every form of the kernel and whatever its neighbours are.  Scales of
// magnitudes between 2^-63 and 2^63 are multiplied one after the other: no intermediate value leaves the normal numbers.  Others too, the smaller one first: |x| >= 1 keeps
// that product a normal number where the scale is one, and it leaves the range upwards only where the result does.
__device__ __forceinline__ bool near_one(float s) { return (__float_as_uint(s) & 0x7FFFFFFFu) - 0x20000000u <= 0x3F000000u; }
template <bool NEAR> __device__ __forceinline__ float scaled(int x, float a, float b, bool add, float addend) {
    const bool swap = !NEAR && !(near_one(a) && near_one(b)) && fabsf(b) < fabsf(a);
    const float y = __fmul_rn((float)x, swap ? b : a), last = swap ? a : b;
    return add ? __fmaf_rn(y, last, addend) : __fmul_rn(y, last);
}

// 128 bytes of each of a warp's rows from shared memory in units of one or two elements, sixteen of them under way (15,348 x 3,109 f16 in 8 bits, K = 279: 85 us with
// four under way, 45; 13,555 x 1,119 bf16, K = 2,536: 54 and 47).
template <typename TO, typename U> __device__ __forceinline__ void out_units(const ProductOut& p, int row0, int col0, const float4* st, int lane) {
    constexpr int V = 16 / sizeof(U), COLS = 128 / (int)sizeof(U) / 32, ROWS = 16 / COLS, E = (int)(sizeof(U) / sizeof(TO));
    const U* const own = reinterpret_cast<const U*>(st);
#pragma unroll 1
    for (int r0 = 0; r0 < 32; r0 += ROWS) {
        U v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = i / COLS, x = i % COLS * 32 + lane;
            v[i] = own[((r0 + r) * 8 + ((x / V) ^ (r & 7))) * V + x % V];
        }
        TO* const dst = static_cast<TO*>(p.out) + (row0 + r0) * p.ld_out + col0 + lane * E;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (row0 + r0 + i / COLS < p.M && col0 + (i % COLS * 32 + lane) * E < p.N) *reinterpret_cast<U*>(dst + i / COLS * p.ld_out + i % COLS * 32 * E) = v[i];
    }
}

// A warp's 32 rows x 64 columns: 128 bytes of each row at a time from tensor memory through shared memory, so that a store instruction covers whole lines.  The
// next sixteen columns' sums are on their way while sixteen are scaled.
template <typename TO, bool NEAR, bool ADD, class F>
__device__ __forceinline__ void i8_store(const IntProductParams& p, int row0, int col0, uint32_t from, float sa, const float* sb, float4* st, int lane, F&& read_all) {
    constexpr int V = 16 / sizeof(TO), PASS = 128 / sizeof(TO);
    const bool inside = p.vec && row0 + 32 <= p.M && col0 + OUT_COLS <= p.N;
    uint32_t v[2][16];
    tmem_ld16(from, v[0]);
#pragma unroll
    for (int c = 0; c < OUT_COLS; c += PASS) {
        if (ADD) {
            if (c > 0) out_fetch_addend<TO>(p, row0, col0, c, st, lane);
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
        }
#pragma unroll
        for (int h = 0; h < PASS; h += 16) {
            const int at16 = (c + h) / 16;
            tmem_wait16(v[at16 & 1]);
            uint32_t x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = v[at16 & 1][i];
            if (at16 + 1 < OUT_COLS / 16) tmem_ld16(from + 16 * (at16 + 1), v[(at16 + 1) & 1]);
            else read_all();
#pragma unroll
            for (int i = 0; i < 16 / V; ++i) {
                float4* const at = st + lane * 8 + ((h / V + i) ^ (lane & 7));
                Pack<TO, V> o;
                if (ADD) o = *reinterpret_cast<const Pack<TO, V>*>(at);
                float y[V];
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    const float4 b = *reinterpret_cast<const float4*>(sb + c + h + i * V + e);
                    const float bs[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int sum = (int)x[i * V + e + k];
                        y[e + k] = scaled<NEAR>(sum, sa, bs[k], ADD, ADD ? to_float(o.v[e + k]) : 0.f);
                    }
                }
                if constexpr (sizeof(TO) == 4) {
#pragma unroll
                    for (int e = 0; e < V; ++e) o.v[e] = y[e];
                } else {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        if constexpr (std::is_same<TO, __nv_bfloat16>::value) *reinterpret_cast<__nv_bfloat162*>(&o.v[e]) = __floats2bfloat162_rn(y[e], y[e + 1]);
                        else *reinterpret_cast<__half2*>(&o.v[e]) = __floats2half2_rn(y[e], y[e + 1]);
                    }
                }
                *at = *reinterpret_cast<const float4*>(&o);
            }
        }
        __syncwarp();
        if (inside) {
            const int r0 = lane / 8, unit = lane % 8;
            TO* dst = static_cast<TO*>(p.out) + (row0 + r0) * p.ld_out + col0 + c + V * unit;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = j * 4 + r0;
                *reinterpret_cast<float4*>(dst) = st[r * 8 + (unit ^ (r & 7))];
                dst += 4 * p.ld_out;
            }
        } else if (sizeof(TO) == 2 && p.twos) {
            out_units<TO, uint32_t>(p, row0, col0 + c, st, lane);
        } else {
            out_units<TO, TO>(p, row0, col0 + c, st, lane);
        }
        __syncwarp();
    }
}

// A cluster's CTAs hold partial sums of one tile in their shared memory; each adds up a share of it.
template <typename TO>
__device__ __forceinline__ void i8_join(const IntProductParams& p, uint32_t part, int m0, int n0, int tid) {
    const int rows = min(I8_BM, (int)p.M - m0);
    const uint32_t size = cluster_size();
    constexpr int THREADS = 32 * i8_epi_warps(I8_SPLIT), PER_ROW = i8_bn(I8_SPLIT) / 4;
    for (int u = (int)cluster_rank() * THREADS + tid; u < rows * PER_ROW; u += (int)size * THREADS) {
        const int r = u / PER_ROW, q = u % PER_ROW, row = m0 + r, col = n0 + 4 * q;
        if (col >= p.N) continue;
        int sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int z = 0; z < I8_MAX_SPLIT; ++z) {
            if (z >= (int)size) break;
            const float4 v = cluster_ld(part + (uint32_t)(r * PER_ROW + (q ^ (r & 7))) * 16, z);
            sum[0] += __float_as_int(v.x); sum[1] += __float_as_int(v.y); sum[2] += __float_as_int(v.z); sum[3] += __float_as_int(v.w);
        }
        const TO* add = static_cast<const TO*>(p.addend) + (p.addend ? row * p.ld_addend + col : 0);
        const float sa = p.sa[row];
        Pack<TO, 4> o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool there = col + e < p.N;
            o.v[e] = from_float<TO>(there ? scaled<false>(sum[e], sa, p.sb[col + e], p.addend, p.addend ? to_float(add[e]) : 0.f) : 0.f);
        }
        out_put<TO, 4>(p, row, col, o);
    }
}

// A 128 x BN tile of C at a time (persistent CTAs), the same for 256 x 256 and a pair of CTAs (TWO), or one tile per cluster, whose CTAs share its K (SPLIT).
// Warp 0 feeds a ring of shared-memory stages by TMA, warp 1 (of a pair: the first CTA's) issues the MMAs of a whole tile into one of two accumulators in
// tensor memory; the other warps, 64 columns at a time, scale and store the tile before it meanwhile.
template <int FORM>
__global__ void __launch_bounds__(i8_threads(FORM), i8_ctas_per_sm(FORM)) int8_product_kernel(const __grid_constant__ CUtensorMap tmA,
                                                                                               const __grid_constant__ CUtensorMap tmB,
                                                                                               const __grid_constant__ IntProductParams p) {
    constexpr bool SPLIT = FORM == I8_SPLIT, TWO = FORM == I8_TWO;
    constexpr int BN = i8_bn(FORM), STAGES = i8_stages(FORM), EW = i8_epi_warps(FORM), GROUPS = i8_groups(FORM), TILE_M = TWO ? 2 * I8_BM : I8_BM;
    constexpr uint32_t STAGE = i8_stage_bytes(FORM), TMEM_COLS = I8_NACC * BN;
    extern __shared__ __align__(1024) unsigned char i8_smem[];
    float4* const stores = reinterpret_cast<float4*>(i8_smem + (size_t)STAGES * STAGE);
    float* const column_scales = reinterpret_cast<float*>(i8_smem + (size_t)STAGES * STAGE + EW * 32 * I8_STORE_ROW);
    uint64_t* full = reinterpret_cast<uint64_t*>(column_scales + EW * OUT_COLS);
    uint64_t* empty = full + STAGES;
    uint64_t* acc_full = empty + STAGES;
    uint64_t* acc_empty = acc_full + I8_NACC;
    uint64_t* done = acc_empty + I8_NACC;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
    volatile uint32_t* stop = tmem_slot + 1;
    volatile uint32_t* filled = tmem_slot + 2;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = TWO || SPLIT ? cluster_rank() : 0u;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], TWO ? 2 : 1); mbar_init(&empty[s], 1); }
        for (int b = 0; b < I8_NACC; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], TWO ? 2 * EW : EW); }
        mbar_init(done, 1);
        *stop = 0;
        *filled = 0;
        mbar_init_fence();
    }
    if (warp == 1) {
        if constexpr (TWO) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (TWO) cluster_sync();         // (the pair's barriers and tensor memory are there)
    tmem_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_dependency_wait();          // (nothing of global memory was touched so far)
    allow_dependents();

    const int step = SPLIT ? p.items : (int)(TWO ? gridDim.x / 2 : gridDim.x);
    const int first = SPLIT ? (int)(blockIdx.x / cluster_size()) : (int)(TWO ? blockIdx.x / 2 : blockIdx.x);
    const int kb0 = SPLIT ? (int)rank * p.kper : 0, kb1 = SPLIT ? min(p.kblocks, kb0 + p.kper) : p.kblocks;

    if (warp < 4) {
        if (warp == 0 && lane == 0) {
            uint32_t s = 0, phase = 1, count = 0;
            bool ok = true;
            for (int item = first; item < p.items && ok; item += step) {
                const int m0 = item / p.tiles_n * TILE_M + (TWO ? (int)rank * I8_BM : 0), n0 = item % p.tiles_n * BN + (TWO ? (int)rank * 128 : 0);
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = mbar_wait_idle(&empty[s], phase, p.wait_limit) && !*stop;
                    if (!ok) { *stop = 1; note_status(p.status, KGE_ERR_TIMEOUT); break; }
                    unsigned char* sa = i8_smem + s * STAGE;
                    if constexpr (TWO) {
                        const uint32_t bar = cluster_addr(&full[s], 0);
                        mbar_arrive_expect_tx_cluster(bar, STAGE);
                        tma_load_pair(sa, &tmA, kb * OPERAND_BK, m0, bar);
                        tma_load_pair(sa + I8_BOX_BYTES, &tmB, kb * OPERAND_BK, n0, bar);
                    } else {
                        mbar_arrive_expect_tx(&full[s], STAGE);
                        tma_load_2d(sa, &tmA, kb * OPERAND_BK, m0, &full[s]);
                        tma_load_2d(sa + I8_BOX_BYTES, &tmB, kb * OPERAND_BK, n0, &full[s]);
                    }
                    ++count;
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                }
            }
            *filled = count;
        } else if (warp == 1 && lane == 0 && (!TWO || rank == 0)) {
            uint32_t s = 0, phase = 0, buf = 0, acc_phase = 1;
            bool ok = true;
            for (int item = first; item < p.items && ok && !*stop; item += step) {
                ok = TWO ? mbar_wait_cluster(&acc_empty[buf], acc_phase, p.wait_limit) : mbar_wait_idle(&acc_empty[buf], acc_phase, p.wait_limit);
                for (int kb = kb0; kb < kb1 && ok; ++kb) {
                    ok = mbar_wait_idle(&full[s], phase, p.wait_limit);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t sa = smem_u32(i8_smem + s * STAGE);
#pragma unroll
                    for (int k = 0; k < OPERAND_BK / 32; ++k) {
                        if constexpr (TWO) i8_mma_pair(tmem + buf * BN, operand_desc(sa + k * 32), operand_desc(sa + I8_BOX_BYTES + k * 32), p.idesc, kb != kb0 || k != 0);
                        else i8_mma(tmem + buf * BN, operand_desc(sa + k * 32), operand_desc(sa + I8_BOX_BYTES + k * 32), p.idesc, kb != kb0 || k != 0);
                    }
                    if constexpr (TWO) mma_commit_pair(&empty[s]);
                    else mma_commit(&empty[s]);
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                }
                if constexpr (TWO) mma_commit_pair(&acc_full[buf]);
                else mma_commit(&acc_full[buf]);
                if (++buf == I8_NACC) { buf = 0; acc_phase ^= 1; }
            }
            if (!ok) { *stop = 1; note_status(p.status, KGE_ERR_TIMEOUT); }
        }
        __syncwarp();
        if (SPLIT) { cluster_sync(); cluster_sync(); }
    } else {
        const int quarter = warp & 3, first_group = (warp - 4) >> 2;      // tensor-memory lanes and columns of this warp
        float4* const st = stores + (warp - 4) * (32 * I8_STORE_ROW / 16);
        float* const sb = column_scales + (warp - 4) * OUT_COLS;
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16);
        uint32_t buf = 0, phase = 0;
        bool ok = true;
        for (int item = first; item < p.items && ok; item += step) {
            const int m0 = item / p.tiles_n * TILE_M + (TWO ? (int)rank * I8_BM : 0) + quarter * 32, nt = item % p.tiles_n * BN;
            float sa = 1.f;
            bool near = true;
            auto begin = [&](int n0) {              // what a group of columns needs beside the sums
                near = near_one(sa);
#pragma unroll
                for (int i = 0; i < OUT_COLS; i += 32) {
                    const float s = n0 + i + lane < p.N ? __ldg(p.sb + n0 + i + lane) : 1.f;
                    near &= near_one(s);
                    sb[i + lane] = s;
                }
                near = __all_sync(0xffffffffu, near);
                if (p.addend) with_out_type(p.out_type, [&](auto t) { out_fetch_addend<decltype(t)>(p, m0, n0, 0, st, lane); });
                __syncwarp();
            };
            if (!SPLIT) {
                sa = m0 + lane < p.M ? __ldg(p.sa + m0 + lane) : 1.f;
                begin(nt + first_group * OUT_COLS);
            }
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&acc_full[buf], phase, p.wait_limit)) && !*stop;
            tmem_fence_after();
            if (!__all_sync(0xffffffffu, ok)) { ok = false; if (lane == 0) { *stop = 1; note_status(p.status, KGE_ERR_TIMEOUT); } break; }
            if (SPLIT) {       // the ring's stages are free: every copy has been multiplied
                float4* part = reinterpret_cast<float4*>(i8_smem);
                const int r = quarter * 32 + lane;
#pragma unroll
                for (int c = 0; c < OUT_COLS; c += 16) {
                    uint32_t v[16];
                    tmem_ld16(taddr + buf * BN + first_group * OUT_COLS + c, v);
                    tmem_wait16(v);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        part[r * (BN / 4) + ((first_group * (OUT_COLS / 4) + c / 4 + i) ^ (r & 7))] =
                            make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                }
            } else {
#pragma unroll 1
                for (int g = 0; g < GROUPS; ++g) {
                    const int col = (first_group + g * (EW / 4)) * OUT_COLS;
                    if (g > 0) begin(nt + col);
                    auto read_all = [&] {                 // the accumulator is read: another tile's MMAs may begin
                        if (g + 1 < GROUPS) return;
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if constexpr (TWO) mbar_arrive_cluster(cluster_addr(&acc_empty[buf], 0));
                            else mbar_arrive(&acc_empty[buf]);
                        }
                    };
                    with_out_type(p.out_type, [&](auto t) {
                        using TO = decltype(t);
                        const uint32_t from = taddr + buf * BN + col;
                        if (!near) {
                            if (p.addend) i8_store<TO, false, true>(p, m0, nt + col, from, sa, sb, st, lane, read_all);
                            else i8_store<TO, false, false>(p, m0, nt + col, from, sa, sb, st, lane, read_all);
                        } else if (p.addend) i8_store<TO, true, true>(p, m0, nt + col, from, sa, sb, st, lane, read_all);
                        else i8_store<TO, true, false>(p, m0, nt + col, from, sa, sb, st, lane, read_all);
                    });
                }
            }
            if (++buf == I8_NACC) { buf = 0; phase ^= 1; }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");       // (an addend's copies, after a wait that ran out)
        if (SPLIT) {       // (every warp of the cluster comes here, also after a wait that ran out)
            cluster_sync();
            const int m0 = first / p.tiles_n * I8_BM, n0 = first % p.tiles_n * BN;
            with_out_type(p.out_type, [&](auto t) { i8_join<decltype(t)>(p, smem_u32(i8_smem), m0, n0, threadIdx.x - 128); });
            cluster_sync();        // no CTA leaves while another reads its partial sums
        }
    }
    tmem_fence_before();
    __syncthreads();
    // Copies and MMAs in flight are waited for before a CTA's memory is given back, where a wait ran out; of a pair, the first CTA does so for both.
    if constexpr (TWO) {
        cluster_sync();
        if (rank == 0 && (*stop || cluster_ld_word(cluster_addr((const void*)stop, 1)))) {
            if (lane == 0 && warp == 0) {
                const int a = (int)*filled, b = (int)cluster_ld_word(cluster_addr((const void*)filled, 1)), n = max(a, b);
                for (int r = min(a, b); r < n; ++r) mbar_arrive(&full[r % STAGES]);          // (a stage that one of the two did not come to)
                for (int r = max(0, n - STAGES); r < n; ++r) mbar_wait_idle(&full[r % STAGES], (r / STAGES) & 1, kDefaultWaitLimit);
            }
            if (lane == 0 && warp == 1) { mma_commit_pair(done); mbar_wait_idle(done, 0, kDefaultWaitLimit); }
            __syncwarp();
        }
        cluster_sync();
        if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    } else {
        if (*stop) {
            if (lane == 0) {
                if (warp == 0) {
                    const int n = (int)*filled;
                    for (int r = max(0, n - STAGES); r < n; ++r) mbar_wait_idle(&full[r % STAGES], (r / STAGES) & 1, kDefaultWaitLimit);
                }
                if (warp == 1) { mma_commit(done); mbar_wait_idle(done, 0, kDefaultWaitLimit); }
            }
            __syncthreads();
        }
        if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

template <int FORM> int configure_product() {
    static DeviceOnce configured;
    return once_per_device(configured, [] {
        return cudaFuncSetAttribute(int8_product_kernel<FORM>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)i8_smem_bytes(FORM));
    }) == cudaSuccess ? KGE_OK : KGE_ERR_CUDA;
}

// How many clusters of `size` CTAs of a form the device runs at a time: asked for once (what is left of a part of the chip takes none).
template <int FORM> int clusters_at_a_time(int size, int* clusters) {
    static std::atomic<int> known[kMaxDevices][I8_MAX_SPLIT + 1];        // one more than their number
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return KGE_ERR_CUDA;
    const bool tracked = dev >= 0 && dev < kMaxDevices;
    int state = tracked ? known[dev][size].load(std::memory_order_acquire) : 0;
    if (state == 0) {
        const int rc = configure_product<FORM>();
        if (rc != KGE_OK) return rc;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)size); cfg.blockDim = dim3(i8_threads(FORM)); cfg.dynamicSmemBytes = i8_smem_bytes(FORM);
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)size; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 1;
        int fit = 0;
        if (cudaOccupancyMaxActiveClusters(&fit, int8_product_kernel<FORM>, &cfg) != cudaSuccess) { (void)cudaGetLastError(); fit = 0; }
        state = 1 + std::max(fit, 0);
        if (tracked) known[dev][size].store(state, std::memory_order_release);
    }
    *clusters = state - 1;
    return KGE_OK;
}

struct ProductPlan { int form, split; };          // split: CTAs that share a tile's K; pairs of CTAs that run at a time (TWO)
// How a product is cut up.
//   shared K      as many CTAs to a tile as run at a time, where the blocks that a CTA is spared outweigh the join: a block takes 0.4 us, the join 0.4 + 2 for 128 rows
//                 (16 x 4,096 x 4,096: four CTAs to each of 32 tiles, 9.3 us)
//   64 columns    of B at most: tiles of 128 x 64 (30,000 x 64 x 1,024: 10.3 us, in tiles of 256 x 256 14.9, of 128 x 128 on one CTA an SM 10.7; 17,479 x 64 x 624: 8.4, 9.0, 8.4.
//                 With a long K others would be ahead by up to a tenth: 30,000 x 64 x 4,096 29.9, 31.7, 27.9; 9,811 x 16 x 7,696 41.9, 38.0, 42.3)
//   else          the least of three estimates, in hundredths of a microsecond: a constant, and for every round of tiles that the chip takes another and one for each block
//                 of K (fitted to 125 shapes; the form chosen is 1.4 % slower than the best of the four on their mean, 18 % with the rule "256 x 256 where they fill the pairs").
//                   256 x 256               the least for a block, the most before and after it: 8,192 x 4,096 x 8,192 174 us, in tiles of 128 x 256 on one CTA 213;
//                                           9,811 x 222 x 7,696 35, in tiles of 128 x 128 50; 40,000 x 500 x 512 36 and 25
//                   128 x 128, two CTAs     a block waits for its copies, another CTA's stores go on meanwhile: K is short
//                   128 x 128, one CTA      in between, and the tiles are half as many as two an SM would take: 700 x 3,000 x 5,000 20 us, with two CTAs 25, 256 x 256 25
int product_plan(int64_t M, int64_t N, int kblocks, int sms, ProductPlan* plan) {
    const int64_t tiles128 = ceil_div(M, I8_BM) * ceil_div(N, 128), tiles256 = ceil_div(M, 256) * ceil_div(N, 256);
    for (int most = (int)std::min<int64_t>({I8_MAX_SPLIT, kblocks, sms / tiles128}); most > 1; --most) {
        const int per = (kblocks + most - 1) / most, split = (kblocks + per - 1) / per;          // every CTA has a block
        if (128 * (kblocks - per - 1) <= 5 * std::min<int64_t>(M, I8_BM)) break;
        int room = 0;
        const int rc = clusters_at_a_time<I8_SPLIT>(split, &room);
        if (rc != KGE_OK) return rc;
        if (tiles128 <= room) { *plan = {I8_SPLIT, split}; return KGE_OK; }
    }
    if (N <= 64) { *plan = {I8_NARROW, 1}; return KGE_OK; }
    int room = 0;
    const int rc = clusters_at_a_time<I8_TWO>(2, &room);
    if (rc != KGE_OK) return rc;
    const int64_t two = room > 0 && kblocks >= 4 ? 600 + ceil_div(tiles256, room) * (32 * kblocks + 200) : INT64_MAX;
    const int64_t pair = 400 + ceil_div(tiles128, 2 * sms) * (60 * kblocks + 100), deep = 450 + ceil_div(tiles128, sms) * (32 * kblocks + 70);
    if (two <= std::min(pair, deep)) *plan = {I8_TWO, (int)std::min<int64_t>(room, tiles256)};
    else *plan = {deep <= pair ? I8_DEEP : I8_PAIR, 1};
    return KGE_OK;
}

template <int FORM>
int launch_product(const CUtensorMap& a, const CUtensorMap& b, IntProductParams& p, int split, int sms, cudaStream_t s) {
    constexpr size_t smem = i8_smem_bytes(FORM);
    static_assert((smem + 1024) * i8_ctas_per_sm(FORM) <= 228 * 1024, "shared memory of an SM");
    const int rc = configure_product<FORM>();
    if (rc != KGE_OK) return rc;
    p.tiles_n = (int)ceil_div(p.N, i8_bn(FORM));
    p.items = (int)(ceil_div(p.M, FORM == I8_TWO ? 2 * I8_BM : I8_BM) * p.tiles_n);
    p.kper = FORM == I8_SPLIT ? (p.kblocks + split - 1) / split : p.kblocks;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(FORM == I8_SPLIT ? p.items * split : (FORM == I8_TWO ? 2 * split : std::min<int64_t>(p.items, (int64_t)sms * i8_ctas_per_sm(FORM)))));
    cfg.blockDim = dim3(i8_threads(FORM)); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)(FORM == I8_TWO ? 2 : split); attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = FORM == I8_SPLIT || FORM == I8_TWO ? 2 : 1;
    return launch_status(cudaLaunchKernelEx(&cfg, int8_product_kernel<FORM>, a, b, p));
}

}  // namespace
}  // namespace kge

using namespace kge;

extern "C" {

int kge_int8_quantize(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx, void* q, int64_t ldq, float* scales, void* stream) {
    if (!is_float_type(x_type) || rows < 0 || rows > INT32_MAX || cols < 0 || cols > INT32_MAX - 65536 || ldx < cols || ldq < cols || ldq % 16 || !aligned_to(q, 16) ||
        !aligned_to(scales, 4)) return KGE_ERR_BAD_ARG;
    if (rows == 0) return KGE_OK;
    if ((cols > 0 && (!x || !q)) || !scales || !aligned_to(x, type_bytes(x_type))) return KGE_ERR_BAD_ARG;          // (rows of no columns have a scale)
    QuantParams p{};
    p.x = x; p.ldx = ldx; p.q = static_cast<int8_t*>(q); p.ldq = ldq; p.scales = scales; p.rows = (int)rows; p.cols = (int)cols;
    p.wide = cols % 8 == 0 && ldx % 8 == 0 && aligned_to(x, (size_t)(8 * type_bytes(x_type)));
    return with_type(x_type, [&](auto t) {
        return p.wide ? launch_quantize<decltype(t), true>(p, static_cast<cudaStream_t>(stream)) : launch_quantize<decltype(t), false>(p, static_cast<cudaStream_t>(stream));
    });
}

int kge_int8_matmul(const void* a, int64_t lda, const float* a_scales, const void* b, int64_t ldb, const float* b_scales, const void* addend, int64_t ld_addend,
                    void* out, int32_t out_type, int64_t ld_out, int64_t M, int64_t N, int64_t K, int32_t* status, void* stream) {
    if (!is_float_type(out_type) || M < 0 || N < 0 || K < 1 || M > INT32_MAX - 256 || N > INT32_MAX - 256 || ld_out < N || (addend && ld_addend < N))
        return KGE_ERR_BAD_ARG;
    if (M == 0 || N == 0) return KGE_OK;
    if (!a || !b || !a_scales || !b_scales || !out || lda < K || ldb < K || lda % 16 || ldb % 16 || !aligned_to(a, 16) || !aligned_to(b, 16) ||
        !aligned_to(a_scales, 4) || !aligned_to(b_scales, 4) || !aligned_to(out, type_bytes(out_type)) ||
        (addend && !aligned_to(addend, type_bytes(out_type))) || !aligned_to(status, 4)) return KGE_ERR_BAD_ARG;
    if (K > 131071 || ceil_div(M, 128) * ceil_div(N, 64) > INT32_MAX / 8) return KGE_ERR_UNSUPPORTED;        // (sums beyond 32 bits; tiles beyond their counters)
    IntProductParams p{};
    p.M = M; p.N = N; p.kblocks = (int)ceil_div(K, OPERAND_BK);
    p.sa = a_scales; p.sb = b_scales;
    p.addend = addend; p.ld_addend = ld_addend; p.out = out; p.ld_out = ld_out; p.out_type = out_type;
    const int ob = type_bytes(out_type);
    p.vec = ld_out * ob % 16 == 0 && aligned_to(out, 16) && (!addend || (ld_addend * ob % 16 == 0 && aligned_to(addend, 16)));
    p.twos = N % 2 == 0 && ld_out % 2 == 0 && aligned_to(out, 2 * ob) && (!addend || (ld_addend % 2 == 0 && aligned_to(addend, 2 * ob)));
    p.status = status; p.wait_limit = product_wait_limit.load(std::memory_order_relaxed);
    int sms = 0, rc = sm_count(&sms);
    if (rc != KGE_OK) return rc;
    ProductPlan plan;
    rc = product_plan(M, N, p.kblocks, sms, &plan);
    if (rc != KGE_OK) return rc;
    alignas(64) CUtensorMap ma, mb;
    rc = operand_map(&ma, a, M, K, lda, I8_BM);
    if (rc == KGE_OK) rc = operand_map(&mb, b, N, K, ldb, i8_box_rows(plan.form));
    if (rc != KGE_OK) return rc;
    p.idesc = i8_idesc(plan.form == I8_TWO ? 2 * I8_BM : I8_BM, i8_bn(plan.form));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (plan.form) {
        case I8_SPLIT: return launch_product<I8_SPLIT>(ma, mb, p, plan.split, sms, s);
        case I8_TWO: return launch_product<I8_TWO>(ma, mb, p, plan.split, sms, s);
        case I8_DEEP: return launch_product<I8_DEEP>(ma, mb, p, 1, sms, s);
        case I8_NARROW: return launch_product<I8_NARROW>(ma, mb, p, 1, sms, s);
        default: return launch_product<I8_PAIR>(ma, mb, p, 1, sms, s);
    }
}

}  // extern "C"
