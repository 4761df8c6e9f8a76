// 8-bit floating point with a scale for each block of 128 along the contraction index: making such operands, and their product.
//   quantise   s = amax / top (or the next power of two), q = the 8-bit value nearest to x / s; one scale per 1 x 128 or 128 x 128 block
//   product    C[m, n] = sum_kb sA[kb, m] sB[kb, n] sum_{k in kb} A[m, k] B[n, k]   (+ C0[m, n])
#include <cuda.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "kge_ops.cuh"

namespace kge {

namespace {

// ---- quantisation ----------------------------------------------------------------------------------------------------

struct QuantParams {
    const void* x; int64_t ldx;
    int64_t rows, cols;
    uint8_t *q, *qt; int64_t ldq, ldqt;
    float *scales, *scales_t;
    int vec;                         // rows of x start at multiples of 16 bytes
    int pow2;
    int64_t tiles_c;
};

template <int FMT> struct Fp8Traits;
template <> struct Fp8Traits<KGE_E4M3> { static constexpr float top = 448.f; };
template <> struct Fp8Traits<KGE_E5M2> { static constexpr float top = 57344.f; };

// Eight consecutive values of a row, and their magnitudes as integers that order as they do (a NaN above all).
template <typename TX> struct Eight;
template <> struct Eight<float> {
    float v[8];
    __device__ __forceinline__ void load(const void* p) { *reinterpret_cast<Pack<float, 8>*>(v) = *static_cast<const Pack<float, 8>*>(p); }
    __device__ __forceinline__ void set(int j, float x) { v[j] = x; }
    __device__ __forceinline__ float value(int j) const { return v[j]; }
    __device__ __forceinline__ uint32_t key(int j) const { return __float_as_uint(v[j]) & 0x7FFFFFFFu; }
    __device__ __forceinline__ uint32_t most() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, key(j));
        return m;
    }
};
template <typename T16> struct Eight16 {
    uint32_t w[4];
    __device__ __forceinline__ void load(const void* p) { *reinterpret_cast<uint4*>(w) = *static_cast<const uint4*>(p); }
    __device__ __forceinline__ void set(int j, T16 x) {
        const uint32_t b = *reinterpret_cast<const uint16_t*>(&x);
        w[j >> 1] = j & 1 ? (w[j >> 1] & 0xFFFFu) | b << 16 : b;
    }
    __device__ __forceinline__ uint32_t key(int j) const { return (j & 1 ? w[j >> 1] >> 16 : w[j >> 1]) & 0x7FFFu; }
    __device__ __forceinline__ uint32_t most() const {
        uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
        for (int j = 1; j < 4; ++j) m = __vmaxu2(m, w[j] & 0x7FFF7FFFu);
        return max(m & 0xFFFFu, m >> 16);
    }
};
template <> struct Eight<__nv_bfloat16> : Eight16<__nv_bfloat16> {
    __device__ __forceinline__ float value(int j) const { return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16); }
};
template <> struct Eight<__half> : Eight16<__half> {
    __device__ __forceinline__ float value(int j) const {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j >> 1]));
        return j & 1 ? f.y : f.x;
    }
};
template <typename TX> __device__ __forceinline__ float key_value(uint32_t key);
template <> __device__ __forceinline__ float key_value<float>(uint32_t key) { return __uint_as_float(key); }
template <> __device__ __forceinline__ float key_value<__nv_bfloat16>(uint32_t key) { return __uint_as_float(key << 16); }
template <> __device__ __forceinline__ float key_value<__half>(uint32_t key) { return __half2float(__ushort_as_half((unsigned short)key)); }

// A block's scale, and what its values are multiplied by.  A block of zeros has scale 1; an infinity or a NaN makes the scale one, and
// the factor 0: the block's values become 0, or NaN where they are an infinity or a NaN themselves, and stand for NaN all of them.
//
// The 8-bit value stored is the one nearest to the true quotient x / s; t = x (1 / s) is within 2^-23 of it, which matters where a
// middle of two 8-bit values is that close.  With 16-bit inputs that has structure.  s = (a / 7 2^k) (1 + e) with a the block's
// largest value, |e| <= 2^-24 the rounding of s; x / a times 7 either is such a middle exactly, or off it by 2^-16 at least (x and
// a have at most 11 bits, a middle 5).  In the first case the true quotient lies on the side of the middle that the sign of e
// says, the same for all values of the block: `inv` leans by 2^-21 to that side.  Where e = 0 the quotient is the middle
// itself, and t is brought back to the multiple of 16 units next to it; the last bit of `inv` says so.  With fp32 inputs
// quotient() compares each value.
struct Block { float s, inv; };
template <typename TX, int FMT, bool POW2>
__device__ __forceinline__ Block block_of(uint32_t key) {
    const float a = key_value<TX>(key);
    Block b;
    b.s = a / Fp8Traits<FMT>::top;
    const bool finite = a < __int_as_float(0x7F800000);       // (false for a NaN)
    float e = 0.f;
    if (finite) {
        if (!POW2 && b.s > 1.17549435e-38f) e = fmaf(-b.s, Fp8Traits<FMT>::top, a);
        b.s = a == 0.f ? 1.f : fmaxf(b.s, 1.17549435e-38f);
        if (POW2) b.s = __uint_as_float((__float_as_uint(b.s) + 0x007FFFFFu) & 0x7F800000u);
    }
    b.inv = finite ? 1.f / b.s : 0.f;
    if (!POW2 && sizeof(TX) == 2 && finite) {
        const float lean = e > 0.f ? 4.76837158e-7f : (e < 0.f ? -4.76837158e-7f : 0.f);
        b.inv = __uint_as_float((__float_as_uint(fmaf(b.inv, lean, b.inv)) & ~1u) | (e == 0.f ? 1u : 0u));
    }
    return b;
}
// |x| / s in fp32 such that rounding it to 8 bits rounds the true quotient: m, the multiple of 16 units next to t (all middles are
// such), is compared with it exactly (the sign of |x| - m s, one fused operation); the result is m or the value next to it.
__device__ __forceinline__ float quotient(float x, float s, float inv) {
    int32_t m = (int32_t)(__float_as_uint(fabsf(x) * inv) + 8u) & ~15;
    const float r = fmaf(-__int_as_float(m), s, fabsf(x));
    if (r > 0.f) ++m;
    if (r < 0.f) --m;
    return __uint_as_float((uint32_t)m | (__float_as_uint(x) & 0x80000000u));
}
template <int FMT>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    constexpr __nv_fp8_interpretation_t f = FMT == KGE_E4M3 ? __NV_E4M3 : __NV_E5M2;
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, f), hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, f);
    return lo | hi << 16;
}
template <typename TX, int FMT, bool POW2>
__device__ __forceinline__ uint2 round8(float (&v)[8], const Block& b) {
    if constexpr (POW2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= b.inv;
    } else if constexpr (sizeof(TX) == 2) {
        const uint32_t snap = __float_as_uint(b.inv) & 1u, add = snap << 3, mask = ~(snap * 15u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float((__float_as_uint(v[j] * b.inv) + add) & mask);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = quotient(v[j], b.s, b.inv);
    }
    return make_uint2(pack4<FMT>(v[0], v[1], v[2], v[3]), pack4<FMT>(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void put8(uint8_t* dst, uint2 w, int64_t valid) {
    if (valid >= 8) *reinterpret_cast<uint2*>(dst) = w;
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (j < valid) dst[j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
}

// Largest of R rows' magnitudes over sixteen lanes (offsets 8 ... 1 of a warp's halves): every exchange halves the rows a lane keeps,
// so that lane l is left with row row_of_lane<R>(l)'s, ready for one division a lane instead of R in all of them.
template <int R>
__device__ __forceinline__ uint32_t rows_max(uint32_t (&m)[R], int lane) {
    int off = 8;
#pragma unroll
    for (int n = R; n > 1; n >>= 1, off >>= 1) {
#pragma unroll
        for (int i = 0; i < n / 2; ++i) {
            const bool upper = lane & off;
            const uint32_t keep = upper ? m[n / 2 + i] : m[i], give = upper ? m[i] : m[n / 2 + i];
            m[i] = max(keep, __shfl_xor_sync(0xffffffffu, give, off));
        }
    }
#pragma unroll
    for (; off > 0; off >>= 1) m[0] = max(m[0], __shfl_xor_sync(0xffffffffu, m[0], off));
    return m[0];
}
// A lane (of its half) that holds row i, and the row that lane l holds.
template <int R> __device__ __forceinline__ int lane_of_row(int i) { return R == 8 ? i << 1 : (R == 4 ? i << 2 : i << 3); }
template <int R> __device__ __forceinline__ int row_of_lane(int l) { return R == 8 ? (l & 15) >> 1 : (R == 4 ? (l & 15) >> 2 : (l & 15) >> 3); }
template <typename TX, int R>
__device__ __forceinline__ Block block_of_row(const Block& mine, int i) {
    Block b;
    b.inv = __shfl_sync(0xffffffffu, mine.inv, lane_of_row<R>(i), 16);
    b.s = sizeof(TX) == 4 ? __shfl_sync(0xffffffffu, mine.s, lane_of_row<R>(i), 16) : 0.f;       // (only fp32 inputs look at it again)
    return b;
}

// Values c0 ... c0 + 7 of row r; zeros beyond the matrix.
template <typename TX>
__device__ __forceinline__ void load8(const QuantParams& p, Eight<TX>& e, int64_t r, int64_t c0) {
    const TX* x = static_cast<const TX*>(p.x) + r * p.ldx + c0;
    if (p.vec && c0 + 8 <= p.cols && r < p.rows) e.load(x);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) e.set(j, r < p.rows && c0 + j < p.cols ? x[j] : from_float<TX>(0.f));
    }
}

// One CTA per 128 x 128 tile: thread (rg, cg) holds rows 8 rg .. + 8 and columns 8 cg .. + 8, so both forms come of one read.  24,576 x 768
// bf16 in 17.5 us, calls in a row (one form alone 10 to 11; 22 with cold caches); issue slots two thirds busy at four CTAs an SM.
template <typename TX, int FMT, bool SQUARE, bool POW2>
__global__ void __launch_bounds__(256, sizeof(TX) == 2 ? 4 : 2) quantize_kernel(QuantParams p) {
    __shared__ uint32_t part[16][128];
    __shared__ Block col_block[128];
    __shared__ alignas(16) uint2 turned[128][16];
    grid_dependency_wait();
    allow_dependents();
    const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4;
    const int64_t tr = blockIdx.x / p.tiles_c, tc = blockIdx.x - tr * p.tiles_c;
    const int64_t r0 = tr * 128 + rg * 8, c0 = tc * 128 + cg * 8;
    Eight<TX> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) load8<TX>(p, x[i], r0 + i, c0);
    Block all{};
    if (SQUARE) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, x[i].most());
        m = __reduce_max_sync(0xffffffffu, m);
        if ((tid & 31) == 0) part[0][tid >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) m = max(m, part[0][w]);
        all = block_of<TX, FMT, POW2>(m);
        if (tid == 0) {
            const int64_t row_blocks = (p.rows + 127) / 128;
            if (p.q) p.scales[tc * row_blocks + tr] = all.s;
            if (p.qt) p.scales_t[tr * p.tiles_c + tc] = all.s;
        }
    }
    if (p.q) {
        Block mine = all;
        if (!SQUARE) {
            uint32_t m[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) m[i] = x[i].most();
            const int lane = tid & 31;
            mine = block_of<TX, FMT, POW2>(rows_max<8>(m, lane));
            const int64_t r = r0 + row_of_lane<8>(lane);
            if ((lane & 1) == 0 && r < p.rows) p.scales[tc * p.rows + r] = mine.s;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Block b = SQUARE ? all : block_of_row<TX, 8>(mine, i);
            float t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = x[i].value(j);
            const uint2 w = round8<TX, FMT, POW2>(t, b);
            if (r0 + i < p.rows) put8(p.q + (r0 + i) * p.ldq + c0, w, p.cols - c0);
        }
    }
    if (p.qt) {
        if (!SQUARE) {
            if constexpr (sizeof(TX) == 2) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t m = x[0].w[j] & 0x7FFF7FFFu;
#pragma unroll
                    for (int i = 1; i < 8; ++i) m = __vmaxu2(m, x[i].w[j] & 0x7FFF7FFFu);
                    *reinterpret_cast<uint2*>(&part[rg][cg * 8 + 2 * j]) = make_uint2(m & 0xFFFFu, m >> 16);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t m = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) m = max(m, x[i].key(j));
                    part[rg][cg * 8 + j] = m;
                }
            }
            __syncthreads();
            if (tid < 128) {
                uint32_t m = 0;
#pragma unroll
                for (int g = 0; g < 16; ++g) m = max(m, part[g][tid]);
                const Block b = block_of<TX, FMT, POW2>(m);
                col_block[tid] = b;
                const int64_t c = tc * 128 + tid;
                if (c < p.cols) p.scales_t[tr * p.cols + c] = b.s;
            }
            __syncthreads();
        }
        // columns become rows of 128 bytes in shared memory; 8-byte unit u of row c lies at u ^ (c / 8), free of bank conflicts
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const Block b = SQUARE ? all : col_block[cg * 8 + j];
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = x[i].value(j);
            turned[cg * 8 + j][rg ^ cg] = round8<TX, FMT, POW2>(t, b);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = k * 32 + (tid >> 3), piece = tid & 7;
            const int64_t col = tc * 128 + c, row = tr * 128 + piece * 16;
            if (col >= p.cols || row >= p.rows) continue;
            const uint2 a = turned[c][(2 * piece) ^ (c >> 3)], b = turned[c][(2 * piece + 1) ^ (c >> 3)];
            uint8_t* dst = p.qt + col * p.ldqt + row;
            if (row + 16 <= p.rows) *reinterpret_cast<uint4*>(dst) = make_uint4(a.x, a.y, b.x, b.y);
            else { put8(dst, a, p.rows - row); if (p.rows - row > 8) put8(dst + 8, b, p.rows - row - 8); }
        }
    }
}

// Blocks of 1 x 128 along the rows only: a warp takes sixteen rows of one block of columns, eight or four at a time (sixteen lanes of
// eight columns each), the next ones' loads under way.  100,000 x 768 bf16 in 46 us (5 TB/s): fourteen instructions an element, issue
// slots 75 % busy.
template <typename TX, int FMT, bool POW2>
__global__ void __launch_bounds__(256, 4) quantize_rows_kernel(QuantParams p) {
    constexpr int STEP = sizeof(TX) == 2 ? 4 : 2, ROWS = 16, STEPS = ROWS / (2 * STEP);
    grid_dependency_wait();
    allow_dependents();
    const int lane = threadIdx.x & 31, cg = lane & 15;
    const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t tr = unit / p.tiles_c, tc = unit - tr * p.tiles_c;
    const int64_t r_first = tr * ROWS + (lane >> 4), c0 = tc * 128 + cg * 8;
    if (tr * ROWS >= p.rows) return;
    Eight<TX> x[2][STEP];
#pragma unroll
    for (int i = 0; i < STEP; ++i) load8<TX>(p, x[0][i], r_first + 2 * i, c0);
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        if (tr * ROWS + 2 * STEP * k >= p.rows) break;
        if (k + 1 < STEPS) {
#pragma unroll
            for (int i = 0; i < STEP; ++i) load8<TX>(p, x[(k + 1) & 1][i], r_first + 2 * (STEP * (k + 1) + i), c0);
        }
        uint32_t m[STEP];
#pragma unroll
        for (int i = 0; i < STEP; ++i) m[i] = x[k & 1][i].most();
        const Block mine = block_of<TX, FMT, POW2>(rows_max<STEP>(m, lane));
        const int64_t r_mine = r_first + 2 * (STEP * k + row_of_lane<STEP>(lane));
        if ((lane & (16 / STEP - 1)) == 0 && r_mine < p.rows) p.scales[tc * p.rows + r_mine] = mine.s;
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const int64_t r = r_first + 2 * (STEP * k + i);
            const Block b = block_of_row<TX, STEP>(mine, i);
            float t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = x[k & 1][i].value(j);
            const uint2 w = round8<TX, FMT, POW2>(t, b);
            if (r < p.rows) put8(p.q + r * p.ldq + c0, w, p.cols - c0);
        }
    }
}

template <typename TX>
int launch_quantize(const QuantParams& p, int fmt, bool square, cudaStream_t s) {
    auto with_format = [&](auto pow2) {
        constexpr bool P = decltype(pow2)::value;
        if (!square && !p.qt) {
            const dim3 grid((unsigned)ceil_div(p.tiles_c * ceil_div(p.rows, 16), 8));
            return fmt == KGE_E4M3 ? launch_dependent(quantize_rows_kernel<TX, KGE_E4M3, P>, grid, dim3(256), 0, s, p)
                                   : launch_dependent(quantize_rows_kernel<TX, KGE_E5M2, P>, grid, dim3(256), 0, s, p);
        }
        const dim3 grid((unsigned)(p.tiles_c * ceil_div(p.rows, 128)));
        if (square)
            return fmt == KGE_E4M3 ? launch_dependent(quantize_kernel<TX, KGE_E4M3, true, P>, grid, dim3(256), 0, s, p)
                                   : launch_dependent(quantize_kernel<TX, KGE_E5M2, true, P>, grid, dim3(256), 0, s, p);
        return fmt == KGE_E4M3 ? launch_dependent(quantize_kernel<TX, KGE_E4M3, false, P>, grid, dim3(256), 0, s, p)
                               : launch_dependent(quantize_kernel<TX, KGE_E5M2, false, P>, grid, dim3(256), 0, s, p);
    };
    return launch_status(p.pow2 ? with_format(std::true_type()) : with_format(std::false_type()));
}

// ---- product ---------------------------------------------------------------------------------------------------------

constexpr int FP_BM = 128, FP_BK = 128;                   // BK bytes = one 128-byte swizzle row
constexpr uint32_t FP_BOX_BYTES = 128 * FP_BK;            // 128 rows of an operand
constexpr int FP_NACC = 2;                                // block sums in tensor memory
constexpr int FP_COLS = 64;                               // columns of the tile per epilogue warp
// Four forms of the kernel: tiles of 256 columns, one CTA an SM, for many blocks of K; tiles of 128, two CTAs an SM (one loads and
// multiplies while the other stores), or of 64, three CTAs an SM, for few; tiles of 128 whose blocks of K a cluster shares, where
// tiles are few.
enum { FP_WIDE = 0, FP_PAIR = 1, FP_SPLIT = 2, FP_NARROW = 3 };
constexpr int FP_MAX_SPLIT = 8;           // CTAs that share a tile's blocks of K
__host__ __device__ constexpr int fp_bn(int form) { return form == FP_WIDE ? 256 : (form == FP_NARROW ? 64 : 128); }
__host__ __device__ constexpr int fp_box_rows(int form) { return form == FP_NARROW ? 64 : 128; }             // of B per copy
__host__ __device__ constexpr int fp_stages(int form) { return form == FP_WIDE ? 4 : (form == FP_SPLIT ? 6 : 2); }
__host__ __device__ constexpr int fp_epi_warps(int form) { return 4 * fp_bn(form) / FP_COLS; }
__host__ __device__ constexpr int fp_threads(int form) { return 32 * (4 + fp_epi_warps(form)); }     // (four more: copies, MMAs, a look at the scales, one idle)
__host__ __device__ constexpr int fp_ctas_per_sm(int form) { return form == FP_PAIR ? 2 : (form == FP_NARROW ? 3 : 1); }
__host__ __device__ constexpr uint32_t fp_stage_bytes(int form) { return FP_BOX_BYTES + (uint32_t)fp_bn(form) * FP_BK; }
// Per epilogue warp: 32 rows x 32 or 128 bytes of the output on their way to memory.
__host__ __device__ constexpr uint32_t fp_store_row(int form) { return form == FP_PAIR || form == FP_NARROW ? 128 : 32; }
// Blocks of K whose scales (and a word about them) are in shared memory.  A slot needs no barrier of its own: its block's scales are read before the epilogue
// hands back the block sum after the next one, without which no MMA of the block FP_NACC later is issued, without which no stage
// that follows by fp_stages() more is filled again -- at least stages + FP_NACC + 1 blocks later.
__host__ __device__ constexpr int fp_slots(int form) { return fp_stages(form) + FP_NACC + 2; }
__host__ __device__ constexpr size_t fp_smem_bytes(int form) {
    return (size_t)fp_stages(form) * fp_stage_bytes(form) + fp_epi_warps(form) * 32 * fp_store_row(form) + fp_slots(form) * (128 + fp_bn(form)) * 4 + 256;
}

struct ProductParams {
    int64_t M, N;
    int kblocks, kper;                    // blocks of K in all, and per CTA of a cluster
    int tiles_n, items;
    const float *sa, *sb;
    int64_t sa_ld, sb_ld;                 // scales per block of K
    int a_square, b_square;               // a scale serves 128 rows
    const void* addend; int64_t ld_addend;
    void* out; int64_t ld_out; int out_type;
    int vec, twos;                        // rows of out (and addend) start at multiples of 16 bytes; of two elements, N even
    int32_t* status; int wait_limit;
    uint32_t idesc;
};

__device__ __forceinline__ void fp_tma_load(void* dst, const CUtensorMap* tm, int x, int y, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}
// Shared-memory descriptor of a K-major operand tile with the 128-byte swizzle: rows of 128 bytes, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t fp_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor: D fp32, A and B 8-bit (0 = e4m3, 1 = e5m2), both K-major.
constexpr uint32_t fp_idesc(int m, int n, int fa, int fb) {
    return (1u << 4) | ((uint32_t)fa << 7) | ((uint32_t)fb << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void fp_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void fp_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fp_copy4(uint32_t dst, const float* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void fp_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fp_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 16 consecutive columns of this thread's tensor-memory lane.  Nothing may look at the registers before fp_tmem_wait has passed them on.
__device__ __forceinline__ void fp_tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
// Waits for this thread's tensor-memory loads; the registers pass through, so that nothing that uses them moves ahead.
__device__ __forceinline__ void fp_tmem_wait(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ uint64_t two_words(uint32_t a, uint32_t b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b)); return r; }
// Two fp32 operations in one instruction, each rounded as a single one would be.
__device__ __forceinline__ uint64_t pair(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 unpair(uint64_t a) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a)); return r; }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }

// A block's sum x joins c as x (a b), a and b the block's scales, where a b is a normal number (or not finite: a block that stands for NaN).
// Where it is not, as (x a) b.  |x| is 0 or between 2^-32 and 2^39 (products of 8-bit values, 128 of them): with a b below the normal
// numbers a and b are below 1 and x a is off by half a step of the smallest numbers at most; with a b beyond the largest number, scales
// of finite blocks (up to 2^119) are both above 2^8, and x a is infinite only where x a b is.
__device__ __forceinline__ float fp_add_far(float x, float a, float b, float c) {
    const float ab = a * b, size = fabsf(ab);
    const bool far = size < 1.17549435e-38f || (size == __int_as_float(0x7F800000) && fabsf(a) < size && fabsf(b) < size);
    return far ? fmaf(x * a, b, c) : fmaf(x, ab, c);
}
__device__ __forceinline__ uint64_t fp_add_far(uint64_t x, float a, float b0, float b1, uint64_t c) {
    const float2 u = unpair(x), v = unpair(c);
    return pair(fp_add_far(u.x, a, b0, v.x), fp_add_far(u.y, a, b1, v.y));
}
// Between 2^-63 and 2^63: the product of two such scales is a normal number.
__device__ __forceinline__ bool fp_near_one(float s) { return __float_as_uint(s) - 0x20000000u <= 0x3F000000u; }

// Scales of a tile's block of K that lane `lane` takes: those i (32 rows or columns apart) with 32 i below the result.
__device__ __forceinline__ int fp_scales_a(const ProductParams& p, int m0, int lane) { return p.a_square ? (lane == 0 ? 1 : 0) : (int)p.M - m0 - lane; }
template <int BN> __device__ __forceinline__ int fp_scales_b(const ProductParams& p, int n0, int lane) {
    return p.b_square ? (lane < (BN + 127) / 128 && n0 + 128 * lane < p.N ? 1 : 0) : (int)p.N - n0 - lane;
}

// Registers of a warpgroup, out of what the block was launched with.
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// Calls f with a value of the output type.
template <class F> __device__ __forceinline__ void fp_with_out(int t, F&& f) {
    if (t == KGE_F32) f(float());
    else if (t == KGE_BF16) f(__nv_bfloat16());
    else f(__half());
}

// A pack of a row's columns.
template <typename TO, int V>
__device__ __forceinline__ void fp_put(const ProductParams& p, int row, int col, const Pack<TO, V>& o) {
    TO* dst = static_cast<TO*>(p.out) + row * p.ld_out + col;
    if (p.vec && col + V <= p.N) *reinterpret_cast<Pack<TO, V>*>(dst) = o;
    else {
#pragma unroll
        for (int e = 0; e < V; ++e) if (col + e < p.N) dst[e] = o.v[e];
    }
}

// Where rows do not start at multiples of 16 bytes, and at the matrix's edges: f(row, column, place in shared memory) for W elements at a
// time of the warp's 32 rows x ROW bytes, lanes side by side along the columns.
template <typename TO, int ROW, int W, class F>
__device__ __forceinline__ void fp_each(const ProductParams& p, int row0, int col0, float4* st, int lane, F&& f) {
    constexpr int V = 16 / sizeof(TO), UNITS = ROW / 16, TURN = UNITS == 2 ? 2 : 0, PER_ROW = ROW / (int)sizeof(TO) / W;
#pragma unroll 4
    for (int i = 0; i < PER_ROW; ++i) {
        const int at = i * 32 + lane, r = at / PER_ROW, c = at % PER_ROW * W;
        if (row0 + r < p.M && col0 + c < p.N)
            f(row0 + r, col0 + c, reinterpret_cast<TO*>(st) + (r * UNITS + ((c / V) ^ ((r >> TURN) & (UNITS - 1)))) * V + c % V);
    }
}

// A warp's 32 rows x 64 columns, ROW bytes of each row at a time through shared memory, so that a store instruction covers whole
// 32-byte sectors, or, with 128 bytes, whole lines.  (16-byte unit i of row r lies at i ^ (r mod units): no bank conflicts.)
template <typename TO, int ROW>
__device__ __forceinline__ void fp_store(const ProductParams& p, int row0, int col0, const uint64_t (&acc)[FP_COLS / 2], float4* st, int lane) {
    constexpr int V = 16 / sizeof(TO), UNITS = ROW / 16, PASS = ROW / sizeof(TO);      // columns per unit, units and columns per pass
    constexpr int TURN = UNITS == 2 ? 2 : 0;                                            // rows 4 apart share banks at 32 bytes a row
    // a warp's part that lies inside the matrix is stored without a look at its edges
    const bool inside = p.vec && row0 + 32 <= p.M && col0 + FP_COLS <= p.N;
    TO* const first = static_cast<TO*>(p.out) + (row0 + lane / UNITS) * p.ld_out + col0 + V * (lane % UNITS);
    const int64_t step = (32 / UNITS) * p.ld_out;
#pragma unroll
    for (int c = 0; c < FP_COLS; c += PASS) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            Pack<TO, V> own;
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                const float2 x = unpair(acc[(c + i * V + e) / 2]);
                own.v[e] = from_float<TO>(x.x);
                own.v[e + 1] = from_float<TO>(x.y);
            }
            st[lane * UNITS + (i ^ ((lane >> TURN) & (UNITS - 1)))] = *reinterpret_cast<const float4*>(&own);
        }
        __syncwarp();
        const int r0 = lane / UNITS, unit = lane % UNITS;
        if (inside) {
            TO* dst = first + c;
#pragma unroll
            for (int j = 0; j < UNITS; ++j) {
                const int r = j * (32 / UNITS) + r0;
                *reinterpret_cast<float4*>(dst) = st[r * UNITS + (unit ^ ((r >> TURN) & (UNITS - 1)))];
                dst += step;
            }
        } else if (sizeof(TO) == 2 && p.twos) {
            fp_each<TO, ROW, 2>(p, row0, col0 + c, st, lane, [&](int row, int col, TO* at) {
                *reinterpret_cast<uint32_t*>(static_cast<TO*>(p.out) + row * p.ld_out + col) = *reinterpret_cast<const uint32_t*>(at);
            });
        } else {
            fp_each<TO, ROW, 1>(p, row0, col0 + c, st, lane, [&](int row, int col, TO* at) { static_cast<TO*>(p.out)[row * p.ld_out + col] = *at; });
        }
        __syncwarp();
    }
}

// The addend of the same tile joins the accumulators in fp32 before they are rounded.
// With 128-byte rows it passes through the warp's shared memory: fp_fetch_addend starts the copies of a pass (the first one's while
// the tile is computed), fp_add_staged waits for them.
// (a copy takes 16 bytes, or 4: two 16-bit elements; rows of 16-bit elements that start in between are read by the lanes themselves)
template <typename TO>
__device__ __forceinline__ void fp_fetch_addend(const ProductParams& p, int row0, int col0, int c, float4* st, int lane) {
    constexpr int V = 16 / sizeof(TO), FOUR = 4 / (int)sizeof(TO);
    const TO* const add = static_cast<const TO*>(p.addend);
    if (p.vec) {
        const int unit = lane & 7, col = col0 + c + V * unit;
        const int bytes = min(V, (int)p.N - col) * (int)sizeof(TO);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = j * 4 + (lane >> 3), row = row0 + r;
            if (row < p.M && bytes > 0)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(st + r * 8 + (unit ^ (r & 7)))), "l"(add + row * p.ld_addend + col),
                             "r"(bytes) : "memory");
        }
    } else if (sizeof(TO) == 4 || p.twos) {
        fp_each<TO, 128, FOUR>(p, row0, col0 + c, st, lane, [&](int row, int col, TO* at) { fp_copy4(smem_u32(at), reinterpret_cast<const float*>(add + row * p.ld_addend + col)); });
    } else {
        fp_each<TO, 128, 1>(p, row0, col0 + c, st, lane, [&](int row, int col, TO* at) { *at = add[row * p.ld_addend + col]; });
    }
}
template <typename TO>
__device__ __forceinline__ void fp_add_staged(const ProductParams& p, int row0, int col0, uint64_t (&acc)[FP_COLS / 2], float4* st, int lane) {
    constexpr int V = 16 / sizeof(TO), PASS = 128 / sizeof(TO);
#pragma unroll
    for (int c = 0; c < FP_COLS; c += PASS) {
        if (c > 0) fp_fetch_addend<TO>(p, row0, col0, c, st, lane);
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 w = st[lane * 8 + (i ^ (lane & 7))];
            const Pack<TO, V> a = *reinterpret_cast<const Pack<TO, V>*>(&w);
#pragma unroll
            for (int e = 0; e < V; e += 2) acc[(c + i * V + e) / 2] = add2(acc[(c + i * V + e) / 2], pair(to_float(a.v[e]), to_float(a.v[e + 1])));
        }
        __syncwarp();
    }
}
// Or a lane reads its own row, a 32-byte sector at a time (fetched into L2 when the tile began).
template <typename TO>
__device__ __forceinline__ void fp_add_rows(const ProductParams& p, int row, int col0, uint64_t (&acc)[FP_COLS / 2]) {
    constexpr int V = 16 / sizeof(TO);
    if (row >= p.M) return;
    const TO* const add = static_cast<const TO*>(p.addend) + row * p.ld_addend + col0;
    if (p.vec && col0 + FP_COLS <= p.N) {
#pragma unroll
        for (int c = 0; c < FP_COLS; c += V) {
            const Pack<TO, V> a = *reinterpret_cast<const Pack<TO, V>*>(add + c);
#pragma unroll
            for (int e = 0; e < V; e += 2) acc[(c + e) / 2] = add2(acc[(c + e) / 2], pair(to_float(a.v[e]), to_float(a.v[e + 1])));
        }
    } else {
#pragma unroll
        for (int c = 0; c < FP_COLS; ++c) {
            if (col0 + c < p.N) acc[c / 2] = add2(acc[c / 2], c & 1 ? pair(0.f, to_float(add[c])) : pair(to_float(add[c]), 0.f));
        }
    }
}
template <typename TO>
__device__ __forceinline__ void fp_prefetch_addend(const ProductParams& p, int row, int col0) {
    if (row >= p.M) return;
    const char* add = reinterpret_cast<const char*>(static_cast<const TO*>(p.addend) + row * p.ld_addend + col0);
#pragma unroll
    for (int b = 0; b < FP_COLS * (int)sizeof(TO); b += 128)
        if (col0 + b / (int)sizeof(TO) < p.N) asm volatile("prefetch.global.L2 [%0];" ::"l"(add + b));
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ float4 cluster_ld(uint32_t addr, uint32_t rank) {
    uint32_t at;
    float4 v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}

// A cluster's CTAs hold partial sums of one tile in their shared memory; each adds up a share of it in the order of their ranks.
template <typename TO>
__device__ __forceinline__ void fp_join(const ProductParams& p, uint32_t part, int m0, int n0, int tid) {
    const int rows = min(FP_BM, (int)p.M - m0);
    const uint32_t size = cluster_size();
    constexpr int THREADS = 32 * fp_epi_warps(FP_SPLIT), PER_ROW = fp_bn(FP_SPLIT) / 4;
    for (int u = (int)cluster_rank() * THREADS + tid; u < rows * PER_ROW; u += (int)size * THREADS) {
        const int r = u / PER_ROW, q = u % PER_ROW, row = m0 + r, col = n0 + 4 * q;
        if (col >= p.N) continue;
        float4 v[FP_MAX_SPLIT];
#pragma unroll
        for (int z = 0; z < FP_MAX_SPLIT; ++z) v[z] = z < (int)size ? cluster_ld(part + (uint32_t)(r * PER_ROW + (q ^ (r & 7))) * 16, z) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int z = 1; z < FP_MAX_SPLIT; ++z) { v[0].x += v[z].x; v[0].y += v[z].y; v[0].z += v[z].z; v[0].w += v[z].w; }
        float f[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
        Pack<TO, 4> o;
        if (p.addend) {
            const TO* add = static_cast<const TO*>(p.addend) + row * p.ld_addend + col;
#pragma unroll
            for (int e = 0; e < 4; ++e) if (col + e < p.N) f[e] += to_float(add[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o.v[e] = from_float<TO>(f[e]);
        fp_put<TO, 4>(p, row, col, o);
    }
}

// A 128 x BN tile of C at a time (persistent CTAs), or one per cluster, whose CTAs share its blocks of K (SPLIT).  Warp 0 feeds a
// ring of shared-memory stages by TMA, warp 1 issues the MMAs of one block of 128 k into one of two accumulators in tensor memory,
// warp 2 looks whether two of a block's scales may multiply to a number that is not normal, the other warps, 64 columns each, multiply
// finished block sums by their scales and add them up in registers (the tensor cores cannot carry an fp32 scale from block to block).
template <int FORM>
__global__ void __launch_bounds__(fp_threads(FORM), fp_ctas_per_sm(FORM)) fp8_product_kernel(const __grid_constant__ CUtensorMap tmA,
                                                                                              const __grid_constant__ CUtensorMap tmB,
                                                                                              const __grid_constant__ ProductParams p) {
    constexpr bool SPLIT = FORM == FP_SPLIT;
    constexpr int BN = fp_bn(FORM), STAGES = fp_stages(FORM), EW = fp_epi_warps(FORM), SLOTS = fp_slots(FORM), STORE_ROW = fp_store_row(FORM);
    constexpr uint32_t STAGE = fp_stage_bytes(FORM), TMEM_COLS = FP_NACC * BN;
    // registers per thread as launched (20 warps x 96, 12 x 80 twice, 8 x 80 three times, or 12 x 168), and how they are shared out: the epilogue's 64 sums
    // and 32 loaded values do not fit the launch's share
    constexpr int REGS = FORM == FP_WIDE ? 96 : (FORM == FP_SPLIT ? 168 : 80), REGS_CONTROL = 32;
    constexpr int REGS_EPI = FORM == FP_SPLIT ? 168 : REGS + 4 * (REGS - REGS_CONTROL) / EW / 8 * 8;
    static_assert(4 * REGS_CONTROL + EW * REGS_EPI <= (4 + EW) * REGS, "register shares exceed the launch's");
    extern __shared__ __align__(1024) unsigned char fp_smem[];
    float4* const stores = reinterpret_cast<float4*>(fp_smem + (size_t)STAGES * STAGE);
    float* const scales = reinterpret_cast<float*>(fp_smem + (size_t)STAGES * STAGE + EW * 32 * STORE_ROW);     // per slot: 128 of A, BN of B
    uint64_t* full = reinterpret_cast<uint64_t*>(scales + SLOTS * (128 + BN));
    uint64_t* empty = full + STAGES;
    uint64_t* acc_full = empty + STAGES;
    uint64_t* acc_empty = acc_full + FP_NACC;
    uint64_t* done = acc_empty + FP_NACC;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
    volatile uint32_t* stop = tmem_slot + 1;
    volatile uint32_t* filled = tmem_slot + 2;
    volatile uint32_t* looked = tmem_slot + 3;
    volatile uint32_t* far = tmem_slot + 4;        // [SLOTS] a product of two of the block's scales may not be a normal number
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 34); mbar_init(&empty[s], 1); }
        for (int b = 0; b < FP_NACC; ++b) { mbar_init(&acc_full[b], 2); mbar_init(&acc_empty[b], EW); }
        mbar_init(done, 1);
        *stop = 0;
        mbar_init_fence();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fp_fence_before();
    __syncthreads();
    fp_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_dependency_wait();          // (nothing of global memory was touched so far)
    allow_dependents();

    const int step = SPLIT ? p.items : (int)gridDim.x;
    const int first = SPLIT ? (int)(blockIdx.x / cluster_size()) : (int)blockIdx.x;
    const int kb0 = SPLIT ? (int)cluster_rank() * p.kper : 0, kb1 = SPLIT ? min(p.kblocks, kb0 + p.kper) : p.kblocks;

    if (warp < 4) {
        registers_down<REGS_CONTROL>();
        if (warp == 0) {
            // lane 0 the operands, all lanes the scales (four bytes each: a row of scales may begin anywhere)
            uint32_t s = 0, phase = 1, count = 0, slot = 0;
            bool ok = true;
            for (int item = first; item < p.items && ok; item += step) {
                const int m0 = item / p.tiles_n * FP_BM, n0 = item % p.tiles_n * BN;
                const float* const sa0 = p.sa + (p.a_square ? m0 >> 7 : m0 + lane);
                const float* const sb0 = p.sb + (p.b_square ? (n0 >> 7) + lane : n0 + lane);
                const int na = fp_scales_a(p, m0, lane), nb = fp_scales_b<BN>(p, n0, lane);
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = mbar_wait_idle(&empty[s], phase, p.wait_limit) && !*stop;
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) { if (lane == 0) { *stop = 1; note_status(p.status, KGE_ERR_TIMEOUT); } break; }
                    if (lane == 0) {
                        unsigned char* sa = fp_smem + s * STAGE;
                        mbar_arrive_expect_tx(&full[s], STAGE);
                        fp_tma_load(sa, &tmA, kb * FP_BK, m0, &full[s]);
    #pragma unroll
                        for (int g = 0; g < (BN + 127) / 128; ++g) fp_tma_load(sa + FP_BOX_BYTES * (1 + g), &tmB, kb * FP_BK, n0 + 128 * g, &full[s]);
                    }
                    const uint32_t at = smem_u32(scales + slot * (128 + BN) + lane);
    #pragma unroll
                    for (int i = 0; i < 4; ++i) if (32 * i < na) fp_copy4(at + 128 * i, sa0 + kb * p.sa_ld + 32 * i);
    #pragma unroll
                    for (int i = 0; i < BN / 32; ++i) if (32 * i < nb) fp_copy4(at + 512 + 128 * i, sb0 + kb * p.sb_ld + 32 * i);
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[s])) : "memory");
                    ++count;
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                    if (++slot == SLOTS) slot = 0;
                }
            }
            if (lane == 0) *filled = count;
            asm volatile("cp.async.wait_all;" ::: "memory");
        } else if (warp == 1) {
            if (lane == 0) {
                uint32_t s = 0, phase = 0, buf = 0, acc_phase = 1;
                bool ok = true;
                for (int item = first; item < p.items && ok && !*stop; item += step) {
                    for (int kb = kb0; kb < kb1; ++kb) {
                        if (!mbar_wait_idle(&acc_empty[buf], acc_phase, p.wait_limit) || !mbar_wait_idle(&full[s], phase, p.wait_limit)) { ok = false; break; }
                        fp_fence_after();
                        const uint32_t sa = smem_u32(fp_smem + s * STAGE);
    #pragma unroll
                        for (int k = 0; k < FP_BK / 32; ++k)
                            fp_mma(tmem + buf * BN, fp_desc(sa + k * 32), fp_desc(sa + FP_BOX_BYTES + k * 32), p.idesc, k != 0);
                        fp_commit(&empty[s]);
                        mbar_arrive(&acc_full[buf]);       // (hands on what the wait for the stage made visible: the scales)
                        fp_commit(&acc_full[buf]);
                        if (++s == STAGES) { s = 0; phase ^= 1; }
                        if (++buf == FP_NACC) { buf = 0; acc_phase ^= 1; }
                    }
                }
                if (!ok) { *stop = 1; note_status(p.status, KGE_ERR_TIMEOUT); }
            }
        } else if (warp == 2) {
            // looks at the scales of the blocks as they are loaded and leaves the epilogue one word for each (8192 x 4096 x 8192: 287 -> 291 us;
            // with a vote in the epilogue 320, with the MMAs' warp looking some 360)
            uint32_t s = 0, phase = 1, slot = 0, count = 0;
            bool ok = true;
            for (int item = first; item < p.items && ok; item += step) {
                const int m0 = item / p.tiles_n * FP_BM, n0 = item % p.tiles_n * BN;
                const float* const sa0 = p.sa + (p.a_square ? m0 >> 7 : m0 + lane);
                const float* const sb0 = p.sb + (p.b_square ? (n0 >> 7) + lane : n0 + lane);
                const int na = fp_scales_a(p, m0, lane), nb = fp_scales_b<BN>(p, n0, lane);
                float a[4], b[BN / 32];
                auto load = [&](int kb) {
    #pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] = 32 * i < na ? sa0[kb * p.sa_ld + 32 * i] : 1.f;
    #pragma unroll
                    for (int i = 0; i < BN / 32; ++i) b[i] = 32 * i < nb ? sb0[kb * p.sb_ld + 32 * i] : 1.f;
                };
                load(kb0);
                for (int kb = kb0; kb < kb1; ++kb) {
                    bool near = true;
    #pragma unroll
                    for (int i = 0; i < 4; ++i) near &= fp_near_one(a[i]);
    #pragma unroll
                    for (int i = 0; i < BN / 32; ++i) near &= fp_near_one(b[i]);
                    near = __all_sync(0xffffffffu, near);
                    if (kb + 1 < kb1) load(kb + 1);
                    ok = __all_sync(0xffffffffu, mbar_wait_idle(&empty[s], phase, p.wait_limit) && !*stop);
                    if (!ok) break;
                    if (lane == 0) { far[slot] = near ? 0u : 1u; mbar_arrive(&full[s]); }
                    ++count;
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                    if (++slot == SLOTS) slot = 0;
                }
            }
            if (lane == 0) { *looked = count; if (!ok) { *stop = 1; note_status(p.status, KGE_ERR_TIMEOUT); } }
        }
        __syncwarp();
        if (SPLIT) { cluster_sync(); cluster_sync(); }
    } else {
        registers_up<REGS_EPI>();
        const int quarter = warp & 3, group = (warp - 4) >> 2;      // tensor-memory lanes and columns of this warp
        float4* const st = stores + (warp - 4) * (32 * STORE_ROW / 16);
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(group * FP_COLS);
        uint32_t buf = 0, phase = 0, slot = 0;
        bool ok = true;
        for (int item = first; item < p.items && ok; item += step) {
            const int m0 = item / p.tiles_n * FP_BM + quarter * 32, n0 = item % p.tiles_n * BN + group * FP_COLS;
            uint64_t acc[FP_COLS / 2];
#pragma unroll
            for (int i = 0; i < FP_COLS / 2; ++i) acc[i] = 0ull;
            if (!SPLIT && p.addend) fp_with_out(p.out_type, [&](auto t) {
                using TO = decltype(t);
                if constexpr (STORE_ROW == 128) fp_fetch_addend<TO>(p, m0, n0, 0, st, lane);
                if (STORE_ROW != 128 || sizeof(TO) == 4) fp_prefetch_addend<TO>(p, m0 + lane, n0);
            });
#pragma unroll 1
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(&acc_full[buf], phase, p.wait_limit));
                fp_fence_after();
                if (!ok) { if (lane == 0) { *stop = 1; note_status(p.status, KGE_ERR_TIMEOUT); } break; }
                const uint32_t from = taddr + buf * BN;
                uint32_t v[2][16];
                fp_tmem_ld16(from, v[0]);
                const float* const sa = scales + slot * (128 + BN) + (p.a_square ? 0 : quarter * 32 + lane);
                const float* const sb = scales + slot * (128 + BN) + 128 + (p.b_square ? group * FP_COLS / 128 : group * FP_COLS);
                auto hand_back = [&] {                 // the accumulator is read: the next block's MMAs may begin
                    fp_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&acc_empty[buf]);
                };
                if (!far[slot]) {
                    const float s = p.b_square ? *sa * *sb : *sa;
                    const uint64_t s2 = pair(s, s);
#pragma unroll
                    for (int c = 0; c < FP_COLS / 16; ++c) {
                        fp_tmem_wait(v[c & 1]);
                        uint64_t w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = two_words(v[c & 1][2 * i], v[c & 1][2 * i + 1]);
                        if (c + 1 < FP_COLS / 16) fp_tmem_ld16(from + (uint32_t)(c + 1) * 16, v[(c + 1) & 1]);
                        else hand_back();
                        if (p.b_square) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) acc[c * 8 + i] = fma2(w[i], s2, acc[c * 8 + i]);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float4 b = reinterpret_cast<const float4*>(sb)[c * 4 + i];
                                acc[c * 8 + 2 * i] = fma2(w[2 * i], mul2(s2, pair(b.x, b.y)), acc[c * 8 + 2 * i]);
                                acc[c * 8 + 2 * i + 1] = fma2(w[2 * i + 1], mul2(s2, pair(b.z, b.w)), acc[c * 8 + 2 * i + 1]);
                            }
                        }
                    }
                } else {
                    const int each = p.b_square ? 0 : 1;
#pragma unroll
                    for (int c = 0; c < FP_COLS / 16; ++c) {
                        if (c > 0) fp_tmem_ld16(from + (uint32_t)c * 16, v[0]);
                        fp_tmem_wait(v[0]);
                        if (c + 1 == FP_COLS / 16) hand_back();
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            acc[c * 8 + i] = fp_add_far(two_words(v[0][2 * i], v[0][2 * i + 1]), *sa, sb[each * (c * 16 + 2 * i)], sb[each * (c * 16 + 2 * i + 1)], acc[c * 8 + i]);
                    }
                }
                if (++buf == FP_NACC) { buf = 0; phase ^= 1; }
                if (++slot == SLOTS) slot = 0;
            }
            if (!ok) break;
            if (SPLIT) {       // the ring's stages are free: every copy has been multiplied, every product read
                float4* part = reinterpret_cast<float4*>(fp_smem);
                const int r = quarter * 32 + lane;
#pragma unroll
                for (int i = 0; i < FP_COLS / 4; ++i) {
                    const float2 a = unpair(acc[2 * i]), b = unpair(acc[2 * i + 1]);
                    part[r * (BN / 4) + ((group * (FP_COLS / 4) + i) ^ (r & 7))] = make_float4(a.x, a.y, b.x, b.y);
                }
            } else {
                fp_with_out(p.out_type, [&](auto t) {
                    using TO = decltype(t);
                    if (p.addend) {
                        if constexpr (STORE_ROW == 128) fp_add_staged<TO>(p, m0, n0, acc, st, lane);
                        else fp_add_rows<TO>(p, m0 + lane, n0, acc);
                    }
                    fp_store<TO, STORE_ROW>(p, m0, n0, acc, st, lane);
                });
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");       // (an addend's copies, after a wait that ran out)
        if (SPLIT) {       // (every warp of the cluster comes here, also after a wait that ran out)
            cluster_sync();
            const int m0 = first / p.tiles_n * FP_BM, n0 = first % p.tiles_n * BN;
            fp_with_out(p.out_type, [&](auto t) { fp_join<decltype(t)>(p, smem_u32(fp_smem), m0, n0, threadIdx.x - 128); });
            cluster_sync();        // no CTA leaves while another reads its partial sums
        }
    }
    fp_fence_before();
    __syncthreads();
    if (*stop) {       // copies and MMAs in flight are waited for before the CTA's memory is given back (warp 2 may owe a stage its arrival)
        if (lane == 0) {
            if (warp == 0) {
                const int n = (int)*filled;
                for (int r = (int)*looked; r < n; ++r) mbar_arrive(&full[r % STAGES]);
                for (int r = max(0, n - STAGES); r < n; ++r) mbar_wait_idle(&full[r % STAGES], (r / STAGES) & 1, kDefaultWaitLimit);
            }
            if (warp == 1) { fp_commit(done); mbar_wait_idle(done, 0, kDefaultWaitLimit); }
        }
        __syncthreads();
    }
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int operand_map(CUtensorMap* map, const void* base, int64_t rows, int64_t k, int64_t ld, int box_rows) {
    static const EncodeTiledFn fn = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiledFn>(ptr) : nullptr;
    }();
    if (!fn) return KGE_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {FP_BK, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? KGE_OK : KGE_ERR_CUDA;
}

// Streaming multiprocessors of the current device.
int sm_count(int* sms) {
    static std::atomic<int> known[kMaxDevices];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return KGE_ERR_CUDA;
    const bool tracked = dev >= 0 && dev < kMaxDevices;
    *sms = tracked ? known[dev].load(std::memory_order_relaxed) : 0;
    if (*sms == 0) {
        e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return KGE_ERR_CUDA;
        if (tracked) known[dev].store(*sms, std::memory_order_relaxed);
    }
    return KGE_OK;
}

template <int FORM> int configure_product() {
    static DeviceOnce configured;
    return once_per_device(configured, [] {
        return cudaFuncSetAttribute(fp8_product_kernel<FORM>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)fp_smem_bytes(FORM));
    }) == cudaSuccess ? KGE_OK : KGE_ERR_CUDA;
}

std::atomic<int> product_wait_limit{kDefaultWaitLimit};       // tries of a bounded wait, unless a test shortens it

// How many clusters of `split` CTAs the device runs at a time: asked for once (what is left of a part of the chip takes none).
int split_clusters(int split, int* clusters) {
    static std::atomic<int> known[kMaxDevices][FP_MAX_SPLIT + 1];        // one more than their number
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return KGE_ERR_CUDA;
    const bool tracked = dev >= 0 && dev < kMaxDevices;
    int state = tracked ? known[dev][split].load(std::memory_order_acquire) : 0;
    if (state == 0) {
        const int rc = configure_product<FP_SPLIT>();
        if (rc != KGE_OK) return rc;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)split); cfg.blockDim = dim3(fp_threads(FP_SPLIT)); cfg.dynamicSmemBytes = fp_smem_bytes(FP_SPLIT);
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)split; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 1;
        int fit = 0;
        if (cudaOccupancyMaxActiveClusters(&fit, fp8_product_kernel<FP_SPLIT>, &cfg) != cudaSuccess) { (void)cudaGetLastError(); fit = 0; }
        state = 1 + std::max(fit, 0);
        if (tracked) known[dev][split].store(state, std::memory_order_release);
    }
    *clusters = state - 1;
    return KGE_OK;
}

// How a product is cut up: columns of a tile, and CTAs that share a tile's blocks of K.
//   shared K      as many CTAs to a tile as run at a time (512 x 768 x 4096: six to each of 24 tiles, of which some wait, 16.0 us, four 9.3,
//                 one 16.2), where the blocks that a CTA is spared outweigh the join: a block takes 0.4 us, the join 0.4 + 2 for 128 rows
//                 (128 x 768 x 512: 5.8 us shared, 4.5 not; x 4096: 7.5 and 15.5; one row, 256 x 512: 4.2 and 4.9)
//   256 columns   where K is long and they fill the SMs (8192 x 4096 x 8192 bf16: 291 us, in pairs of 128 columns 334; 4096 x 4096 x 4096: 90
//                 and 96; 2048 x 4096 x 1024: no difference; 16,384 x 8192 x 512: 145 and 128)
//   64 columns    or pairs: 24,576 x 256 x 768 with an addend 18.2 and 21.2 us, 24,576 x 768 x 256 21.1 and 20.8, 500,000 x 256 x 768
//                 295 and 280
struct ProductPlan { int form, split; };
int product_plan(int64_t M, int64_t N, int kblocks, bool ragged_addend, int sms, ProductPlan* plan) {
    const int64_t tiles128 = ceil_div(M, FP_BM) * ceil_div(N, 128), tiles256 = ceil_div(M, FP_BM) * ceil_div(N, 256);
    for (int most = (int)std::min<int64_t>({FP_MAX_SPLIT, kblocks, sms / tiles128}); most > 1; --most) {
        const int per = (kblocks + most - 1) / most, split = (kblocks + per - 1) / per;          // every CTA has a block
        if (128 * (kblocks - per - 1) <= 5 * std::min<int64_t>(M, FP_BM)) break;
        int room = 0;
        const int rc = split_clusters(split, &room);
        if (rc != KGE_OK) return rc;
        if (tiles128 <= room) { *plan = {FP_SPLIT, split}; return KGE_OK; }
    }
    // (an addend whose rows are not whole 16-byte words passes through shared memory that the wide form has not: 187 us there, 149 in
    // pairs at 4096 x 4095 x 4096)
    if (tiles256 >= sms && kblocks >= 16 && !ragged_addend) { *plan = {FP_WIDE, 1}; return KGE_OK; }
    // few blocks of K: memory sets the pace, and what counts is how well whole rounds of tiles fill the SMs
    const int64_t pair = ceil_div(tiles128, 2 * sms) * 256, narrow = ceil_div(ceil_div(M, FP_BM) * ceil_div(N, 64), 3 * sms) * 192;
    *plan = {narrow < pair ? FP_NARROW : FP_PAIR, 1};
    return KGE_OK;
}

template <int FORM>
int launch_product(const CUtensorMap& a, const CUtensorMap& b, ProductParams& p, int split, int sms, cudaStream_t s) {
    constexpr size_t smem = fp_smem_bytes(FORM);
    static_assert((smem + 1024) * fp_ctas_per_sm(FORM) <= 228 * 1024, "shared memory of an SM");
    const int rc = configure_product<FORM>();
    if (rc != KGE_OK) return rc;
    p.tiles_n = (int)ceil_div(p.N, fp_bn(FORM));
    p.items = (int)(ceil_div(p.M, FP_BM) * p.tiles_n);
    p.kper = (p.kblocks + split - 1) / split;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(FORM == FP_SPLIT ? p.items * split : std::min<int64_t>(p.items, (int64_t)sms * fp_ctas_per_sm(FORM))));
    cfg.blockDim = dim3(fp_threads(FORM)); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = FORM == FP_SPLIT ? 2 : 1;
    return launch_status(cudaLaunchKernelEx(&cfg, fp8_product_kernel<FORM>, a, b, p));
}

}  // namespace
}  // namespace kge

using namespace kge;

extern "C" {

int kge_fp8_quantize(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx, int32_t fp8_type, int32_t block_rows, int32_t pow2,
                     void* q, int64_t ldq, float* scales, void* qt, int64_t ldqt, float* scales_t, void* stream) {
    if (!is_float_type(x_type) || !is_fp8_type(fp8_type) || rows < 0 || rows > INT32_MAX || cols < 0 || cols > INT32_MAX || ldx < cols ||
        (block_rows != 1 && block_rows != 128) || (pow2 != 0 && pow2 != 1) || (!q && !qt)) return KGE_ERR_BAD_ARG;
    if ((q && (!scales || ldq < cols || ldq % 16 || !aligned_to(q, 16) || !aligned_to(scales, 4))) ||
        (qt && (!scales_t || ldqt < rows || ldqt % 16 || !aligned_to(qt, 16) || !aligned_to(scales_t, 4)))) return KGE_ERR_BAD_ARG;
    if (rows == 0 || cols == 0) return KGE_OK;
    if (!x || !aligned_to(x, type_bytes(x_type))) return KGE_ERR_BAD_ARG;
    QuantParams p{};
    p.x = x; p.ldx = ldx; p.rows = rows; p.cols = cols;
    p.q = static_cast<uint8_t*>(q); p.ldq = ldq; p.scales = scales;
    p.qt = static_cast<uint8_t*>(qt); p.ldqt = ldqt; p.scales_t = scales_t;
    p.pow2 = pow2; p.tiles_c = ceil_div(cols, 128);
    p.vec = aligned_to(x, 16) && ldx * type_bytes(x_type) % 16 == 0;
    if (p.tiles_c * ceil_div(rows, 128) > INT32_MAX) return KGE_ERR_UNSUPPORTED;
    return with_type(x_type, [&](auto t) { return launch_quantize<decltype(t)>(p, fp8_type, block_rows == 128, static_cast<cudaStream_t>(stream)); });
}

int kge_fp8_matmul(const void* a, int32_t a_type, int64_t lda, const float* a_scales, int32_t a_block, const void* b, int32_t b_type, int64_t ldb,
                   const float* b_scales, int32_t b_block, const void* addend, int64_t ld_addend, void* out, int32_t out_type, int64_t ld_out,
                   int64_t M, int64_t N, int64_t K, int32_t* status, void* stream) {
    if (!is_fp8_type(a_type) || !is_fp8_type(b_type) || !is_float_type(out_type) || (a_block != 1 && a_block != 128) || (b_block != 1 && b_block != 128) ||
        M < 0 || N < 0 || K < 1 || M > INT32_MAX - 256 || N > INT32_MAX - 256 || K > INT32_MAX - 256 || ld_out < N || (addend && ld_addend < N))
        return KGE_ERR_BAD_ARG;
    if (M == 0 || N == 0) return KGE_OK;
    if (!a || !b || !a_scales || !b_scales || !out || lda < K || ldb < K || lda % 16 || ldb % 16 || !aligned_to(a, 16) || !aligned_to(b, 16) ||
        !aligned_to(a_scales, 4) || !aligned_to(b_scales, 4) || !aligned_to(out, type_bytes(out_type)) ||
        (addend && !aligned_to(addend, type_bytes(out_type))) || !aligned_to(status, 4)) return KGE_ERR_BAD_ARG;
    ProductParams p{};
    p.M = M; p.N = N; p.kblocks = (int)ceil_div(K, FP_BK);
    p.sa = a_scales; p.sb = b_scales; p.a_square = a_block == 128; p.b_square = b_block == 128;
    p.sa_ld = p.a_square ? ceil_div(M, 128) : M; p.sb_ld = p.b_square ? ceil_div(N, 128) : N;
    p.addend = addend; p.ld_addend = ld_addend; p.out = out; p.ld_out = ld_out; p.out_type = out_type;
    const int ob = type_bytes(out_type);
    p.vec = ld_out * ob % 16 == 0 && aligned_to(out, 16) && (!addend || (ld_addend * ob % 16 == 0 && aligned_to(addend, 16)));
    p.twos = N % 2 == 0 && ld_out % 2 == 0 && aligned_to(out, 2 * ob) && (!addend || (ld_addend % 2 == 0 && aligned_to(addend, 2 * ob)));
    p.status = status; p.wait_limit = product_wait_limit.load(std::memory_order_relaxed);
    int sms = 0, rc = sm_count(&sms);
    if (rc != KGE_OK) return rc;
    if (ceil_div(M, 128) * ceil_div(N, 64) > INT32_MAX / 8) return KGE_ERR_UNSUPPORTED;
    ProductPlan plan;
    rc = product_plan(M, N, p.kblocks, addend && !p.vec, sms, &plan);
    if (rc != KGE_OK) return rc;
    alignas(64) CUtensorMap ma, mb;
    rc = operand_map(&ma, a, M, K, lda, FP_BM);
    if (rc == KGE_OK) rc = operand_map(&mb, b, N, K, ldb, fp_box_rows(plan.form));
    if (rc != KGE_OK) return rc;
    p.idesc = fp_idesc(FP_BM, fp_bn(plan.form), a_type == KGE_E5M2, b_type == KGE_E5M2);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (plan.form) {
        case FP_SPLIT: return launch_product<FP_SPLIT>(ma, mb, p, plan.split, sms, s);
        case FP_WIDE: return launch_product<FP_WIDE>(ma, mb, p, 1, sms, s);
        case FP_NARROW: return launch_product<FP_NARROW>(ma, mb, p, 1, sms, s);
        default: return launch_product<FP_PAIR>(ma, mb, p, 1, sms, s);
    }
}

int kge_debug_set_product_wait_limit(int32_t tries) {
    if (tries < 0) return KGE_ERR_BAD_ARG;
    product_wait_limit.store(tries == 0 ? kDefaultWaitLimit : tries, std::memory_order_relaxed);
    return KGE_OK;
}

}  // extern "C"
