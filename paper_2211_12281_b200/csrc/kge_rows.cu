// Rows of a table for a list of ids, times a scale, and the gradient of that.
//   lookup    out[i] = scale T[ids[i]]
//   gradient  dT[e] = scale sum_{i : ids[i] = e} g[i]      (+ the old dT[e])
// The gradient sorts the ids (stable radix sort of (id, position) pairs), walks the sorted list in chunks of rows, adds a chunk's
// rows of one id in fp32 in ascending position, and joins the ids that span chunks in a second, fixed order: what is added to what
// follows from the ids, their number, the table's rows and the width alone.  Rows of the dense gradient that no id names are set to zero by CTAs beside the sort's.
//   short lists         one launch: every CTA owns a range of table rows, picks the ids that fall into it and sorts those
//   up to 65,536        one cluster of sixteen CTAs sorts in shared memory, exchanging counts and pairs between its CTAs
//   more                hist     digit counts of every tile, per pass (counted by atomics while the pass before scatters, frequent ids cost 12 us of 24)
//                       scan     the counts become sums over the tiles before
//                       scatter  one stable split by a digit
//   then                sum      chunks of sorted rows; what ends inside its chunk or the next one is final, the rest leaves partial sums
//                       join     one CTA per (id that spans more, 64 columns): partial sums in a fixed order
#include <algorithm>
#include <type_traits>

#include "kge_ops.cuh"

namespace kge {

namespace {

// ---- lookup ----------------------------------------------------------------------------------------------------------

struct LookupParams {
    const void* table; void* out;
    const int32_t* ids;
    int64_t rows, ld_table, ld_out;
    int n, dim, rows_per_cta;
    int32_t padding_id;
    float scale;
    FastDiv vecs;                 // packs per row (of four single elements in lookup_single_kernel)
    int32_t* status;
};

constexpr int LOOKUP_THREADS = 256, LOOKUP_UNROLL = 4;

// Bound by memory: 24,576 x 200 fp32 rows of a table of 1.6 GB in 5.5 us (7.1 TB/s, part of it out of L2).
template <typename TT, typename TO, int V>
__global__ void __launch_bounds__(LOOKUP_THREADS) lookup_kernel(LookupParams p) {
    grid_dependency_wait();
    allow_dependents();
    const TT* table = static_cast<const TT*>(p.table);
    TO* out = static_cast<TO*>(p.out);
    const int r0 = blockIdx.x * p.rows_per_cta, nr = min(p.rows_per_cta, p.n - r0);
    const uint32_t items = (uint32_t)nr * p.vecs.d;
    for (uint32_t i0 = threadIdx.x; i0 < items; i0 += LOOKUP_THREADS * LOOKUP_UNROLL) {
        Pack<TT, V> v[LOOKUP_UNROLL];
        int row[LOOKUP_UNROLL];
        uint32_t col[LOOKUP_UNROLL];
#pragma unroll
        for (int u = 0; u < LOOKUP_UNROLL; ++u) {
            const uint32_t i = i0 + u * LOOKUP_THREADS;
            row[u] = -1;
            if (i < items) {
                const uint32_t r = p.vecs.div(i);
                col[u] = i - r * p.vecs.d;
                row[u] = r0 + (int)r;
                const int32_t id = p.ids[row[u]];
                const bool in = id >= 0 && id < p.rows;
                if (in && id != p.padding_id) v[u] = *reinterpret_cast<const Pack<TT, V>*>(table + id * p.ld_table + (int64_t)col[u] * V);
                else {
                    if (!in && id != p.padding_id) note_status(p.status, KGE_ERR_ID_RANGE);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[u].v[e] = from_float<TT>(0.f);
                    row[u] = ~row[u] - 1;     // a zero row, whatever the scale
                }
            }
        }
#pragma unroll
        for (int u = 0; u < LOOKUP_UNROLL; ++u) {
            if (row[u] == -1) continue;
            const bool zero = row[u] < -1;
            const int64_t r = zero ? ~(row[u] + 1) : row[u];
            Pack<TO, V> o;
#pragma unroll
            for (int e = 0; e < V; ++e) o.v[e] = from_float<TO>(zero ? 0.f : to_float(v[u].v[e]) * p.scale);
            *reinterpret_cast<Pack<TO, V>*>(out + r * p.ld_out + (int64_t)col[u] * V) = o;
        }
    }
}

// Rows that are no whole packs: four single elements an item, so that finding an item's row and place is shared by four.  With a 16-bit side
// rows back to back are put together in shared memory and stored as whole words (351,964 x 45 bf16: to fp16 28 -> 21 us, to fp32 36 -> 22;
// fp32 to fp32 it would cost, 19 -> 22).
template <typename TT, typename TO>
__global__ void __launch_bounds__(LOOKUP_THREADS) lookup_single_kernel(LookupParams p) {
    constexpr bool STAGED = sizeof(TT) == 2 || sizeof(TO) == 2;
    constexpr int MOST = LOOKUP_THREADS * LOOKUP_UNROLL, W = 16 / (int)sizeof(TO);
    __shared__ alignas(16) TO stage[STAGED ? MOST * 4 + W : 1];
    grid_dependency_wait();
    allow_dependents();
    const TT* table = static_cast<const TT*>(p.table);
    TO* out = static_cast<TO*>(p.out);
    const int r0 = blockIdx.x * p.rows_per_cta, nr = min(p.rows_per_cta, p.n - r0);
    const uint32_t items = (uint32_t)nr * p.vecs.d;
    TO* const first = out + r0 * p.ld_out;
    const bool flat = STAGED && p.ld_out == p.dim && items <= MOST;
    const int shift = (int)((reinterpret_cast<uintptr_t>(first) & 15) / sizeof(TO));       // elements of the first word that are not this CTA's
    for (uint32_t i = threadIdx.x; i < items; i += LOOKUP_THREADS) {
        const uint32_t r = p.vecs.div(i), col = (i - r * p.vecs.d) * 4;
        const int row = r0 + (int)r, m = min(4, p.dim - (int)col);
        const int32_t id = p.ids[row];
        const bool in = id >= 0 && id < p.rows, real = in && id != p.padding_id;
        if (!in && id != p.padding_id) note_status(p.status, KGE_ERR_ID_RANGE);
        const TT* src = table + (real ? id : 0) * p.ld_table + col;
        TO* dst = flat ? stage + shift + (int)r * p.dim + (int)col : out + row * p.ld_out + col;
        TT v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = src[e < m ? e : 0];
#pragma unroll
        for (int e = 0; e < 4; ++e) if (e < m) dst[e] = from_float<TO>(real ? to_float(v[e]) * p.scale : 0.f);
    }
    if constexpr (STAGED) {
        if (!flat) return;
        __syncthreads();
        const int end = shift + nr * p.dim;
        for (int w = threadIdx.x * W; w < end; w += LOOKUP_THREADS * W) {
            TO* const dst = first + (w - shift);
            if (w >= shift && w + W <= end) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(stage + w);
            else {
                for (int e = 0; e < W; ++e) if (w + e >= shift && w + e < end) dst[e] = stage[w + e];
            }
        }
    }
}

// ---- gradient --------------------------------------------------------------------------------------------------------

constexpr int GS_THREADS = 256, GS_WARPS = GS_THREADS / 32, GS_ITEMS = 8;
constexpr int GS_TILE = GS_THREADS * GS_ITEMS;     // ids per CTA of the sort in global memory
constexpr int GS_MAX_BITS = 9;
constexpr int CS_CTAS = 16, CS_CTAS_PORTABLE = 8, CS_THREADS = 512, CS_WARPS = CS_THREADS / 32, CS_ITEMS = 16;      // the cluster's sort
// (At 128 columns 65,536 ids take 33.5 us with the cluster, 65,537 with the sort in global memory 31.8: about where they meet, and where
// a cluster of eight has no room for more.)
constexpr int CS_SHARE = CS_THREADS * CS_ITEMS, CS_MAX = CS_CTAS_PORTABLE * CS_SHARE, CS_MAX_BITS = 11;
constexpr int SMALL_MAX = 2048, SMALL_THREADS = 256, SMALL_BITS = 11;      // (SMALL_BITS: of a position)
static_assert(SMALL_MAX == 1 << SMALL_BITS, "positions of a short list");
constexpr int SUM_THREADS = 256;
constexpr int JOIN_THREADS = 256;
constexpr int GRAD_MAX_DIM = INT32_MAX - 1024;    // columns are counted in 32 bits, up to 256 past the last one

struct SortPlan { int tiles, key_bits, passes, bits; };

SortPlan sort_plan(int64_t rows, int n) {
    SortPlan s;
    s.tiles = (int)ceil_div(n, GS_TILE);
    s.key_bits = 1;
    while (s.key_bits < 31 && (1ll << s.key_bits) <= rows) ++s.key_bits;      // keys 0 .. rows (rows: no row of the table)
    const int most = n <= CS_MAX ? CS_MAX_BITS : GS_MAX_BITS;
    s.passes = (s.key_bits + most - 1) / most;
    s.bits = (s.key_bits + s.passes - 1) / s.passes;
    return s;
}
// One CTA adds up all rows of an id, so longer lists go this way only where ids can be expected to differ: 2,048 rows of 1 KB take 8.9
// us against 13.8 with the sort if they do, 53 against 15 if all are one id's (1,024: 29 against 15).
bool short_list(int64_t rows, int n) { return n <= SMALL_MAX / 2 || (n <= SMALL_MAX && rows >= 4ll * n); }
// Rows to a thread of grad_sum_kernel: few where there would be too few threads (24,576 x 128: 23.7 us a call with 8, 28.2 with 32; 131,071 x
// 256: 70 and 74), else enough that the partial sums of frequent ids stay few (500,000 x 256, sum + join: 66 + 21 us with 32, 61 + 38 with
// 16, 79 + 13 with 64).
int chunk_rows(int n) { return n < (1 << 17) ? 8 : 32; }

// In what order an id's rows are added must follow from the ids, the list's and the table's length and the width: not from the packs that
// the types and the rows' alignment allow.  So the sizes of what is added together first are functions of the width: chunks that a CTA
// joins (a power of two; its threads are whole groups whatever the pack, at most 1,024 of them), and stripes of a run in a short list.
// (Groups of 2,048 columns instead of 1,024, which single columns' threads cannot hold: 300,000 x 256 bf16 of one id 64 us, with 1,024 71.)
int group_chunks(int dim) { return 1024 % dim == 0 ? std::min(1024 / dim, SUM_THREADS) : 1; }
int run_stripes(int dim) {
    const int pack = dim % 8 == 0 ? 8 : (dim % 4 == 0 ? 4 : (dim % 2 == 0 ? 2 : 1));
    return SMALL_THREADS / std::min(dim / pack, SMALL_THREADS);
}

struct GradScratch {
    uint2* pairs[2];                 // [n] (id, position) in the order of a pass, in turn
    uint32_t* hist;                  // [tiles][1 << bits]
    uint32_t* total;                 // [1 << bits]
    float* part;                     // [chunks][2][dim rounded up to 4]
    int2* list; int32_t* list_count; // (chunk in which an id begins that spans more, id)
    size_t bytes;
};

GradScratch carve_grad(char* base, int64_t rows, int dim, int n) {
    size_t used = 0;
    auto take = [&](size_t bytes) { char* q = base ? base + used : nullptr; used += (bytes + 255) / 256 * 256; return q; };
    const SortPlan s = sort_plan(rows, n);
    const int64_t chunks = ceil_div(n, chunk_rows(n));
    GradScratch g{};
    if (short_list(rows, n)) return g;       // (one launch: nothing is kept)
    for (int i = 0; i < (n > CS_MAX ? 2 : 1); ++i) g.pairs[i] = reinterpret_cast<uint2*>(take((size_t)n * 8));
    if (n > CS_MAX) {
        g.hist = reinterpret_cast<uint32_t*>(take((size_t)s.tiles * (4u << s.bits)));
        g.total = reinterpret_cast<uint32_t*>(take((size_t)4 << s.bits));
    }
    g.part = reinterpret_cast<float*>(take((size_t)chunks * 2 * ((dim + 3) / 4 * 4) * 4));
    g.list = reinterpret_cast<int2*>(take((size_t)chunks * 8));
    g.list_count = reinterpret_cast<int32_t*>(take(256));
    g.bytes = used;
    return g;
}

struct SortParams {
    const int32_t* ids;
    int n, tiles, bits, shift, pass, passes;
    uint32_t rows;
    int32_t padding_id;
    const uint2* pairs_in;
    uint2* pairs_out;
    uint32_t *hist, *total;               // [tiles][1 << bits] counts of a pass, then sums over the tiles before; [1 << bits]
    int32_t *list_count, *status;
    // dense gradient rows set to zero by CTAs beside the sort's
    char* zero; int64_t zero_row_bytes, zero_ld_bytes, zero_first, zero_last;     // the rows, and which of them in this launch
    int zero_flat;                        // the rows lie back to back
};

__device__ __forceinline__ uint32_t grad_key(const SortParams& p, int32_t id) {
    if (id == p.padding_id) return p.rows;
    if (id < 0 || (uint32_t)id >= p.rows) { note_status(p.status, KGE_ERR_ID_RANGE); return p.rows; }
    return (uint32_t)id;
}

// Bytes [base, base + all) (whole 16-bit elements) set to zero by thread `first` of `step`.
__device__ __forceinline__ void zero_bytes(char* base, int64_t all, int64_t first, int64_t step) {
    const int64_t head = min(all, (int64_t)(-reinterpret_cast<intptr_t>(base) & 15)), words = (all - head) / 16;
    uint4* z = reinterpret_cast<uint4*>(base + head);
#pragma unroll 4
    for (int64_t i = first; i < words; i += step) z[i] = make_uint4(0u, 0u, 0u, 0u);
    for (int64_t i = 2 * first; i < head; i += 2 * step) *reinterpret_cast<uint16_t*>(base + i) = 0;
    for (int64_t i = head + words * 16 + 2 * first; i < all; i += 2 * step) *reinterpret_cast<uint16_t*>(base + i) = 0;
}
// Rows apart: a warp to a row, or, where a warp would mostly idle, a thread to an element (55,864 x 496 fp32, 504 apart, and 3,010 ids: 31 to
// 34 us, element by element 281).
__device__ __forceinline__ void zero_strided(char* base, int64_t rows, int64_t row_bytes, int64_t ld_bytes, int64_t first, int64_t step) {
    if (row_bytes >= 64) {
        for (int64_t r = first >> 5; r < rows; r += step >> 5) zero_bytes(base + r * ld_bytes, row_bytes, first & 31, 32);
        return;
    }
    const int unit = ((reinterpret_cast<intptr_t>(base) | row_bytes | ld_bytes) & 3) == 0 ? 4 : 2, units = (int)row_bytes / unit;
    for (int64_t i = first; i < rows * units; i += step) {
        const int64_t r = i >> 32 ? i / units : (uint32_t)i / (uint32_t)units;
        char* const at = base + r * ld_bytes + (i - r * units) * unit;
        if (unit == 4) *reinterpret_cast<uint32_t*>(at) = 0;
        else *reinterpret_cast<uint16_t*>(at) = 0;
    }
}
// Rows [zero_first, zero_last) by CTA `cta` of `ctas`.
__device__ __forceinline__ void zero_rows(const SortParams& p, int64_t cta, int64_t ctas) {
    const int64_t first = cta * blockDim.x + threadIdx.x, step = ctas * blockDim.x, rows = p.zero_last - p.zero_first;
    char* const base = p.zero + p.zero_first * p.zero_ld_bytes;
    if (p.zero_flat) zero_bytes(base, rows * p.zero_row_bytes, first, step);
    else zero_strided(base, rows, p.zero_row_bytes, p.zero_ld_bytes, first, step);
}

// The lanes (of those that are `in`) that hold this lane's digit of at most BITS bits: a vote per bit, all of them independent.
template <int BITS>
__device__ __forceinline__ unsigned same_digit(uint32_t digit, bool in) {
    unsigned same = __ballot_sync(0xffffffffu, in);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const bool one = digit >> b & 1;
        const unsigned v = __ballot_sync(0xffffffffu, one);
        same &= one ? v : ~v;
    }
    return same;
}

__global__ void __launch_bounds__(GS_THREADS) grad_hist_kernel(SortParams p) {
    __shared__ uint32_t count[1 << GS_MAX_BITS];
    grid_dependency_wait();
    allow_dependents();
    const int digits = 1 << p.bits, tid = threadIdx.x;
    if ((int)blockIdx.x >= p.tiles) { zero_rows(p, blockIdx.x - p.tiles, gridDim.x - p.tiles); return; }
    for (int d = tid; d < digits; d += GS_THREADS) count[d] = 0;
    if (blockIdx.x == 0 && tid == 0) *p.list_count = 0;
    __syncthreads();
    uint32_t v[GS_ITEMS];
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        const int64_t i = min((int64_t)blockIdx.x * GS_TILE + k * GS_THREADS + tid, (int64_t)p.n - 1);
        v[k] = load_now<uint32_t>(p.pass == 0 ? reinterpret_cast<const uint32_t*>(p.ids) + i : &p.pairs_in[i].x);
    }
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) asm volatile("" ::"r"(v[k]));
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        const int64_t i = (int64_t)blockIdx.x * GS_TILE + k * GS_THREADS + tid;
        if (i < p.n) atomicAdd(&count[((p.pass == 0 ? grad_key(p, (int32_t)v[k]) : v[k]) >> p.shift) & (digits - 1)], 1u);
    }
    __syncthreads();
    for (int d = tid; d < digits; d += GS_THREADS) p.hist[(int64_t)blockIdx.x * digits + d] = count[d];
}

// A warp per digit turns the tiles' counts into sums over the tiles before.
__global__ void __launch_bounds__(256) grad_scan_kernel(SortParams p) {
    grid_dependency_wait();
    allow_dependents();
    const int digits = 1 << p.bits, d = (blockIdx.x * 256 + threadIdx.x) >> 5, lane = threadIdx.x & 31;
    if (d >= digits) return;
    uint32_t run = 0;
    for (int t0 = 0; t0 < p.tiles; t0 += 256) {
        uint32_t c[8], sum = 0;                     // lane l: tiles t0 + 8 l ... + 8
#pragma unroll
        for (int u = 0; u < 8; ++u) { const int t = t0 + 8 * lane + u; c[u] = t < p.tiles ? p.hist[(int64_t)t * digits + d] : 0u; }
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += c[u];
        uint32_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
        uint32_t at = run + incl - sum;
#pragma unroll
        for (int u = 0; u < 8; ++u) { const int t = t0 + 8 * lane + u; if (t < p.tiles) p.hist[(int64_t)t * digits + d] = at; at += c[u]; }
        run += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) p.total[d] = run;
}

// Stable split of one tile by a digit: a warp takes its 256 elements 32 at a time in order, lanes of one digit find each other
// by a vote and a running count per (warp, digit) carries over; the warps' counts and the tiles' give every element its place.
__global__ void __launch_bounds__(GS_THREADS) grad_scatter_kernel(SortParams p) {
    __shared__ uint16_t cnt[GS_WARPS][1 << GS_MAX_BITS];
    __shared__ uint32_t base[1 << GS_MAX_BITS];
    __shared__ uint32_t warp_tot[GS_WARPS];
    const int digits = 1 << p.bits, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, tile = blockIdx.x;
    grid_dependency_wait();
    allow_dependents();
    if (tile >= p.tiles) { zero_rows(p, tile - p.tiles, gridDim.x - p.tiles); return; }
    for (int d = lane; d < digits; d += 32) cnt[warp][d] = 0;
    __syncwarp();
    uint32_t key[GS_ITEMS], pos[GS_ITEMS], at[GS_ITEMS];
    const int64_t i0 = (int64_t)tile * GS_TILE + warp * 32 * GS_ITEMS;
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        const int64_t i = min(i0 + k * 32 + lane, (int64_t)p.n - 1);
        if (p.pass == 0) { key[k] = load_now<uint32_t>(p.ids + i); pos[k] = (uint32_t)i; }
        else { const uint2 v = load_now<uint2>(p.pairs_in + i); key[k] = v.x; pos[k] = v.y; }
    }
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) asm volatile("" ::"r"(key[k]), "r"(pos[k]));
    if (p.pass == 0) {
#pragma unroll
        for (int k = 0; k < GS_ITEMS; ++k) if (i0 + k * 32 + lane < p.n) key[k] = grad_key(p, (int32_t)key[k]);
    }
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        const bool in = i0 + k * 32 + lane < p.n;
        const uint32_t digit = (key[k] >> p.shift) & (digits - 1);
        const unsigned same = same_digit<GS_MAX_BITS>(digit, in), before = same & ((1u << lane) - 1u);
        uint32_t seen = 0;
        if (in) seen = cnt[warp][digit];
        __syncwarp();
        if (in && before == 0) cnt[warp][digit] = (uint16_t)(seen + __popc(same));
        __syncwarp();
        at[k] = seen + __popc(before);
    }
    __syncthreads();
    // where this tile's share of a digit begins: the smaller digits of all tiles, and this one's in the tiles before
    const int per = max(1, digits / GS_THREADS), d0 = tid * per;
    constexpr int PER = (1 << GS_MAX_BITS) / GS_THREADS;
    uint32_t sum = 0, tot[PER], mine[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        tot[j] = mine[j] = 0;
        if (d0 < digits && j < per) { tot[j] = p.total[d0 + j]; mine[j] = p.hist[(int64_t)tile * digits + d0 + j]; }
        sum += tot[j];
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
    if (lane == 31) warp_tot[warp] = incl;
    __syncthreads();
    uint32_t run = incl - sum;
    for (int w = 0; w < warp; ++w) run += warp_tot[w];
    if (d0 < digits) {
#pragma unroll
        for (int j = 0; j < PER; ++j) if (j < per) {
            base[d0 + j] = run + mine[j];
            run += tot[j];
            uint32_t w_run = 0;
            for (int w = 0; w < GS_WARPS; ++w) { const uint32_t c = cnt[w][d0 + j]; cnt[w][d0 + j] = (uint16_t)w_run; w_run += c; }
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        if (i0 + k * 32 + lane >= p.n) continue;
        const uint32_t digit = (key[k] >> p.shift) & (digits - 1);
        const uint32_t dst = base[digit] + cnt[warp][digit] + at[k];
        p.pairs_out[dst] = make_uint2(key[k], pos[k]);
    }
}

// ---- up to 65,536 ids: one cluster sorts them in shared memory ----

__device__ __forceinline__ void cs_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cs_map(uint32_t addr, uint32_t rank) { uint32_t r; asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank)); return r; }
__device__ __forceinline__ uint32_t cs_load(uint32_t addr) { uint32_t v; asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory"); return v; }
__device__ __forceinline__ void cs_store2(uint32_t addr, uint32_t a, uint32_t b) { asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory"); }

size_t cluster_sort_smem(int n, int bits, int ctas) {       // pairs twice, warps' counts, digits' counts and bases
    return (size_t)ceil_div(n, ctas) * 16 + ((size_t)CS_WARPS * 2 + 8) * ((size_t)1 << bits) + 128;
}

// Cluster 0 sorts: each of its CTAs holds a share of the list, a warp a contiguous piece of that.  Per pass a warp ranks its elements
// among its own (as in grad_scatter_kernel), the CTAs read each other's digit counts, and every pair is stored into the CTA that
// holds its new place; the last pass stores to global memory.  The other clusters set rows to zero.  Bound by latency: two passes over
// 24,576 ids take 14 us, of which ids 2, ranks 2, counts of the other CTAs 3, scattered stores 3, barriers the rest.
template <int CTAS>
__global__ void __launch_bounds__(CS_THREADS, 1) grad_cluster_sort_kernel(SortParams p) {
    extern __shared__ __align__(16) unsigned char cs_smem[];
    grid_dependency_wait();
    allow_dependents();
    if (blockIdx.x >= CTAS) { zero_rows(p, blockIdx.x - CTAS, gridDim.x - CTAS); return; }
    __shared__ uint32_t warp_tot[CS_WARPS];
    const int digits = 1 << p.bits, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int share = (p.n + CTAS - 1) / CTAS, rank = blockIdx.x;
    const int have = max(0, min(share, p.n - rank * share));                        // of this CTA
    const int per_warp = ((share + CS_WARPS - 1) / CS_WARPS + 31) / 32 * 32;        // at most 32 CS_ITEMS
    uint2* const pairs[2] = {reinterpret_cast<uint2*>(cs_smem), reinterpret_cast<uint2*>(cs_smem) + share};
    uint32_t* const count = reinterpret_cast<uint32_t*>(pairs[1] + share);          // [digits] of this CTA
    uint32_t* const base = count + digits;                                          // [digits]
    uint16_t* const cnt = reinterpret_cast<uint16_t*>(base + digits);               // [CS_WARPS][digits]
    if (rank == 0 && tid == 0) *p.list_count = 0;
    const int rounds = per_warp / 32, first = warp * per_warp;
    uint32_t key[CS_ITEMS], pos[CS_ITEMS], at[CS_ITEMS];
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * p.bits;
        for (int d = lane; d < digits; d += 32) cnt[warp * digits + d] = 0;
        if (pass == 0) {
#pragma unroll
            for (int k = 0; k < CS_ITEMS; ++k) {
                pos[k] = (uint32_t)min((int64_t)rank * share + first + k * 32 + lane, (int64_t)p.n - 1);
                key[k] = k < rounds ? load_now<uint32_t>(reinterpret_cast<const uint32_t*>(p.ids) + pos[k]) : 0u;
            }
#pragma unroll
            for (int k = 0; k < CS_ITEMS; ++k) asm volatile("" ::"r"(key[k]));
#pragma unroll
            for (int k = 0; k < CS_ITEMS; ++k) if (k < rounds && first + k * 32 + lane < have) key[k] = grad_key(p, (int32_t)key[k]);
        } else {
#pragma unroll
            for (int k = 0; k < CS_ITEMS; ++k) {
                const int i = first + k * 32 + lane;
                if (k < rounds && i < have) { const uint2 v = pairs[pass & 1][i]; key[k] = v.x; pos[k] = v.y; }
            }
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < CS_ITEMS; ++k) {
            if (k >= rounds) break;
            const bool in = first + k * 32 + lane < have;
            const uint32_t digit = (key[k] >> shift) & (digits - 1);
            const unsigned same = same_digit<CS_MAX_BITS>(digit, in), before = same & ((1u << lane) - 1u);
            uint32_t seen = 0;
            if (in) seen = cnt[warp * digits + digit];
            __syncwarp();
            if (in && before == 0) cnt[warp * digits + digit] = (uint16_t)(seen + __popc(same));
            __syncwarp();
            at[k] = seen + __popc(before);
        }
        __syncthreads();
        for (int d = tid; d < digits; d += CS_THREADS) {       // the warps' counts become sums over the warps before
            uint32_t run = 0;
#pragma unroll
            for (int w = 0; w < CS_WARPS; ++w) { const uint32_t c = cnt[w * digits + d]; cnt[w * digits + d] = (uint16_t)run; run += c; }
            count[d] = run;
        }
        cs_sync();
        // first place of every digit's elements of this CTA: smaller digits of all CTAs, this digit in the CTAs before
        const int per = max(1, digits / CS_THREADS), d0 = tid * per;
        constexpr int PER = (1 << CS_MAX_BITS) / CS_THREADS;
        uint32_t sum = 0, tot[PER], mine[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) { tot[j] = 0; mine[j] = 0; }
        if (d0 < digits) {
            const uint32_t from = smem_u32(count + d0);
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                if (j >= per) break;
                uint32_t c[CTAS];                       // (all of them under way together)
#pragma unroll
                for (int r = 0; r < CTAS; ++r) c[r] = cs_load(cs_map(from + 4 * j, r));
#pragma unroll
                for (int r = 0; r < CTAS; ++r) asm volatile("" ::"r"(c[r]));
#pragma unroll
                for (int r = 0; r < CTAS; ++r) { tot[j] += c[r]; if (r < rank) mine[j] += c[r]; }
            }
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) sum += tot[j];
        uint32_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
        if (lane == 31) warp_tot[warp] = incl;
        __syncthreads();
        uint32_t run = incl - sum;
        for (int w = 0; w < warp; ++w) run += warp_tot[w];
        if (d0 < digits) {
#pragma unroll
            for (int j = 0; j < PER; ++j) if (j < per) { base[d0 + j] = run + mine[j]; run += tot[j]; }
        }
        __syncthreads();
        const bool last = pass + 1 == p.passes;
        const uint32_t out = smem_u32(pairs[(pass + 1) & 1]);
#pragma unroll
        for (int k = 0; k < CS_ITEMS; ++k) {
            if (k >= rounds || first + k * 32 + lane >= have) continue;
            const uint32_t digit = (key[k] >> shift) & (digits - 1);
            const uint32_t dst = base[digit] + cnt[warp * digits + digit] + at[k];
            if (last) p.pairs_out[dst] = make_uint2(key[k], pos[k]);
            else { const uint32_t r = dst / share; cs_store2(cs_map(out + (dst - r * share) * 8, r), key[k], pos[k]); }
        }
        cs_sync();         // the pairs are in place; nobody reads this pass's counts any more
    }
}

struct SumParams {
    const uint2* pairs;                    // (id, position) in order
    int n, chunks, dim, part_ld;
    uint32_t rows;
    const void* grads; int64_t ld_grads;
    void* out; int64_t ld_out;
    float scale;
    int accumulate;
    float* part;
    int2* list; int32_t* list_count;
    int group;                             // chunks of one id that a CTA of grad_sum_kernel joins
    int first_col;                         // of a launch of grad_join_kernel
    FastDiv vecs;
    const int32_t* ids; int32_t padding_id; int rows_per_cta, stripes; int32_t* status;     // grad_small_kernel
};

template <typename TO, int V>
__device__ __forceinline__ void finish_pack(const SumParams& p, uint32_t row, int64_t col, const float (&a)[V]) {
    TO* dst = static_cast<TO*>(p.out) + row * p.ld_out + col;
    Pack<TO, V> o;
    if (p.accumulate) o = *reinterpret_cast<const Pack<TO, V>*>(dst);
#pragma unroll
    for (int e = 0; e < V; ++e) o.v[e] = from_float<TO>(p.accumulate ? fmaf(a[e], p.scale, to_float(o.v[e])) : a[e] * p.scale);
    *reinterpret_cast<Pack<TO, V>*>(dst) = o;
}

// ---- short lists: one launch ----

// CTA c owns the table rows [c rows_per_cta, + rows_per_cta): it picks the ids that name them, sorts those as (row, position) words
// in shared memory, and adds up each row's gradients: runs of up to SHORT by one group of threads (a pack of columns each),
// longer ones in stripes, every stripes-th row to one, by all groups, and then the stripes in order.  Bound by latency: 256 ids of 1,000 x 32 fp32 in 7.9 us a call.
template <typename TG, typename TO, int V>
__global__ void __launch_bounds__(SMALL_THREADS) grad_small_kernel(SumParams p) {
    constexpr int SHORT = 32, U = 8;
    __shared__ uint32_t list[SMALL_MAX];       // local row << SMALL_BITS | position
    __shared__ uint16_t start[SMALL_MAX + 1];
    __shared__ uint32_t warp_cnt[SMALL_THREADS / 32];
    __shared__ float red[SMALL_THREADS * 8];      // stripes x columns at a time x V are at most as many
    grid_dependency_wait();
    allow_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t r0 = (int64_t)blockIdx.x * p.rows_per_cta;
    const int nr = (int)min((int64_t)p.rows_per_cta, (int64_t)p.rows - r0);
    // the ids of this CTA's rows, eight to a thread in the list's order
    int32_t id[SMALL_MAX / SMALL_THREADS];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < SMALL_MAX / SMALL_THREADS; ++k) {
        const int i = tid * (SMALL_MAX / SMALL_THREADS) + k;
        id[k] = -1;
        if (i < p.n) {
            const int32_t v = p.ids[i];
            if (v != p.padding_id) {
                if (v < 0 || (uint32_t)v >= p.rows) { if (blockIdx.x == 0) note_status(p.status, KGE_ERR_ID_RANGE); }
                else if (v >= r0 && v < r0 + nr) { id[k] = (int32_t)(v - r0); ++mine; }
            }
        }
    }
    if (!p.accumulate) {
        char* const base = static_cast<char*>(p.out) + r0 * p.ld_out * (int64_t)sizeof(TO);
        const int64_t row = (int64_t)p.dim * sizeof(TO);
        if (p.ld_out == p.dim) zero_bytes(base, nr * row, tid, SMALL_THREADS);
        else zero_strided(base, nr, row, p.ld_out * (int64_t)sizeof(TO), tid, SMALL_THREADS);
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
    if (lane == 31) warp_cnt[warp] = incl;
    __syncthreads();
    int at = incl - mine, m = 0;
#pragma unroll
    for (int w = 0; w < SMALL_THREADS / 32; ++w) { if (w < warp) at += warp_cnt[w]; m += warp_cnt[w]; }
    if (m == 0) return;
#pragma unroll
    for (int k = 0; k < SMALL_MAX / SMALL_THREADS; ++k)
        if (id[k] >= 0) list[at++] = (uint32_t)id[k] << SMALL_BITS | (uint32_t)(tid * (SMALL_MAX / SMALL_THREADS) + k);
    int m2 = 1;
    while (m2 < m) m2 <<= 1;
    for (int i = m + tid; i < m2; i += SMALL_THREADS) list[i] = ~0u;
    __syncthreads();
    for (int size = 2; size <= m2; size <<= 1)
        for (int stride = size >> 1; stride > 0; stride >>= 1) {
            for (int t = tid; t < m2 / 2; t += SMALL_THREADS) {
                const int lo = 2 * t - (t & (stride - 1)), hi = lo + stride;
                const uint32_t x = list[lo], y = list[hi];
                if ((x > y) == ((lo & size) == 0)) { list[lo] = y; list[hi] = x; }
            }
            __syncthreads();
        }
    // where each row's run begins
    int heads = 0;
#pragma unroll
    for (int k = 0; k < SMALL_MAX / SMALL_THREADS; ++k) {
        const int i = tid * (SMALL_MAX / SMALL_THREADS) + k;
        if (i < m && (i == 0 || list[i] >> SMALL_BITS != list[i - 1] >> SMALL_BITS)) heads |= 1 << k;
    }
    incl = __popc(heads);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
    if (lane == 31) warp_cnt[warp] = incl;
    __syncthreads();
    int u = incl - __popc(heads), runs = 0;
#pragma unroll
    for (int w = 0; w < SMALL_THREADS / 32; ++w) { if (w < warp) u += warp_cnt[w]; runs += warp_cnt[w]; }
#pragma unroll
    for (int k = 0; k < SMALL_MAX / SMALL_THREADS; ++k) if (heads >> k & 1) start[u++] = (uint16_t)(tid * (SMALL_MAX / SMALL_THREADS) + k);
    if (tid == 0) start[runs] = (uint16_t)m;
    __syncthreads();

    const int vecs = (int)p.vecs.d, wide = min(vecs, SMALL_THREADS), groups = SMALL_THREADS / wide;
    const int group = tid / wide, v0 = tid - group * wide;
    const TG* grads = static_cast<const TG*>(p.grads);
    auto add_rows = [&](int i, int end, int step, int64_t col, float (&a)[V]) {       // entries i, i + step, ... before `end`, in order
        for (; i < end; i += U * step) {
            Pack<TG, V> g[U];
#pragma unroll
            for (int q = 0; q < U; ++q)        // (beyond the end: the first again, for nothing -- a load under a condition waits for its use)
                g[q] = load_now<Pack<TG, V>>(grads + (int64_t)(list[i + q * step < end ? i + q * step : i] & (SMALL_MAX - 1)) * p.ld_grads + col);
#pragma unroll
            for (int q = 0; q < U; ++q)
#pragma unroll
                for (int e = 0; e < V; ++e) a[e] += i + q * step < end ? to_float(g[q].v[e]) : 0.f;
        }
    };
    if (group < groups)
        for (int r = group; r < runs; r += groups) {
            const int s = start[r], e = start[r + 1];
            if (e - s > SHORT) continue;
            for (int c = v0; c < vecs; c += wide) {
                float a[V];
#pragma unroll
                for (int q = 0; q < V; ++q) a[q] = 0.f;
                add_rows(s, e, 1, (int64_t)c * V, a);
                finish_pack<TO, V>(p, (uint32_t)(r0 + (list[s] >> SMALL_BITS)), (int64_t)c * V, a);
            }
        }
    for (int r = 0; r < runs; ++r) {
        const int s = start[r], e = start[r + 1];
        if (e - s <= SHORT) continue;
        const int parts = min(p.stripes, e - s);
        for (int c = v0; c - v0 < vecs; c += wide) {
            if (group < groups && c < vecs)
                for (int k = group; k < parts; k += groups) {
                    float a[V];
#pragma unroll
                    for (int q = 0; q < V; ++q) a[q] = 0.f;
                    add_rows(s + k, e, p.stripes, (int64_t)c * V, a);
#pragma unroll
                    for (int q = 0; q < V; ++q) red[(k * wide + v0) * V + q] = a[q];
                }
            __syncthreads();
            if (group == 0 && c < vecs) {
                float a[V];
#pragma unroll
                for (int q = 0; q < V; ++q) a[q] = red[v0 * V + q];
                for (int k = 1; k < parts; ++k) {
#pragma unroll
                    for (int q = 0; q < V; ++q) a[q] += red[(k * wide + v0) * V + q];
                }
                finish_pack<TO, V>(p, (uint32_t)(r0 + (list[s] >> SMALL_BITS)), (int64_t)c * V, a);
            }
            __syncthreads();
        }
    }
}

// Where a run's sum goes: a partial sum (slot 0: of the chunk's first run, 1: of its last) or the row itself.
template <typename TO, int V>
__device__ __forceinline__ void flush_run(const SumParams& p, int c, bool head, bool tail, uint32_t row, int64_t col, const float (&a)[V]) {
    if (head || tail) {
        float* dst = p.part + ((int64_t)c * 2 + (head ? 0 : 1)) * p.part_ld + col;
        if constexpr (V % 4 == 0) {
#pragma unroll
            for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(dst + e) = make_float4(a[e], a[e + 1], a[e + 2], a[e + 3]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) dst[e] = a[e];
        }
        if (!head && col == 0) p.list[atomicAdd(p.list_count, 1)] = make_int2(c, (int)row);
    } else finish_pack<TO, V>(p, row, col, a);
}

// One thread per (chunk of L sorted positions, pack of V columns).  An id whose rows lie within its first chunk and the next one
// is added up by the thread that meets its first row; one that reaches further leaves a partial sum per chunk.
// A thread's packs of the next DEPTH rows are on their way into its own places in shared memory, so the loop over the rows is one short
// body: unrolled by eight with the packs in registers it did not stay in the instruction cache (136 us against 84 at 500,000 x 256, 60 now
// that the rows are found by bisection: 4.9 TB/s).
// CTAs have 256 threads, or, where smaller packs take more for a group of chunks, 512 or 1,024.
constexpr int SUM_DEPTH = 8;
__host__ __device__ constexpr int sum_threads(int v) { return v >= 4 ? SUM_THREADS : 1024 / v; }       // at most
__host__ __device__ constexpr int sum_ring_bytes(int pack_bytes) { return pack_bytes >= 4 ? SUM_DEPTH * pack_bytes : 4; }       // per thread: rows on their way, then V sums
template <typename TG, typename TO, int V, int L>
__global__ void __launch_bounds__(sum_threads(V)) grad_sum_kernel(SumParams p) {
    constexpr int BYTES = V * (int)sizeof(TG);
    constexpr bool ASYNC = BYTES >= 4;                    // (asynchronous copies take 4, 8 or 16 bytes)
    static_assert(sum_ring_bytes(BYTES) >= 4 * V && sum_ring_bytes(BYTES) * sum_threads(V) <= 48 * 1024, "a thread's places in shared memory");
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_wait();
    allow_dependents();
    const int threads = V >= 4 ? SUM_THREADS : (int)blockDim.x;
    const int64_t item = (int64_t)blockIdx.x * threads + threadIdx.x;
    const int64_t vecs = p.vecs.d;
    const int c = item < (1ll << 31) ? (int)p.vecs.div((uint32_t)item) : (int)(item / vecs);
    if (c >= p.chunks) return;
    const int64_t col = (item - c * vecs) * V;
    const int64_t first = (int64_t)c * L, last = min((int64_t)p.n, first + L);        // [first, last): this chunk
    const TG* grads = static_cast<const TG*>(p.grads) + col;
    const uint2* const pairs = p.pairs + first;               // (indices below count from here)
    const int size = (int)(last - first), room = (int)min((int64_t)p.n - first, (int64_t)2 * L);
    const uint32_t none = p.rows, beyond = ~0u;
    const uint32_t lead = pairs[0].x, end_key = pairs[size - 1].x;
    const uint32_t before = c > 0 ? pairs[-1].x : beyond, early = c > 1 ? pairs[-L - 1].x : beyond;
    const uint32_t after = size < room ? pairs[size].x : beyond, far = first + 2 * L < p.n ? pairs[2 * L].x : beyond;
    if (lead == none) return;                                   // only ids of no row from here on
    // a first run that began in the chunk before is that chunk's, unless it reaches across a whole chunk: then a partial sum
    const bool head_part = before == lead && (early == lead || after == lead), skip = before == lead && !head_part;
    // a run that goes on beyond this chunk is taken along if it ends within the next one, else a partial sum
    const bool on = end_key != none && after == end_key && !(head_part && end_key == lead);
    const bool tail_part = on && far == end_key;
    // this thread's rows: [from, to), without a skipped run at the front and ids of no row at the end
    auto bound = [&](int lo, int hi, uint32_t key, bool above) {       // first index whose key is not below (above: greater than) `key`
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            const uint32_t k = pairs[mid].x;
            if (above ? k <= key : k < key) lo = mid + 1; else hi = mid;
        }
        return lo;
    };
    const int from = skip ? bound(0, size, lead, true) : 0;
    const int to = end_key == none ? bound(from, size, none, false) : (on && !tail_part ? bound(size, room, end_key, true) : size);
    if (from >= to) return;
    const uint32_t place = smem_u32(ring) + threadIdx.x * BYTES;
    auto issue = [&](int i) {
        if constexpr (ASYNC) {
            if (i < to) {
                const TG* src = grads + (int64_t)pairs[i].y * p.ld_grads;
                const uint32_t dst = place + (i % SUM_DEPTH) * (threads * BYTES);
                if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
#pragma unroll
    for (int u = 0; u < SUM_DEPTH - 1; ++u) issue(from + u);
    float a[V];
#pragma unroll
    for (int e = 0; e < V; ++e) a[e] = 0.f;
    uint32_t cur = pairs[from].x;
    bool is_head = head_part;
    auto add = [&](uint32_t k, const Pack<TG, V>& g) {
        if (k != cur) {
            flush_run<TO, V>(p, c, is_head, false, cur, col, a);
            is_head = false;
            cur = k;
#pragma unroll
            for (int e = 0; e < V; ++e) a[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) a[e] += to_float(g.v[e]);
    };
    if constexpr (ASYNC) {
#pragma unroll 1
        for (int i = from; i < to; ++i) {
            issue(i + SUM_DEPTH - 1);
            const uint32_t k = pairs[i].x;
            asm volatile("cp.async.wait_group %0;" ::"n"(SUM_DEPTH - 1) : "memory");
            add(k, *reinterpret_cast<const Pack<TG, V>*>(ring + (i % SUM_DEPTH) * (threads * BYTES) + threadIdx.x * BYTES));
        }
    } else {             // single 16-bit elements: eight rows' loads together
#pragma unroll 1
        for (int i0 = from; i0 < to; i0 += SUM_DEPTH) {
            Pack<TG, V> g[SUM_DEPTH];
            uint32_t k[SUM_DEPTH];
#pragma unroll
            for (int u = 0; u < SUM_DEPTH; ++u) {
                const uint2 at = pairs[min(i0 + u, to - 1)];
                k[u] = at.x;
                g[u] = load_now<Pack<TG, V>>(grads + (int64_t)at.y * p.ld_grads);
            }
#pragma unroll
            for (int u = 0; u < SUM_DEPTH; ++u) asm volatile("" ::"h"(*reinterpret_cast<const uint16_t*>(&g[u])));
#pragma unroll
            for (int u = 0; u < SUM_DEPTH; ++u) if (i0 + u < to) add(k[u], g[u]);
        }
    }
    // a group of chunks that lies inside one run leaves one partial sum, its first chunk's
    if (p.group > 1 && is_head) {
        const int64_t c0 = c & ~(p.group - 1), r1 = (c0 + p.group) * L;                   // (the same answer in all threads of the group)
        if (c0 > 0 && r1 < p.n && p.pairs[c0 * L - 1].x == cur && p.pairs[r1].x == cur) {
            const int vecs32 = (int)vecs, size = p.group * vecs32, at = (int)threadIdx.x / size;           // (128 threads or more)
            // a thread's sums lie in its own places of the ring, which it has read
            auto sum_of = [&](int thread, int e) -> float& {
                constexpr int PLACE = ASYNC ? BYTES : 4;
                return *reinterpret_cast<float*>(ring + (e * 4 / PLACE) * (threads * PLACE) + thread * PLACE + e * 4 % PLACE);
            };
#pragma unroll
            for (int e = 0; e < V; ++e) sum_of(threadIdx.x, e) = a[e];
            if (V == 8 && at) asm volatile("barrier.sync 2, %0;" ::"r"(size) : "memory");                  // (at most two groups, and those with packs of eight)
            else asm volatile("barrier.sync 1, %0;" ::"r"(size) : "memory");
            if (c != c0) return;
            for (int g = 1; g < p.group; ++g) {
#pragma unroll
                for (int e = 0; e < V; ++e) a[e] += sum_of(threadIdx.x + g * vecs32, e);
            }
        }
    }
    flush_run<TO, V>(p, c, is_head, tail_part && cur == end_key, cur, col, a);
}

// Ids that span more than two chunks: CTA (x, y) takes the x-th, (x + grid)-th, ... of the list and 64 columns from first_col on.  Sixteen
// stripes of sixteen threads add every 16th chunk's partial sum, then the stripes are added in order.
constexpr int JOIN_COLS = 64;
__device__ __forceinline__ int64_t ceil_div_dev(int64_t a, int64_t b) { return (a + b - 1) / b; }
template <typename TO, int L>
__global__ void __launch_bounds__(JOIN_THREADS) grad_join_kernel(SumParams p) {
    constexpr int LANES = JOIN_COLS / 4, STRIPES = JOIN_THREADS / LANES, U = 8;
    __shared__ float4 red[STRIPES][LANES];
    __shared__ float4 ring[U][JOIN_THREADS];
    grid_dependency_wait();
    const int lane = threadIdx.x % LANES, stripe = threadIdx.x / LANES;
    const int col0 = p.first_col + blockIdx.y * JOIN_COLS, col = col0 + lane * 4;
    const int count = *p.list_count;
    for (int x = blockIdx.x; x < count; x += gridDim.x) {
        const int2 run = p.list[x];
        const int c0 = run.x;
        const uint32_t key = (uint32_t)run.y;
        // the last chunk that begins with this id: 256 chunks looked at per round
        int64_t end = (int64_t)c0 + 1;
        for (;;) {
            const int64_t at = end + 1 + threadIdx.x;
            const int got = __syncthreads_count(at < p.chunks && p.pairs[at * L].x == key);
            end += got;
            if (got < JOIN_THREADS) break;
        }
        // partial sum j of the id: slot 1 of chunk c0, then slot 0 of the following ones, where a group of chunks that lies inside the
        // run counts as one; eight of a thread's on their way into shared memory at a time (with registers as their target they came
        // one by one, 4.5 us a round of eight)
        const int64_t g0 = ceil_div_dev(c0 + 1, p.group), g1 = max(g0, end / p.group);    // those groups: [g0, g1)
        const int64_t lead = g1 > g0 ? g0 * p.group - c0 : end - c0 + 1;                  // parts before the first of them
        const int64_t parts = g1 > g0 ? lead + (g1 - g0) + (end - g1 * p.group + 1) : lead;
        auto chunk_of = [&](int64_t j) { return j < lead ? c0 + j : (j < lead + g1 - g0 ? (g0 + j - lead) * p.group : g1 * p.group + j - lead - (g1 - g0)); };
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int64_t j0 = stripe; j0 < parts && col < p.part_ld; j0 += U * STRIPES) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t j = j0 + u * STRIPES;
                if (j < parts)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(&ring[u][threadIdx.x])),
                                 "l"(p.part + (chunk_of(j) * 2 + (j == 0)) * p.part_ld + col) : "memory");
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j0 + u * STRIPES < parts) { const float4 v = ring[u][threadIdx.x]; a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w; }
        }
        red[stripe][lane] = a;
        __syncthreads();
        if (threadIdx.x < JOIN_COLS) {
            const int cc = col0 + threadIdx.x;
            if (cc < p.dim) {
                float sum = 0.f;
#pragma unroll
                for (int s = 0; s < STRIPES; ++s) sum += reinterpret_cast<const float*>(&red[s][0])[threadIdx.x];
                const float one[1] = {sum};
                finish_pack<TO, 1>(p, key, cc, one);
            }
        }
        __syncthreads();
    }
}

// Calls f with the pack length as a constant.
template <bool EIGHT, class F> int with_vector(int vec, F&& f) {
    if constexpr (EIGHT) { if (vec == 8) return f(std::integral_constant<int, 8>()); }
    if (vec == 4) return f(std::integral_constant<int, 4>());
    if (vec == 2) return f(std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 1>());
}

int launch_lookup(LookupParams& p, int tt, int to, int vec, int dim, cudaStream_t s) {
    p.dim = dim;
    p.vecs = FastDiv((uint32_t)(vec == 1 ? ceil_div(dim, 4) : dim / vec));
    p.rows_per_cta = (int)std::max<int64_t>(1, LOOKUP_THREADS * LOOKUP_UNROLL / p.vecs.d);
    const dim3 grid((unsigned)ceil_div(p.n, p.rows_per_cta));
    return with_type(tt, [&](auto a) {
        return with_type(to, [&](auto b) {
            using TT = decltype(a); using TO = decltype(b);
            if (vec == 1) return launch_status(launch_dependent(lookup_single_kernel<TT, TO>, grid, dim3(LOOKUP_THREADS), 0, s, p));
            return with_vector<sizeof(TT) == 2 && sizeof(TO) == 2>(vec, [&](auto v) {
                return launch_status(launch_dependent(lookup_kernel<TT, TO, decltype(v)::value>, grid, dim3(LOOKUP_THREADS), 0, s, p));
            });
        });
    });
}

template <typename TG, typename TO>
int launch_small(SumParams& p, int vec, cudaStream_t s) {
    p.vecs = FastDiv((uint32_t)(p.dim / vec));
    // four CTAs an SM, more where a CTA's rows would not fit the words it sorts
    int64_t per = ceil_div(p.rows, 148 * 4);
    per = std::max<int64_t>(1, std::min<int64_t>(per, (1ll << (32 - SMALL_BITS)) - 1));
    p.rows_per_cta = (int)per;
    p.stripes = run_stripes(p.dim);
    return with_vector<sizeof(TG) == 2>(vec, [&](auto v) {
        return launch_status(launch_dependent(grad_small_kernel<TG, TO, decltype(v)::value>, dim3((unsigned)ceil_div(p.rows, per)), dim3(SMALL_THREADS), 0, s, p));
    });
}

template <typename TG, typename TO, int L>
int launch_sum(SumParams& p, int vec, cudaStream_t s) {
    p.vecs = FastDiv((uint32_t)(p.dim / vec));
    p.group = group_chunks(p.dim);
    const int threads = p.group > 1 ? std::max(SUM_THREADS, p.group * (int)p.vecs.d) : SUM_THREADS;
    const dim3 grid((unsigned)ceil_div((int64_t)p.chunks * p.vecs.d, threads));
    const int rc = with_vector<sizeof(TG) == 2>(vec, [&](auto v) {
        constexpr int V = decltype(v)::value;
        return launch_status(launch_dependent(grad_sum_kernel<TG, TO, V, L>, grid, dim3((unsigned)threads), (size_t)threads * sum_ring_bytes(V * (int)sizeof(TG)), s, p));
    });
    if (rc != KGE_OK || p.chunks < 3) return rc;
    constexpr int64_t COLS = 65535ll * JOIN_COLS;           // a grid is no higher
    for (int64_t first = 0; first < p.dim; first += COLS) {
        p.first_col = (int)first;
        const dim3 joins((unsigned)std::min<int64_t>(p.chunks / 2, 592), (unsigned)ceil_div(std::min(p.dim - first, COLS), JOIN_COLS));
        const int rj = launch_status(launch_dependent(grad_join_kernel<TO, L>, joins, dim3(JOIN_THREADS), 0, s, p));
        if (rj != KGE_OK) return rj;
    }
    return KGE_OK;
}

// Clusters of sixteen CTAs are no promise of the architecture: how many of them the device runs at a time is asked once.
int wide_clusters(int* clusters) {
    static std::atomic<int> known[kMaxDevices];        // one more than their number
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return KGE_ERR_CUDA;
    const bool tracked = dev >= 0 && dev < kMaxDevices;
    int state = tracked ? known[dev].load(std::memory_order_acquire) : 0;
    if (state == 0) {
        const int most = (int)cluster_sort_smem(CS_MAX, CS_MAX_BITS, CS_CTAS), most8 = (int)cluster_sort_smem(CS_MAX, CS_MAX_BITS, CS_CTAS_PORTABLE);
        if (cudaFuncSetAttribute(grad_cluster_sort_kernel<CS_CTAS_PORTABLE>, cudaFuncAttributeMaxDynamicSharedMemorySize, most8) != cudaSuccess ||
            cudaFuncSetAttribute(grad_cluster_sort_kernel<CS_CTAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess ||
            cudaFuncSetAttribute(grad_cluster_sort_kernel<CS_CTAS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return KGE_ERR_CUDA;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(CS_CTAS); cfg.blockDim = dim3(CS_THREADS); cfg.dynamicSmemBytes = (size_t)most;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = CS_CTAS; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 1;
        int fit = 0;
        if (cudaOccupancyMaxActiveClusters(&fit, grad_cluster_sort_kernel<CS_CTAS>, &cfg) != cudaSuccess) { (void)cudaGetLastError(); fit = 0; }
        state = 1 + std::max(fit, 0);
        if (tracked) known[dev].store(state, std::memory_order_release);
    }
    *clusters = state - 1;
    return KGE_OK;
}

// `beside`: clusters that set rows to zero while the first one sorts, no more than run at the same time (55,864 x 496 fp32 and 3,010
// ids: 30 us a call with six, 38 with a seventh, which waits until one ends).
template <int CTAS>
int launch_cluster_sort(SortParams& q, const SortPlan& plan, bool zero, int64_t rows, int beside, cudaStream_t s) {
    const int zero_clusters = zero ? (int)std::min<int64_t>(std::max(1, beside), ceil_div(rows * q.zero_row_bytes, 8192 * CTAS)) : 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(CTAS * (1 + zero_clusters))); cfg.blockDim = dim3(CS_THREADS); cfg.stream = s;
    cfg.dynamicSmemBytes = cluster_sort_smem(q.n, plan.bits, CTAS);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CTAS; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return launch_status(cudaLaunchKernelEx(&cfg, grad_cluster_sort_kernel<CTAS>, q));
}

// The (id, position) pairs in order, in g.pairs[*where]; the rows of a dense gradient set to zero.
int sort_ids(const GradScratch& g, const SortPlan& plan, SortParams& q, bool zero, int64_t rows, int* where, cudaStream_t s) {
    const int digits = 1 << plan.bits;
    if (q.n <= CS_MAX) {
        q.pairs_out = g.pairs[0];
        q.zero_first = 0; q.zero_last = rows;
        *where = 0;
        int wide = 0;
        const int rc = wide_clusters(&wide);
        if (rc != KGE_OK) return rc;
        return wide > 0 ? launch_cluster_sort<CS_CTAS>(q, plan, zero, rows, wide - 1, s)
                        : launch_cluster_sort<CS_CTAS_PORTABLE>(q, plan, zero, rows, 128 / CS_CTAS_PORTABLE, s);
    }
    // the zeroing is shared out over the launches: the sort leaves most of the memory's bandwidth unused
    const int launches = 2 * plan.passes;
    int nth = 0, rc = KGE_OK;
    auto zero_ctas = [&] {
        q.zero_first = rows * nth / launches; q.zero_last = rows * (nth + 1) / launches;
        ++nth;
        return zero ? (int)std::min<int64_t>(148 * 6, ceil_div((q.zero_last - q.zero_first) * q.zero_row_bytes, 16 * GS_THREADS)) : 0;
    };
    for (int pass = 0; pass < plan.passes && rc == KGE_OK; ++pass) {
        q.pass = pass; q.shift = pass * plan.bits;
        q.pairs_in = g.pairs[(pass + 1) & 1];
        q.pairs_out = g.pairs[pass & 1];
        int ctas = plan.tiles + zero_ctas();
        rc = launch_status(launch_dependent(grad_hist_kernel, dim3((unsigned)ctas), dim3(GS_THREADS), 0, s, q));
        if (rc == KGE_OK) rc = launch_status(launch_dependent(grad_scan_kernel, dim3((unsigned)((digits * 32 + 255) / 256)), dim3(256), 0, s, q));
        ctas = plan.tiles + zero_ctas();
        if (rc == KGE_OK) rc = launch_status(launch_dependent(grad_scatter_kernel, dim3((unsigned)ctas), dim3(GS_THREADS), 0, s, q));
    }
    *where = (plan.passes - 1) & 1;
    return rc;
}

}  // namespace
}  // namespace kge

using namespace kge;

extern "C" {

int kge_embedding_lookup(const void* table, int32_t table_type, int64_t rows, int32_t dim, int64_t ld_table, const int32_t* ids, int32_t n,
                         float scale, int32_t padding_id, void* out, int32_t out_type, int64_t ld_out, int32_t* status, void* stream) {
    if (!is_float_type(table_type) || !is_float_type(out_type) || rows < 1 || rows > INT32_MAX || dim < 1 || ld_table < dim || ld_out < dim || n < 0)
        return KGE_ERR_BAD_ARG;
    if (n == 0) return KGE_OK;
    if (!table || !ids || !out || !aligned_to(table, type_bytes(table_type)) || !aligned_to(out, type_bytes(out_type)) || !aligned_to(ids, 4) ||
        !aligned_to(status, 4)) return KGE_ERR_BAD_ARG;
    LookupParams p{};
    p.table = table; p.out = out; p.ids = ids; p.rows = rows; p.ld_table = ld_table; p.ld_out = ld_out; p.n = n;
    p.padding_id = padding_id; p.scale = scale; p.status = status;
    const int tb = type_bytes(table_type), ob = type_bytes(out_type);
    const int vec = vector_length(tb == 2 && ob == 2 ? 8 : 4, dim, ld_table, tb, table, ld_out, ob, out);
    return launch_lookup(p, table_type, out_type, vec, dim, static_cast<cudaStream_t>(stream));
}

size_t kge_embedding_grad_scratch_bytes(int64_t rows, int32_t dim, int32_t n) {
    if (rows < 1 || rows > INT32_MAX || dim < 1 || dim > GRAD_MAX_DIM || n < 1) return 0;
    return carve_grad(nullptr, rows, dim, n).bytes;
}

int kge_embedding_grad(const int32_t* ids, int32_t n, const void* grads, int32_t grads_type, int64_t ld_grads, float scale, int32_t padding_id,
                       int32_t accumulate, void* table_grad, int32_t table_type, int64_t rows, int32_t dim, int64_t ld_table, void* scratch,
                       size_t scratch_bytes, int32_t* status, void* stream) {
    if (!is_float_type(grads_type) || !is_float_type(table_type) || rows < 1 || rows > INT32_MAX || dim < 1 || ld_grads < dim || ld_table < dim ||
        n < 0 || (accumulate != 0 && accumulate != 1)) return KGE_ERR_BAD_ARG;
    if (dim > GRAD_MAX_DIM) return KGE_ERR_UNSUPPORTED;
    if (!table_grad || !aligned_to(table_grad, type_bytes(table_type)) || !aligned_to(status, 4)) return KGE_ERR_BAD_ARG;
    if (n > 0 && (!ids || !grads || !aligned_to(ids, 4) || !aligned_to(grads, type_bytes(grads_type)))) return KGE_ERR_BAD_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int gb = type_bytes(grads_type), tb = type_bytes(table_type);
    if (n == 0) {
        if (accumulate) return KGE_OK;
        return launch_status(cudaMemset2DAsync(table_grad, (size_t)ld_table * tb, 0, (size_t)dim * tb, (size_t)rows, s));
    }
    const size_t need = kge_embedding_grad_scratch_bytes(rows, dim, n);
    if (need > 0 && (!scratch || !aligned_to(scratch, 256) || scratch_bytes < need)) return KGE_ERR_WORKSPACE;
    const int vec = vector_length(gb == 2 ? 8 : 4, dim, ld_grads, gb, grads, ld_table, tb, table_grad);
    SumParams p{};
    p.n = n; p.dim = dim; p.part_ld = (dim + 3) / 4 * 4; p.rows = (uint32_t)rows;
    p.grads = grads; p.ld_grads = ld_grads; p.out = table_grad; p.ld_out = ld_table; p.scale = scale; p.accumulate = accumulate;
    p.ids = ids; p.padding_id = padding_id; p.status = status;
    if (short_list(rows, n))
        return with_type(grads_type, [&](auto a) { return with_type(table_type, [&](auto b) { return launch_small<decltype(a), decltype(b)>(p, vec, s); }); });
    const GradScratch g = carve_grad(static_cast<char*>(scratch), rows, dim, n);
    const SortPlan plan = sort_plan(rows, n);
    SortParams q{};
    q.ids = ids; q.n = n; q.tiles = plan.tiles; q.bits = plan.bits; q.passes = plan.passes; q.rows = (uint32_t)rows; q.padding_id = padding_id;
    q.hist = g.hist; q.total = g.total; q.list_count = g.list_count; q.status = status;
    q.zero = static_cast<char*>(table_grad); q.zero_row_bytes = (int64_t)dim * tb; q.zero_ld_bytes = ld_table * tb;
    q.zero_flat = ld_table == dim;
    int where = 0;
    const int rc = sort_ids(g, plan, q, !accumulate, rows, &where, s);
    if (rc != KGE_OK) return rc;
    p.pairs = g.pairs[where];
    p.chunks = (int)ceil_div(n, chunk_rows(n));
    p.part = g.part; p.list = g.list; p.list_count = g.list_count;
    return with_type(grads_type, [&](auto a) {
        return with_type(table_type, [&](auto b) {
            using TG = decltype(a); using TO = decltype(b);
            return chunk_rows(n) == 8 ? launch_sum<TG, TO, 8>(p, vec, s) : launch_sum<TG, TO, 32>(p, vec, s);
        });
    });
}

}  // extern "C"
