// Rows of a table for a list of ids, times a scale, and the gradient of that.
//   lookup    out[i] = scale T[ids[i]]
//   gradient  dT[e] = scale sum_{i : ids[i] = e} g[i]      (+ the old dT[e])
// The gradient sorts the ids (stable radix sort of (id, position) pairs), walks the sorted list in chunks of rows, adds a chunk's
// rows of one id in fp32 in ascending position, and joins the ids that span chunks in a second, fixed order: the result is a
// function of the inputs alone.
//   hist      digit counts of every tile; clears the later passes' counts and, side by side with that, the dense gradient
//   scatter   one stable split by a digit of up to eleven bits; counts the next digit on the way
//   sum       chunks of sorted rows; what ends inside its chunk or the next one is final, the rest leaves partial sums
//   join      one CTA per (id that spans more, 32 columns): partial sums in a fixed order
#include <algorithm>

#include "kge_ops.cuh"

namespace kge {

namespace {

// ---- lookup ----------------------------------------------------------------------------------------------------------

struct LookupParams {
    const void* table; void* out;
    const int32_t* ids;
    int64_t rows, ld_table, ld_out;
    int n, rows_per_cta;
    int32_t padding_id;
    float scale;
    FastDiv vecs;                 // packs per row
    int32_t* status;
};

constexpr int LOOKUP_THREADS = 256, LOOKUP_UNROLL = 4;

template <typename TT, typename TO, int V>
__global__ void __launch_bounds__(LOOKUP_THREADS) lookup_kernel(LookupParams p) {
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

// ---- gradient --------------------------------------------------------------------------------------------------------

constexpr int GS_THREADS = 256, GS_WARPS = GS_THREADS / 32, GS_ITEMS = 8;
constexpr int GS_TILE = GS_THREADS * GS_ITEMS;     // ids per CTA of the sort
constexpr int GS_MAX_BITS = 11, GS_MAX_PASSES = 4;
constexpr int GS_DIRECT_TILES = 256;               // up to here every scatter CTA adds up the tiles' counts itself
constexpr int SUM_THREADS = 256;
constexpr int JOIN_THREADS = 256;

struct SortPlan { int tiles, key_bits, passes, bits; };

SortPlan sort_plan(int64_t rows, int n) {
    SortPlan s;
    s.tiles = (int)ceil_div(n, GS_TILE);
    s.key_bits = 1;
    while (s.key_bits < 31 && (1ll << s.key_bits) <= rows) ++s.key_bits;      // keys 0 .. rows (rows: no row of the table)
    // few tiles: wide digits, two passes up to four million rows; many: the counts of 2,048 digits a tile cost more than a pass
    const int most = s.tiles <= 64 ? GS_MAX_BITS : 9;
    s.passes = (s.key_bits + most - 1) / most;
    s.bits = (s.key_bits + s.passes - 1) / s.passes;
    return s;
}
int chunk_rows(int n) { return n < (1 << 17) ? 8 : 32; }

struct GradScratch {
    uint32_t *keys[2], *pos[2];      // [n] sorted ids and positions, in turn
    uint32_t* hist;                  // [passes][tiles][1 << bits]
    uint32_t* total;                 // [1 << bits] (many tiles only)
    float* part;                     // [chunks][2][dim rounded up to 4]
    int32_t *list, *list_count;      // chunks in which an id begins that spans more
    size_t bytes;
};

GradScratch carve_grad(char* base, int64_t rows, int dim, int n) {
    size_t used = 0;
    auto take = [&](size_t bytes) { char* q = base ? base + used : nullptr; used += (bytes + 255) / 256 * 256; return q; };
    const SortPlan s = sort_plan(rows, n);
    const int64_t chunks = ceil_div(n, chunk_rows(n));
    GradScratch g{};
    for (int i = 0; i < 2; ++i) { g.keys[i] = reinterpret_cast<uint32_t*>(take((size_t)n * 4 + 128)); g.pos[i] = reinterpret_cast<uint32_t*>(take((size_t)n * 4 + 128)); }
    g.hist = reinterpret_cast<uint32_t*>(take((size_t)s.passes * s.tiles * (4u << s.bits)));
    g.total = reinterpret_cast<uint32_t*>(take((size_t)4 << s.bits));
    g.part = reinterpret_cast<float*>(take((size_t)chunks * 2 * ((dim + 3) / 4 * 4) * 4));
    g.list = reinterpret_cast<int32_t*>(take((size_t)chunks * 4));
    g.list_count = reinterpret_cast<int32_t*>(take(256));
    g.bytes = used;
    return g;
}

struct SortParams {
    const int32_t* ids;
    int n, tiles, bits, shift, pass, passes;
    uint32_t rows;
    int32_t padding_id;
    const uint32_t *keys_in, *pos_in;
    uint32_t *keys_out, *pos_out;
    uint32_t *hist, *hist_next, *total;   // this pass's and the next one's [tiles][1 << bits]
    int scanned;                          // hist holds sums over the tiles before, total the digits' counts
    int32_t *list_count, *status;
    // dense gradient rows set to zero side by side with the first counts
    void* zero; int64_t zero_rows, zero_row_bytes, zero_ld_bytes;
    int zero_vec;                         // rows are whole 16-byte words and lie back to back
};

__device__ __forceinline__ uint32_t grad_key(const SortParams& p, int i) {
    const int32_t id = p.ids[i];
    if (id == p.padding_id) return p.rows;
    if (id < 0 || (uint32_t)id >= p.rows) { note_status(p.status, KGE_ERR_ID_RANGE); return p.rows; }
    return (uint32_t)id;
}

__global__ void __launch_bounds__(GS_THREADS) grad_hist_kernel(SortParams p) {
    __shared__ uint32_t count[1 << GS_MAX_BITS];
    const int digits = 1 << p.bits, tid = threadIdx.x;
    if ((int)blockIdx.x >= p.tiles) {
        const int64_t first = (int64_t)(blockIdx.x - p.tiles) * GS_THREADS + tid, step = (int64_t)(gridDim.x - p.tiles) * GS_THREADS;
        if (p.zero_vec) {
            uint4* z = static_cast<uint4*>(p.zero);
            const int64_t words = p.zero_rows * (p.zero_row_bytes / 16);
            for (int64_t i = first; i < words; i += step) z[i] = make_uint4(0u, 0u, 0u, 0u);
        } else {
            const int64_t halves = p.zero_row_bytes / 2, all = p.zero_rows * halves;
            for (int64_t i = first; i < all; i += step) {
                const int64_t r = i / halves;
                *reinterpret_cast<uint16_t*>(static_cast<char*>(p.zero) + r * p.zero_ld_bytes + (i - r * halves) * 2) = 0;
            }
        }
        return;
    }
    for (int d = tid; d < digits; d += GS_THREADS) {
        count[d] = 0;
        for (int q = 1; q < p.passes; ++q) p.hist[((int64_t)q * p.tiles + blockIdx.x) * digits + d] = 0;
    }
    if (blockIdx.x == 0 && tid == 0) *p.list_count = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        const int i = blockIdx.x * GS_TILE + k * GS_THREADS + tid;
        if (i < p.n) atomicAdd(&count[grad_key(p, i) & (digits - 1)], 1u);
    }
    __syncthreads();
    for (int d = tid; d < digits; d += GS_THREADS) p.hist[(int64_t)blockIdx.x * digits + d] = count[d];
}

// Many tiles: one thread per digit turns the tiles' counts into sums over the tiles before.
__global__ void __launch_bounds__(32) grad_scan_kernel(SortParams p) {
    const int digits = 1 << p.bits, d = blockIdx.x * 32 + threadIdx.x;
    if (d >= digits) return;
    uint32_t run = 0;
    for (int t0 = 0; t0 < p.tiles; t0 += 16) {
        uint32_t c[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) c[u] = t0 + u < p.tiles ? p.hist[(int64_t)(t0 + u) * digits + d] : 0u;
#pragma unroll
        for (int u = 0; u < 16; ++u) if (t0 + u < p.tiles) { p.hist[(int64_t)(t0 + u) * digits + d] = run; run += c[u]; }
    }
    p.total[d] = run;
}

// Stable split of one tile by a digit: a warp takes its 256 elements 32 at a time in order, lanes of one digit find each other
// by a vote and a running count per (warp, digit) carries over; the warps' counts and the tiles' give every element its place.
__global__ void __launch_bounds__(GS_THREADS) grad_scatter_kernel(SortParams p) {
    __shared__ uint16_t cnt[GS_WARPS][1 << GS_MAX_BITS];
    __shared__ uint32_t base[1 << GS_MAX_BITS];
    __shared__ uint32_t warp_tot[GS_WARPS];
    const int digits = 1 << p.bits, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, tile = blockIdx.x;
    for (int d = lane; d < digits; d += 32) cnt[warp][d] = 0;
    __syncwarp();
    uint32_t key[GS_ITEMS], pos[GS_ITEMS], at[GS_ITEMS];
    const int i0 = tile * GS_TILE + warp * 32 * GS_ITEMS;
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        const int i = i0 + k * 32 + lane;
        if (i < p.n) {
            key[k] = p.pass == 0 ? grad_key(p, i) : p.keys_in[i];
            pos[k] = p.pass == 0 ? (uint32_t)i : p.pos_in[i];
        }
    }
#pragma unroll
    for (int k = 0; k < GS_ITEMS; ++k) {
        const bool in = i0 + k * 32 + lane < p.n;
        const uint32_t digit = in ? (key[k] >> p.shift) & (digits - 1) : 1u << GS_MAX_BITS;     // (lanes beyond the list: a digit of their own)
        const unsigned same = __match_any_sync(0xffffffffu, digit), before = same & ((1u << lane) - 1u);
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
    uint32_t sum = 0, tot[8], mine[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { tot[j] = 0; mine[j] = 0; }
    if (d0 < digits) {
        if (p.scanned) {
#pragma unroll
            for (int j = 0; j < 8; ++j) if (j < per) { tot[j] = p.total[d0 + j]; mine[j] = p.hist[(int64_t)tile * digits + d0 + j]; }
        } else {
#pragma unroll 4
            for (int t = 0; t < p.tiles; ++t) {
                const uint32_t* h = p.hist + (int64_t)t * digits + d0;
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j < per) { const uint32_t c = h[j]; tot[j] += c; if (t < tile) mine[j] += c; }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += tot[j];
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
        for (int j = 0; j < 8; ++j) if (j < per) {
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
        p.keys_out[dst] = key[k];
        p.pos_out[dst] = pos[k];
        if (p.hist_next) atomicAdd(&p.hist_next[(int64_t)(dst / GS_TILE) * digits + ((key[k] >> (p.shift + p.bits)) & (digits - 1))], 1u);
    }
}

struct SumParams {
    const uint32_t *keys, *pos;
    int n, chunks, dim, part_ld;
    uint32_t rows;
    const void* grads; int64_t ld_grads;
    void* out; int64_t ld_out;
    float scale;
    int accumulate;
    float* part;
    int32_t *list, *list_count;
    FastDiv vecs;
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

// One thread per (chunk of L sorted positions, pack of V columns).  An id whose rows lie within its first chunk and the next one
// is added up by the thread that meets its first row; one that reaches further leaves a partial sum per chunk.
template <typename TG, typename TO, int V, int L>
__global__ void __launch_bounds__(SUM_THREADS) grad_sum_kernel(SumParams p) {
    const int64_t item = (int64_t)blockIdx.x * SUM_THREADS + threadIdx.x;
    const int64_t vecs = p.vecs.d;
    const int c = item < (1ll << 31) ? (int)p.vecs.div((uint32_t)item) : (int)(item / vecs);
    if (c >= p.chunks) return;
    const int64_t col = (item - c * vecs) * V;
    const int first = c * L, last = min(p.n, first + L);        // [first, last): this chunk
    const TG* grads = static_cast<const TG*>(p.grads) + col;
    const uint32_t none = p.rows;
    const uint32_t lead = p.keys[first];
    if (lead == none) return;                                   // only ids of no row from here on
    // the first run: does it begin here, in the chunk before, or earlier?
    int r = first;
    bool head_part = false;
    if (c > 0 && p.keys[first - 1] == lead) {
        const bool early = first - L - 1 >= 0 && p.keys[first - L - 1] == lead;      // it has rows before the chunk before
        const bool through = last < p.n && p.keys[last] == lead;                     // and beyond this one
        if (early || through) head_part = true;
        else { while (r < last && p.keys[r] == lead) ++r; }                          // the chunk before adds these rows
    }
    float a[V];
#pragma unroll
    for (int e = 0; e < V; ++e) a[e] = 0.f;
    int stop = last;                  // one past the last row this thread adds
    bool tail_part = false;
    if (r < last) {
        const uint32_t end_key = p.keys[last - 1];
        // a run that goes on beyond the chunk: taken along if it ends within the next one, else a partial sum
        if (end_key != none && last < p.n && p.keys[last] == end_key && !(head_part && end_key == lead)) {
            const int far = first + 2 * L;
            if (far < p.n && p.keys[far] == end_key) tail_part = true;
            else { const int most = min(p.n, far); while (stop < most && p.keys[stop] == end_key) ++stop; }
        }
    }
    if (r >= stop) return;
    uint32_t cur = p.keys[r];
    bool is_head = head_part;
    constexpr int U = 8;
    for (int r0 = r; r0 < stop; r0 += U) {
        uint32_t k[U];
        Pack<TG, V> g[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u] = r0 + u < stop ? p.keys[r0 + u] : none;
            if (k[u] != none) g[u] = *reinterpret_cast<const Pack<TG, V>*>(grads + (int64_t)p.pos[r0 + u] * p.ld_grads);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r0 + u >= stop) break;
            if (k[u] != cur) {
                if (is_head) {
#pragma unroll
                    for (int e = 0; e < V; ++e) p.part[(int64_t)c * 2 * p.part_ld + col + e] = a[e];
                    is_head = false;
                } else if (cur != none) finish_pack<TO, V>(p, cur, col, a);
                cur = k[u];
#pragma unroll
                for (int e = 0; e < V; ++e) a[e] = 0.f;
            }
            if (k[u] != none) {
#pragma unroll
                for (int e = 0; e < V; ++e) a[e] += to_float(g[u].v[e]);
            }
        }
    }
    if (cur == none) return;
    if (is_head || tail_part) {
        float* dst = p.part + ((int64_t)c * 2 + (is_head ? 0 : 1)) * p.part_ld + col;
#pragma unroll
        for (int e = 0; e < V; ++e) dst[e] = a[e];
        if (!is_head && col == 0) p.list[atomicAdd(p.list_count, 1)] = c;
    } else finish_pack<TO, V>(p, cur, col, a);
}

// Ids that span more than two chunks: CTA (x, y) takes the x-th, (x + grid)-th, ... of the list and 32 columns.  Thirty-two stripes
// of eight threads add every 32nd chunk's partial sum, then the stripes are added in order.
template <typename TO, int L>
__global__ void __launch_bounds__(JOIN_THREADS) grad_join_kernel(SumParams p) {
    constexpr int STRIPES = JOIN_THREADS / 8;
    __shared__ float4 red[STRIPES][8];
    const int lane8 = threadIdx.x & 7, stripe = threadIdx.x >> 3;
    const int col = blockIdx.y * 32 + lane8 * 4;
    const int count = *p.list_count;
    for (int x = blockIdx.x; x < count; x += gridDim.x) {
        const int c0 = p.list[x];
        const uint32_t key = p.keys[(c0 + 1) * L];
        // the last chunk that begins with this id: 256 chunks looked at per round
        int end = c0 + 1;
        for (;;) {
            const int64_t at = (int64_t)end + 1 + threadIdx.x;
            const bool more = at * L < p.n && p.keys[at * L] == key;
            const int got = __syncthreads_count(more);
            end += got;
            if (got < JOIN_THREADS) break;
        }
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        if (col < p.part_ld) {
            // partial sum j of the id: slot 1 of chunk c0, then slot 0 of the following ones
            for (int j0 = stripe; j0 <= end - c0; j0 += 4 * STRIPES) {
                float4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int j = j0 + u * STRIPES;
                    v[u] = j <= end - c0 ? *reinterpret_cast<const float4*>(p.part + ((int64_t)(c0 + j) * 2 + (j == 0)) * p.part_ld + col) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) { a.x += v[u].x; a.y += v[u].y; a.z += v[u].z; a.w += v[u].w; }
            }
        }
        __syncthreads();
        red[stripe][lane8] = a;
        __syncthreads();
        if (threadIdx.x < 32) {
            const int cc = blockIdx.y * 32 + threadIdx.x;
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

int launch_lookup(LookupParams& p, int tt, int to, int vec, int dim, cudaStream_t s) {
    p.vecs = FastDiv((uint32_t)(dim / vec));
    p.rows_per_cta = (int)std::max<int64_t>(1, LOOKUP_THREADS * LOOKUP_UNROLL / p.vecs.d);
    const dim3 grid((unsigned)ceil_div(p.n, p.rows_per_cta));
    return with_type(tt, [&](auto a) {
        return with_type(to, [&](auto b) {
            using TT = decltype(a); using TO = decltype(b);
            constexpr bool wide = sizeof(TT) == 2 && sizeof(TO) == 2;
            if (wide && vec == 8) lookup_kernel<TT, TO, wide ? 8 : 4><<<grid, LOOKUP_THREADS, 0, s>>>(p);
            else if (vec == 4) lookup_kernel<TT, TO, 4><<<grid, LOOKUP_THREADS, 0, s>>>(p);
            else if (vec == 2) lookup_kernel<TT, TO, 2><<<grid, LOOKUP_THREADS, 0, s>>>(p);
            else lookup_kernel<TT, TO, 1><<<grid, LOOKUP_THREADS, 0, s>>>(p);
            return launch_status(cudaGetLastError());
        });
    });
}

template <typename TG, typename TO, int L>
int launch_sum(SumParams& p, int vec, cudaStream_t s) {
    p.vecs = FastDiv((uint32_t)(p.dim / vec));
    const dim3 grid((unsigned)ceil_div((int64_t)p.chunks * p.vecs.d, SUM_THREADS));
    constexpr bool wide = sizeof(TG) == 2 && sizeof(TO) == 2;
    if (wide && vec == 8) grad_sum_kernel<TG, TO, wide ? 8 : 4, L><<<grid, SUM_THREADS, 0, s>>>(p);
    else if (vec == 4) grad_sum_kernel<TG, TO, 4, L><<<grid, SUM_THREADS, 0, s>>>(p);
    else if (vec == 2) grad_sum_kernel<TG, TO, 2, L><<<grid, SUM_THREADS, 0, s>>>(p);
    else grad_sum_kernel<TG, TO, 1, L><<<grid, SUM_THREADS, 0, s>>>(p);
    int rc = launch_status(cudaGetLastError());
    if (rc != KGE_OK || p.chunks < 3) return rc;
    const dim3 joins((unsigned)std::min<int64_t>(p.chunks / 2, 592), (unsigned)ceil_div(p.dim, 32));
    grad_join_kernel<TO, L><<<joins, JOIN_THREADS, 0, s>>>(p);
    return launch_status(cudaGetLastError());
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
    if (rows < 1 || rows > INT32_MAX || dim < 1 || n < 1) return 0;
    return carve_grad(nullptr, rows, dim, n).bytes;
}

int kge_embedding_grad(const int32_t* ids, int32_t n, const void* grads, int32_t grads_type, int64_t ld_grads, float scale, int32_t padding_id,
                       int32_t accumulate, void* table_grad, int32_t table_type, int64_t rows, int32_t dim, int64_t ld_table, void* scratch,
                       size_t scratch_bytes, int32_t* status, void* stream) {
    if (!is_float_type(grads_type) || !is_float_type(table_type) || rows < 1 || rows > INT32_MAX || dim < 1 || ld_grads < dim || ld_table < dim ||
        n < 0 || (accumulate != 0 && accumulate != 1)) return KGE_ERR_BAD_ARG;
    if (!table_grad || !aligned_to(table_grad, type_bytes(table_type)) || !aligned_to(status, 4)) return KGE_ERR_BAD_ARG;
    if (n > 0 && (!ids || !grads || !aligned_to(ids, 4) || !aligned_to(grads, type_bytes(grads_type)))) return KGE_ERR_BAD_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int gb = type_bytes(grads_type), tb = type_bytes(table_type);
    if (n == 0) {
        if (accumulate) return KGE_OK;
        return launch_status(cudaMemset2DAsync(table_grad, (size_t)ld_table * tb, 0, (size_t)dim * tb, (size_t)rows, s));
    }
    if (!scratch || !aligned_to(scratch, 256) || scratch_bytes < kge_embedding_grad_scratch_bytes(rows, dim, n)) return KGE_ERR_WORKSPACE;
    const GradScratch g = carve_grad(static_cast<char*>(scratch), rows, dim, n);
    const SortPlan plan = sort_plan(rows, n);
    const int digits = 1 << plan.bits;
    SortParams q{};
    q.ids = ids; q.n = n; q.tiles = plan.tiles; q.bits = plan.bits; q.passes = plan.passes; q.rows = (uint32_t)rows; q.padding_id = padding_id;
    q.hist = g.hist; q.total = g.total; q.list_count = g.list_count; q.status = status;
    q.scanned = plan.tiles > GS_DIRECT_TILES;
    int zero_ctas = 0;
    if (!accumulate) {
        q.zero = table_grad; q.zero_rows = rows; q.zero_row_bytes = (int64_t)dim * tb; q.zero_ld_bytes = ld_table * tb;
        q.zero_vec = ld_table == dim && aligned_to(table_grad, 16) && q.zero_row_bytes % 16 == 0;
        zero_ctas = (int)std::min<int64_t>(148 * 8, ceil_div(rows * q.zero_row_bytes, 16 * GS_THREADS));
    }
    grad_hist_kernel<<<plan.tiles + zero_ctas, GS_THREADS, 0, s>>>(q);
    int rc = launch_status(cudaGetLastError());
    for (int pass = 0; pass < plan.passes && rc == KGE_OK; ++pass) {
        q.pass = pass; q.shift = pass * plan.bits;
        q.keys_in = g.keys[(pass + 1) & 1]; q.pos_in = g.pos[(pass + 1) & 1];
        q.keys_out = g.keys[pass & 1]; q.pos_out = g.pos[pass & 1];
        q.hist = g.hist + (int64_t)pass * plan.tiles * digits;
        q.hist_next = pass + 1 < plan.passes ? q.hist + (int64_t)plan.tiles * digits : nullptr;
        if (q.scanned) {
            grad_scan_kernel<<<(digits + 31) / 32, 32, 0, s>>>(q);
            rc = launch_status(cudaGetLastError());
            if (rc != KGE_OK) break;
        }
        grad_scatter_kernel<<<plan.tiles, GS_THREADS, 0, s>>>(q);
        rc = launch_status(cudaGetLastError());
    }
    if (rc != KGE_OK) return rc;
    SumParams p{};
    p.keys = g.keys[(plan.passes - 1) & 1]; p.pos = g.pos[(plan.passes - 1) & 1];
    p.n = n; p.dim = dim; p.part_ld = (dim + 3) / 4 * 4; p.rows = (uint32_t)rows;
    p.chunks = (int)ceil_div(n, chunk_rows(n));
    p.grads = grads; p.ld_grads = ld_grads; p.out = table_grad; p.ld_out = ld_table; p.scale = scale; p.accumulate = accumulate;
    p.part = g.part; p.list = g.list; p.list_count = g.list_count;
    const int vec = vector_length(gb == 2 && tb == 2 ? 8 : 4, dim, ld_grads, gb, grads, ld_table, tb, table_grad);
    return with_type(grads_type, [&](auto a) {
        return with_type(table_type, [&](auto b) {
            using TG = decltype(a); using TO = decltype(b);
            return chunk_rows(n) == 8 ? launch_sum<TG, TO, 8>(p, vec, s) : launch_sum<TG, TO, 32>(p, vec, s);
        });
    });
}

}  // extern "C"
