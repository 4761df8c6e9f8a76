// What the library's 8-bit products share: operand tiles through TMA, accumulators in tensor memory, and results on their way to memory.
#pragma once

#include <cuda.h>

#include <atomic>

#include "kge_ops.cuh"

namespace kge {

constexpr int OPERAND_BK = 128;            // bytes of K per tile: one 128-byte swizzle row
constexpr int OUT_COLS = 64;               // columns of a tile per epilogue warp

// Where a product's results go, and what is added to them.
struct ProductOut {
    int64_t M, N;
    const void* addend; int64_t ld_addend;
    void* out; int64_t ld_out; int out_type;
    int vec, twos;                        // rows of out (and addend) start at multiples of 16 bytes; of two elements, N even
};

// Tries of a product's bounded waits, unless a test shortens them.
inline std::atomic<int> product_wait_limit{kDefaultWaitLimit};

#ifdef __CUDACC__
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* tm, int x, int y, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}
// Shared-memory descriptor of a K-major operand tile with the 128-byte swizzle: rows of 128 bytes, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// The same for a pair of CTAs that share a tile (cta_group::2): a copy of a CTA's own operand rows completes on the first CTA's barrier, and a commit arrives
// at the barrier of the same place in both.
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma_commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// Arrivals at a barrier of the cluster, and a wait that sees what was written before them.  (The second kind of arrival says what a copy will bring, and has nothing
// of its own to be seen: ordered like the first, and waited for like it, it cost a block of K three times its MMAs.)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mbar_arrive_expect_tx_cluster(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity, int limit) {
    for (int i = 0; i < limit; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(2000u) : "memory");
        if (ok) return true;
        __nanosleep(96);
    }
    return false;
}
__device__ __forceinline__ uint32_t cluster_ld_word(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void copy4_async(uint32_t dst, const float* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 16 consecutive columns of this thread's tensor-memory lane.  Nothing may look at the registers before tmem_wait16 has passed them on.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
// Waits for this thread's tensor-memory loads; the registers pass through, so that nothing that uses them moves ahead.
__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ uint64_t two_words(uint32_t a, uint32_t b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b)); return r; }
// Registers of a warpgroup, out of what the block was launched with.
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// Calls f with a value of the output type.
template <class F> __device__ __forceinline__ void with_out_type(int t, F&& f) {
    if (t == KGE_F32) f(float());
    else if (t == KGE_BF16) f(__nv_bfloat16());
    else f(__half());
}

// A pack of a row's columns.
template <typename TO, int V>
__device__ __forceinline__ void out_put(const ProductOut& p, int row, int col, const Pack<TO, V>& o) {
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
__device__ __forceinline__ void out_each(const ProductOut& p, int row0, int col0, float4* st, int lane, F&& f) {
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
__device__ __forceinline__ void out_store(const ProductOut& p, int row0, int col0, const uint64_t (&acc)[OUT_COLS / 2], float4* st, int lane) {
    constexpr int V = 16 / sizeof(TO), UNITS = ROW / 16, PASS = ROW / sizeof(TO);      // columns per unit, units and columns per pass
    constexpr int TURN = UNITS == 2 ? 2 : 0;                                            // rows 4 apart share banks at 32 bytes a row
    // a warp's part that lies inside the matrix is stored without a look at its edges
    const bool inside = p.vec && row0 + 32 <= p.M && col0 + OUT_COLS <= p.N;
    TO* const first = static_cast<TO*>(p.out) + (row0 + lane / UNITS) * p.ld_out + col0 + V * (lane % UNITS);
    const int64_t step = (32 / UNITS) * p.ld_out;
#pragma unroll
    for (int c = 0; c < OUT_COLS; c += PASS) {
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
            out_each<TO, ROW, 2>(p, row0, col0 + c, st, lane, [&](int row, int col, TO* at) {
                *reinterpret_cast<uint32_t*>(static_cast<TO*>(p.out) + row * p.ld_out + col) = *reinterpret_cast<const uint32_t*>(at);
            });
        } else {
            out_each<TO, ROW, 1>(p, row0, col0 + c, st, lane, [&](int row, int col, TO* at) { static_cast<TO*>(p.out)[row * p.ld_out + col] = *at; });
        }
        __syncwarp();
    }
}

// The addend of the same tile joins the accumulators in fp32 before they are rounded.
// With 128-byte rows it passes through the warp's shared memory: out_fetch_addend starts the copies of a pass (the first one's while
// the tile is computed), out_add_staged waits for them.
// (a copy takes 16 bytes, or 4: two 16-bit elements; rows of 16-bit elements that start in between are read by the lanes themselves)
template <typename TO>
__device__ __forceinline__ void out_fetch_addend(const ProductOut& p, int row0, int col0, int c, float4* st, int lane) {
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
        out_each<TO, 128, FOUR>(p, row0, col0 + c, st, lane, [&](int row, int col, TO* at) { copy4_async(smem_u32(at), reinterpret_cast<const float*>(add + row * p.ld_addend + col)); });
    } else {
        // (sixteen loads under way: 13,555 x 1,119 bf16 in 8 bits, K = 2,536, with an addend: 121 us with four, 80)
        constexpr int ROWS = 8, COLS = 128 / (int)sizeof(TO) / 32;
        TO* const own = reinterpret_cast<TO*>(st);
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += ROWS) {
            TO v[ROWS * COLS];
#pragma unroll
            for (int i = 0; i < ROWS * COLS; ++i) {
                const int row = row0 + r0 + i / COLS, col = col0 + c + i % COLS * 32 + lane;
                v[i] = row < p.M && col < p.N ? add[row * p.ld_addend + col] : from_float<TO>(0.f);
            }
#pragma unroll
            for (int i = 0; i < ROWS * COLS; ++i) {
                const int r = r0 + i / COLS, x = i % COLS * 32 + lane;
                own[(r * 8 + ((x / V) ^ (r & 7))) * V + x % V] = v[i];
            }
        }
    }
}
template <typename TO>
__device__ __forceinline__ void out_add_staged(const ProductOut& p, int row0, int col0, uint64_t (&acc)[OUT_COLS / 2], float4* st, int lane) {
    constexpr int V = 16 / sizeof(TO), PASS = 128 / sizeof(TO);
#pragma unroll
    for (int c = 0; c < OUT_COLS; c += PASS) {
        if (c > 0) out_fetch_addend<TO>(p, row0, col0, c, st, lane);
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
__device__ __forceinline__ void out_add_rows(const ProductOut& p, int row, int col0, uint64_t (&acc)[OUT_COLS / 2]) {
    constexpr int V = 16 / sizeof(TO);
    if (row >= p.M) return;
    const TO* const add = static_cast<const TO*>(p.addend) + row * p.ld_addend + col0;
    if (p.vec && col0 + OUT_COLS <= p.N) {
#pragma unroll
        for (int c = 0; c < OUT_COLS; c += V) {
            const Pack<TO, V> a = *reinterpret_cast<const Pack<TO, V>*>(add + c);
#pragma unroll
            for (int e = 0; e < V; e += 2) acc[(c + e) / 2] = add2(acc[(c + e) / 2], pair(to_float(a.v[e]), to_float(a.v[e + 1])));
        }
    } else {
#pragma unroll
        for (int c = 0; c < OUT_COLS; ++c) {
            if (col0 + c < p.N) acc[c / 2] = add2(acc[c / 2], c & 1 ? pair(0.f, to_float(add[c])) : pair(to_float(add[c]), 0.f));
        }
    }
}
template <typename TO>
__device__ __forceinline__ void out_prefetch_addend(const ProductOut& p, int row, int col0) {
    if (row >= p.M) return;
    const char* add = reinterpret_cast<const char*>(static_cast<const TO*>(p.addend) + row * p.ld_addend + col0);
#pragma unroll
    for (int b = 0; b < OUT_COLS * (int)sizeof(TO); b += 128)
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

#endif

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline int operand_map(CUtensorMap* map, const void* base, int64_t rows, int64_t k, int64_t ld, int box_rows) {
    static const EncodeTiledFn fn = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiledFn>(ptr) : nullptr;
    }();
    if (!fn) return KGE_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {OPERAND_BK, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? KGE_OK : KGE_ERR_CUDA;
}

}  // namespace kge
