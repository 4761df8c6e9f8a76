// The gradients of the norms around a block: the entry point, and the join of the columns' sums (the kernels: kge_norm_backward.cuh).
#include "kge_norm_backward.cuh"

namespace kge {

namespace {

// The CTAs' sums, added in their order; then what the vectors' gradients are.
struct NormJoinParams {
    const float* part;
    const float *w1, *b1, *scale;
    float *dw1, *db1, *dscale, *dw2, *db2;
    int ctas, sums, d, accumulate;
};
// Eight columns (a sector of 32 bytes) to a CTA: its warps take four rows of sums at a time (24,576 x 256, both kernels: 37.7 us, with 32 columns and 32 rows at a time 39.3).
constexpr int JOIN_COLS = 8, JOIN_WARPS = 32;
__global__ void __launch_bounds__(32 * JOIN_WARPS) norm_join_kernel(const __grid_constant__ NormJoinParams p) {
    __shared__ float part[4][JOIN_WARPS][JOIN_COLS], sum[4][JOIN_COLS];
    grid_dependency_wait();
    allow_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = lane % JOIN_COLS, c = blockIdx.x * JOIN_COLS + col;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < p.d) {
#pragma unroll 2
        for (int g = warp * 4 + lane / JOIN_COLS; g < p.ctas; g += JOIN_WARPS * 4) {
#pragma unroll
            for (int q = 0; q < 4; ++q) if (q < p.sums) v[q] += p.part[((int64_t)g * p.sums + q) * p.d + c];
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v[q] += __shfl_xor_sync(0xffffffffu, v[q], 8);
        v[q] += __shfl_xor_sync(0xffffffffu, v[q], 16);
        if (lane < JOIN_COLS) part[q][warp][col] = v[q];
    }
    __syncthreads();
    if (warp > 0) return;
    float s = 0.f;
#pragma unroll 8
    for (int w = 0; w < JOIN_WARPS; ++w) s += part[lane / JOIN_COLS][w][col];
    sum[lane / JOIN_COLS][col] = s;
    __syncwarp();
    if (lane >= JOIN_COLS || c >= p.d) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = sum[q][col];
    auto give = [&](float* to, float x) { if (to) to[c] = p.accumulate ? to[c] + x : x; };
    const float scale = p.scale ? p.scale[c] : 1.f, w1 = p.w1 ? p.w1[c] : 1.f, b1 = p.b1 ? p.b1[c] : 0.f;
    give(p.dw2, v[0]);
    give(p.db2, v[2]);
    give(p.dw1, scale * v[1]);
    give(p.db1, scale * v[3]);
    give(p.dscale, p.b1 ? fmaf(w1, v[1], b1 * v[3]) : w1 * v[1]);
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
        auto moves = [&](int w) {
            auto packs = [&](const void* p, int64_t ld, int size) { return !p || (ld % w == 0 && aligned_to(p, (size_t)(w * size))); };
            for (int i = 0; i < 4; ++i) if (!aligned_to(vectors[i], (size_t)(4 * std::min(w, 4)))) return false;
            return d % w == 0 && packs(b->x, b->ldx, xs) && packs(b->y, b->ldy, bs) && packs(b->gate, b->ld_gate, bs) && packs(dz, ld_dz, bs) && packs(dh, ld_dh, xs) &&
                   packs(o->dx, o->ld_dx, xs) && packs(o->dy, o->ld_dy, bs) && packs(o->dgate, o->ld_dgate, bs);
        };
        NormGradParams p{};
        p.access = moves(8) ? 8 : (moves(2) ? 2 : 1);
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
        const int rc = b->x_type == KGE_F32 ? launch_norm_grad_f32(p, b->block_type, ctas, s)
                                            : (b->x_type == KGE_BF16 ? launch_norm_grad_bf16(p, b->block_type, ctas, s) : launch_norm_grad_f16(p, b->block_type, ctas, s));
        if (rc != KGE_OK) return rc;
        j.part = p.part; j.ctas = ctas;
    }
    if (!wanted || (n == 0 && accumulate)) return KGE_OK;
    return launch_status(launch_dependent(norm_join_kernel, dim3((unsigned)ceil_div(d, JOIN_COLS)), dim3(32 * JOIN_WARPS), 0, s, j));
}

}  // extern "C"
