// The norms around a block: the entry point of the forward pass (the kernels: kge_norm_forward.cuh).
#include <cmath>

#include "kge_norm_forward.cuh"

using namespace kge;

extern "C" int kge_block_norm(const kge_norm_block* b, int64_t n, int32_t d, void* h, int64_t ldh, void* z, int32_t z_int8, int64_t ldz, float* z_scales,
                              float eps, float* stats, void* stream) {
    if (!b || !is_float_type(b->x_type) || !is_float_type(b->block_type) || n < 0 || n > INT32_MAX || d < 1 || d > INT32_MAX - 65536 || (b->layer != 0 && b->layer != 1) ||
        (b->gate && (b->gate_act < 0 || b->gate_act > 2)) || (z_int8 != 0 && z_int8 != 1) || !(eps >= 0.f) || std::isinf(eps)) return KGE_ERR_BAD_ARG;
    if (n == 0) return KGE_OK;
    if ((!h && !z) || (!b->y && (h || b->gate || b->post_weight || b->post_bias || b->scale))) return KGE_ERR_BAD_ARG;
    if ((b->post_bias && !b->post_weight) || (z && !b->pre_weight) || (z && z_int8 && !z_scales)) return KGE_ERR_BAD_ARG;
    const int xs = type_bytes(b->x_type), bs = type_bytes(b->block_type), zs = z_int8 ? 1 : bs;
    auto ok = [&](const void* p, int64_t ld, int size) { return !p || (ld >= d && aligned_to(p, (size_t)size)); };
    if (!b->x || !ok(b->x, b->ldx, xs) || !ok(b->y, b->ldy, bs) || !ok(b->gate, b->ld_gate, bs) || !ok(h, ldh, xs) || !ok(z, ldz, zs)) return KGE_ERR_BAD_ARG;
    const float* vectors[5] = {b->post_weight, b->post_bias, b->scale, b->pre_weight, b->pre_bias};
    // elements that move as one access: eight or two, where every row and vector starts at a multiple of them
    auto moves = [&](int w) {
        auto packs = [&](const void* p, int64_t ld, int size) { return !p || (ld % w == 0 && aligned_to(p, (size_t)(w * size))); };
        for (const float* v : vectors) if (!aligned_to(v, (size_t)(4 * std::min(w, 4)))) return false;
        return d % w == 0 && packs(b->x, b->ldx, xs) && packs(b->y, b->ldy, bs) && packs(b->gate, b->ld_gate, bs) && packs(h, ldh, xs) && packs(z, ldz, zs);
    };
    for (const float* v : vectors) if (!aligned_to(v, 4)) return KGE_ERR_BAD_ARG;
    if (!aligned_to(z_scales, 4) || !aligned_to(stats, 16)) return KGE_ERR_BAD_ARG;
    NormParams p{};
    p.x = b->x; p.y = b->y; p.gate = b->gate; p.h = h; p.z = z;
    p.w1 = b->post_weight; p.b1 = b->post_bias; p.scale = b->scale; p.w2 = b->pre_weight; p.b2 = b->pre_bias;
    p.stats = stats; p.z_scales = z_scales;
    p.ldx = b->ldx; p.ldy = b->ldy; p.ldg = b->ld_gate; p.ldh = ldh; p.ldz = ldz;
    p.n = (int)n; p.d = d; p.post = b->post_weight != nullptr; p.layer = b->layer; p.act = b->gate_act; p.z8 = z_int8; p.access = moves(8) ? 8 : (moves(2) ? 2 : 1);
    p.eps = eps; p.inv_d = 1.f / (float)d;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return b->x_type == KGE_F32 ? launch_norm_f32(p, b->block_type, s) : (b->x_type == KGE_BF16 ? launch_norm_bf16(p, b->block_type, s) : launch_norm_f16(p, b->block_type, s));
}
