// The norms' gradient kernels for fp16 rows of the residual stream.
#include "kge_norm_backward.cuh"

namespace kge {

int launch_norm_grad_f16(const NormGradParams& p, int block_type, int ctas, cudaStream_t s) {
    return with_type(block_type, [&](auto tb) { return launch_norm_grad<__half, decltype(tb)>(p, ctas, s); });
}

}  // namespace kge
