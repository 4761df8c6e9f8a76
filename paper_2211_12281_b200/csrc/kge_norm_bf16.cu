// The norms' forward kernels for bf16 rows of the residual stream.
#include "kge_norm_forward.cuh"

namespace kge {

int launch_norm_bf16(const NormParams& p, int block_type, cudaStream_t s) {
    return with_type(block_type, [&](auto tb) { return launch_norm<__nv_bfloat16, decltype(tb)>(p, s); });
}

}  // namespace kge
