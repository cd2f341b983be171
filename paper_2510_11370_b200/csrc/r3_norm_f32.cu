// The norm kernels for float32 rows.
#include "r3_norm.cuh"

namespace r3 {

r3_status launch_norm_f32(bool w_bf16, const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs) {
    return w_bf16 ? launch_norm_size<float, __nv_bfloat16>(a, p, bwd, cs)
                  : launch_norm_size<float, float>(a, p, bwd, cs);
}

}  // namespace r3
