// The norm kernels for bfloat16 rows.
#include "r3_norm.cuh"

namespace r3 {

r3_status launch_norm_bf16(bool w_bf16, const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs) {
    return w_bf16 ? launch_norm_size<__nv_bfloat16, __nv_bfloat16>(a, p, bwd, cs)
                  : launch_norm_size<__nv_bfloat16, float>(a, p, bwd, cs);
}

}  // namespace r3
