// Shared by the two forms of the orthogonalised update (r3_muon.cu, r3_muon_small.cu).
#pragma once

#include <cuda_fp16.h>

#include "r3_common.cuh"
#include "r3_internal.h"
#include "r3_tc.cuh"

namespace r3 {
namespace ns {

using namespace tc;

// An fp16 operand is its value times a power of two, the largest that keeps all iterates within MAX_HALF (2^14 for
// the usual coefficients).  Its lo plane holds what hi leaves times LO more, or small elements would lose it
// (without that, and with 2^10 for all, rows a millionth of the others were 7e-3 off in float32 results, with both 8e-7).
constexpr float LEAST_SCALE = 1024.f, MOST_SCALE = 16384.f, MAX_HALF = 61440.f;
constexpr int LO_SHIFT = 11;              // (a value within MAX_HALF leaves 16 at most)
constexpr float LO = 1 << LO_SHIFT;
constexpr int MAX_STACKS = 64;            // per launch: the table travels in the kernel's parameters
constexpr int MAX_STEPS = 16;

__device__ __forceinline__ void fence_async() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ bool scale_of(const float* grad_scale, float* s) {
    *s = grad_scale ? *grad_scale : 1.f;
    return isfinite(*s);
}
// Eight consecutive elements as float32.
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
    constexpr int N = Vec16<T>::N;
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) {
        Vec16<T> v;
        v.v = *reinterpret_cast<const decltype(v.v)*>(p + i * N);
        v.unpack(f + i * N);
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
    constexpr int N = Vec16<T>::N;
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) {
        Vec16<T> v;
        v.pack(f + i * N);
        *reinterpret_cast<decltype(v.v)*>(p + i * N) = v.v;
    }
}
// u from the gradient and the momentum after this step; every product and sum is rounded by itself.
__device__ __forceinline__ float direction(bool nesterov, float momentum, bool has, float g, float m) {
    if (!has) return g;
    return nesterov ? __fadd_rn(g, __fmul_rn(momentum, m)) : m;
}
// What u is multiplied with to give X times LEAST_SCALE.  A matrix of zeros stays one; anything not finite reaches
// every element.
__device__ __forceinline__ float start_scale(double sum, float eps) {
    const double norm = sqrt(sum);
    return norm == 0.0 ? 0.f : (float)((double)LEAST_SCALE / (norm + (double)eps));
}

// ---- matrices whose smaller side is at most SMALL_SIDE: r3_muon_small.cu ---------------------------------
constexpr int SMALL_SIDE = 128;
constexpr int SMALL_SLAB = 256;           // columns of X per CTA
constexpr int SMALL_CTAS = 8;             // CTAs of a cluster at most

struct SmallStack {
    void* param;                          // or the result of an orthogonalisation
    float* master;                        // or null
    const void* grad;                     // or its input
    float* momentum;                      // null: none
    int first, rows, cols;                // number of its first matrix in the launch
    float decay, scale;
};
struct SmallArgs {
    int stacks, cluster, steps;
    int grad_dtype, param_dtype, step, nesterov;
    int x_blocks, a_blocks, a_bytes, tmem_cols;      // set by run_small
    float momentum, eps, lr, scale;       // scale: of the operands
    float coefs[MAX_STEPS][3];
    const float *grad_scale, *lr_now;
    int32_t* dev_status;
    SmallStack stack[MAX_STACKS];
};
// CTAs per matrix, or 0 where this form does not take the shape.
int small_cluster(int rows, int cols);
// One launch over all stacks of `a` (all of a.cluster CTAs per matrix).
r3_status run_small(SmallArgs& a, int terms, int matrices, cudaStream_t cs);

}  // namespace ns
}  // namespace r3
