// r3_norm_residual and its gradient: checks, the plan of a launch, and the column sums behind the gradient.
#include <initializer_list>

#include "r3_norm.cuh"

namespace r3 {

// Column sums of the partial rows, in order; out[0] = dw_pre from plane 0, and from plane 1 (the
// sums of g n) out[1] = dw_post = branch_scale gate A and out[2] = dgate = branch_scale w_post A.
// COLS columns per CTA; 1024 / COLS groups of threads take the rows in turn, so that few loads follow one
// another.  32 columns are the better width for the memory (1023 x 8192 bf16: 5 us less than 16), 16 where
// 32 would leave SMs idle (4097 x 1160 float32: 1.5 us less).
struct NormSumArgs {
    const float* part;
    float* out[3];
    const void* w_post;
    const void* channel;
    int parts, d, w_bf16;
    float branch;
};
template <int COLS>
__global__ void __launch_bounds__(1024) norm_sum_kernel(const NormSumArgs a) {
    constexpr int TURNS = 1024 / COLS;
    __shared__ float s[TURNS][COLS + 1];
    if (!(blockIdx.y == 0 ? a.out[0] != nullptr : a.out[1] || a.out[2])) return;
    tc::grid_dependency_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int mine = threadIdx.x % COLS, turn = threadIdx.x / COLS, col = blockIdx.x * COLS + mine;
    const float* p = a.part + (size_t)blockIdx.y * a.parts * a.d;
    float v = 0.f;
    if (col < a.d) {
#pragma unroll 8
        for (int b = turn; b < a.parts; b += TURNS) v += p[(size_t)b * a.d + col];
    }
    s[turn][mine] = v;
    __syncthreads();
    // warp w < COLS takes column COLS blockIdx.x + w: its sums, added as a tree
    if (w >= COLS) return;
    v = s[lane][w];
#pragma unroll
    for (int k = 32; k < TURNS; k += 32) v += s[lane + k][w];
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) v += __shfl_xor_sync(0xffffffffu, v, k);
    const int c = blockIdx.x * COLS + w;
    if (lane != 0 || c >= a.d) return;
    if (blockIdx.y == 0) {
        a.out[0][c] = v;
        return;
    }
    auto weight = [&](const void* q) {
        if (!q) return 1.f;
        return a.w_bf16 ? to_f32(static_cast<const __nv_bfloat16*>(q)[c]) : static_cast<const float*>(q)[c];
    };
    v *= a.branch;
    if (a.out[1]) a.out[1][c] = v * weight(a.channel);
    if (a.out[2]) a.out[2][c] = v * weight(a.w_post);
}

// ---- host side ------------------------------------------------------------------------------------
constexpr int kNormRun = 8;                  // forward: rows per CTA of a large batch
constexpr int kNormMaxRows = 1 << 30;        // a few strides (of up to an eighth) ahead stay in 32 bits

static r3_status check_norm(const r3_norm* s) {
    if (!s) return R3_ERR_INVALID_ARG;
    if (s->T < 0 || s->T > kNormMaxRows || s->d <= 0 || s->d % 8 != 0) return R3_ERR_INVALID_ARG;
    if ((s->act_dtype != R3_F32 && s->act_dtype != R3_BF16) ||
        (s->w_dtype != R3_F32 && s->w_dtype != R3_BF16))
        return R3_ERR_INVALID_ARG;
    if (s->gate_kind < R3_GATE_NONE || s->gate_kind > R3_GATE_FULL) return R3_ERR_INVALID_ARG;
    if (!(s->eps > 0.f) || !(s->eps < 1e30f)) return R3_ERR_INVALID_ARG;
    if (!(s->residual_scale > -1e30f && s->residual_scale < 1e30f) ||
        !(s->branch_scale > -1e30f && s->branch_scale < 1e30f))
        return R3_ERR_INVALID_ARG;
    return R3_OK;
}

// Rows of up to 32 kNormPieces pieces: one warp each, several to a CTA.  Longer ones: a CTA with
// kNormPieces pieces per thread, twice as many past kNormPieces kNormMaxThreads pieces.  Rows of more
// than kNormBwdThreads threads are the wide form, which has fewer registers a thread.
static bool plan_norm(const r3_norm* s, bool bwd, NormPlan* p) {
    const int vecs = s->d / (s->act_dtype == R3_BF16 ? 8 : 4);
    p->pieces = kNormPieces;
    p->warp = vecs <= 32 * p->pieces;
    if (vecs > kNormMaxThreads * p->pieces) p->pieces *= 2;
    if (vecs > kNormMaxThreads * p->pieces) return false;
    p->threads = (vecs + 32 * p->pieces - 1) / (32 * p->pieces) * 32;
    p->wide = p->threads > kNormBwdThreads || p->pieces > kNormPieces;
    // Backward, rows of more than half the threads of an SM: two at a time, so that one's arithmetic stands
    // beside the other's reductions (8192 x 4096 bf16: 88 -> 82 us, 8192 x 2048 float32: 77 -> 70; shorter
    // rows lose: 8192 x 2560 bf16: 55 -> 76, 16384 x 2048: 76 -> 79, 16384 x 1160 float32: 89 -> 111).
    p->pair = bwd && p->threads > kNormBwdThreads / 2 && p->threads <= kNormPairThreads;
    const int resident = !bwd ? kNormFwdThreads
                              : norm_bwd_threads(p->wide, s->act_dtype == R3_F32, s->gate_kind == R3_GATE_FULL,
                                                 p->pair ? 2 : 1);
    int rows = 1;
    if (p->warp) {
        // backward, one CTA fills the SM with rows, so that their sums of the weight gradients leave it
        // as one; a small batch is spread over the SMs
        const int each = (int)(((long long)s->T + sm_count() - 1) / sm_count());
        rows = !bwd ? kWarpRows : each < resident / 32 ? each : resident / 32;
        if (rows < 1) rows = 1;
        p->threads = 32 * rows;
    }
    p->smem = (size_t)norm_stages(p->pieces, bwd) * norm_ring_bytes(p->pieces, bwd, p->threads) * (p->pair ? 2 : 1);
    int per_sm = resident / p->threads;
    const int by_smem = (int)(kNormRingBytes / p->smem);
    if (per_sm > by_smem) per_sm = by_smem;
    if (per_sm < 1) per_sm = 1;
    const int want = (int)(((long long)s->T + rows - 1) / rows), most = sm_count() * per_sm;
    p->grid = want < most ? want : most;
    // Forward, four CTAs or more per SM: CTAs of kNormRun rows each rather than as many as are resident at
    // once, since not all SMs see the memory at the same speed and the fast ones take more of them then
    // (65536 x 2048 bf16: 202 -> 177 us; with two CTAs per SM their starts show, 8192 x 4096: 49 -> 57).
    if (!bwd && per_sm >= 4 && want / kNormRun > most) p->grid = want / kNormRun;
    return true;
}

static r3_status launch_norm_types(const r3_norm* s, const NormArgs& a, const NormPlan& p, bool bwd,
                                   cudaStream_t cs) {
    return s->act_dtype == R3_BF16 ? launch_norm_bf16(s->w_dtype == R3_BF16, a, p, bwd, cs)
                                   : launch_norm_f32(s->w_dtype == R3_BF16, a, p, bwd, cs);
}
static NormArgs norm_args(const r3_norm* s) {
    NormArgs a = {};
    a.T = s->T;
    a.d = s->d;
    a.gate_kind = s->gate_kind;
    a.eps = s->eps;
    a.res = s->residual_scale;
    a.branch = s->branch_scale;
    return a;
}
static bool all_aligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (!aligned(p, 16)) return false;
    return true;
}

}  // namespace r3

extern "C" r3_status r3_norm_residual(const r3_norm* shape, const void* x, const void* y,
                                      const void* w_post, const void* gate, const void* w_pre,
                                      void* x_out, void* h, void* stream) {
    const r3_status st = r3::check_norm(shape);
    if (st != R3_OK) return st;
    r3::NormPlan plan;
    if (!r3::plan_norm(shape, false, &plan)) return R3_ERR_UNSUPPORTED;
    const bool gated = shape->gate_kind != R3_GATE_NONE;
    if (shape->T == 0) return R3_OK;
    if (!x || (!y && !w_pre) || (!y && (w_post || gated || x_out)) || (y && !x_out) ||
        gated != (gate != nullptr) || (w_pre != nullptr) != (h != nullptr) || (x_out && x_out == h))
        return R3_ERR_INVALID_ARG;
    if (!r3::all_aligned({x, y, w_post, w_pre, x_out, h}) ||
        !r3::aligned(gate, shape->gate_kind == R3_GATE_TOKEN ? 4 : 16))
        return R3_ERR_INVALID_ARG;
    r3::NormArgs a = r3::norm_args(shape);
    a.x = x;
    a.y = y;
    a.w_post = w_post;
    a.gate = gate;
    a.w_pre = w_pre;
    a.out0 = x_out;
    a.out1 = h;
    return r3::launch_norm_types(shape, a, plan, false, static_cast<cudaStream_t>(stream));
}

extern "C" size_t r3_norm_residual_bwd_workspace_bytes(const r3_norm* shape) {
    r3::NormPlan plan;
    if (r3::check_norm(shape) != R3_OK || !r3::plan_norm(shape, true, &plan)) return 0;
    return r3::round_up((size_t)2 * plan.grid * shape->d * sizeof(float), 256);
}

extern "C" r3_status r3_norm_residual_bwd(const r3_norm* shape, const void* x_out, const void* y,
                                          const void* w_post, const void* gate, const void* w_pre,
                                          const void* dx_out, const void* dh, void* dx, void* dy,
                                          float* dw_post, void* dgate, float* dw_pre,
                                          void* workspace, size_t ws_bytes, void* stream) {
    const r3_status st = r3::check_norm(shape);
    if (st != R3_OK) return st;
    r3::NormPlan plan;
    if (!r3::plan_norm(shape, true, &plan)) return R3_ERR_UNSUPPORTED;
    const bool gated = shape->gate_kind != R3_GATE_NONE, empty = shape->T == 0;
    // the weights and their gradients are there for an empty batch too: its sums are zero
    if ((w_post != nullptr) != (dw_post != nullptr) || (w_pre != nullptr) != (dw_pre != nullptr))
        return R3_ERR_INVALID_ARG;
    if (!empty && (!dx || (!y && !w_pre) || (!y && (w_post || gated)) ||
                   (y != nullptr) != (dy != nullptr) || gated != (gate != nullptr) ||
                   gated != (dgate != nullptr) || (w_pre && (!x_out || !dh)) ||
                   (!w_pre && (!dx_out || dh)) || dx == dy))
        return R3_ERR_INVALID_ARG;
    if (!r3::all_aligned({x_out, y, w_post, w_pre, dx_out, dh, dx, dy, dw_post, dw_pre}) ||
        !r3::aligned(gate, shape->gate_kind == R3_GATE_TOKEN ? 4 : 16) ||
        !r3::aligned(dgate, shape->gate_kind == R3_GATE_TOKEN ? 4 : 16))
        return R3_ERR_INVALID_ARG;
    const bool channel = shape->gate_kind == R3_GATE_CHANNEL && dgate;
    const bool sums = dw_pre || dw_post || channel;
    if (!empty && sums &&
        (!workspace || !r3::aligned(workspace, 256) ||
         ws_bytes < r3_norm_residual_bwd_workspace_bytes(shape)))
        return R3_ERR_WORKSPACE;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    r3::NormSumArgs sum = {};
    if (!empty) {
        r3::NormArgs a = r3::norm_args(shape);
        a.x = x_out;
        a.y = y;
        a.w_post = w_post;
        a.gate = gate;
        a.w_pre = w_pre;
        a.dx_out = dx_out;
        a.dh = dh;
        a.out0 = dx;
        a.out1 = dy;
        a.dgate = dgate;
        a.part = sums ? static_cast<float*>(workspace) : nullptr;
        const r3_status rc = r3::launch_norm_types(shape, a, plan, true, cs);
        if (rc != R3_OK) return rc;
        sum.part = a.part;
        sum.parts = plan.grid;
    }
    if (sums) {
        sum.out[0] = dw_pre;
        sum.out[1] = dw_post;
        sum.out[2] = channel ? static_cast<float*>(dgate) : nullptr;
        sum.w_post = w_post;
        sum.channel = shape->gate_kind == R3_GATE_CHANNEL ? gate : nullptr;
        sum.d = shape->d;
        sum.w_bf16 = shape->w_dtype == R3_BF16;
        sum.branch = shape->branch_scale;
        // launched while the rows are still being worked on; it waits for them itself
        const bool narrow = (shape->d + 31) / 32 * 2 < r3::sm_count();
        const int cols = narrow ? 16 : 32;
        if (r3::tc::launch_dependent(narrow ? r3::norm_sum_kernel<16> : r3::norm_sum_kernel<32>,
                                     dim3((shape->d + cols - 1) / cols, 2), dim3(1024), 0, cs,
                                     sum) != cudaSuccess) {
            cudaGetLastError();
            return R3_ERR_CUDA;
        }
    }
    return r3::launch_status();
}
