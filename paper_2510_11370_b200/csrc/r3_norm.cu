// What stands between two replayed blocks: RMSNorm of the block's output, its gate, the scaled
// residual, and the RMSNorm in front of the next block, in one pass over the rows; and the gradients
// of all of it in one pass.
//
//   n     = y rsqrt(mean(y^2) + eps) w_post          (n = y without w_post)
//   x_out = residual_scale x + branch_scale gate n
//   h     = x_out rsqrt(mean(x_out^2) + eps) w_pre
//
// Bound by HBM: forward 4 rows moved per token (x, y in; x_out, h out), backward 6 (x_out, y,
// dx_out, dh in; dx, dy out); each element is read once and stays in registers through both row
// reductions.  A row belongs to a group of threads, the whole CTA or (rows of up to kWarpPieces
// pieces per lane) one warp, which then needs no barrier.  A thread owns P pieces of 16 bytes of
// the row and walks over the rows with a stride, so that the sums of the weight gradients stay in
// its registers.  What hides the memory latency is a ring in shared memory that is private to the
// thread: it copies its own pieces of the rows to come there (cp.async), S rows ahead, so no
// barrier or wait between threads belongs to the copies.
#include <initializer_list>

#include "r3_common.cuh"
#include "r3_internal.h"
#include "r3_tc.cuh"

namespace r3 {

constexpr int kNormMaxThreads = 512;
constexpr int kWarpPieces = 2;         // P of the one-warp form
constexpr int kWarpRows = 4;           // its warps (rows) per CTA

struct NormArgs {
    const void* x;          // forward: x.  backward: x_out
    const void* y;
    const void* w_post;
    const void* gate;
    const void* w_pre;
    const void* dx_out;     // backward
    const void* dh;
    void* out0;             // forward: x_out.  backward: dx
    void* out1;             // forward: h.      backward: dy
    void* dgate;            // backward: [T] float32 or [T, d] act (per-column sums go to part)
    float* part;            // backward: [3][grid][d] partial sums of dw_pre, dw_post, dgate
    int T, d, gate_kind;
    float eps, res, branch;
};

__device__ __forceinline__ void copy_ahead(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                 ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// Sum of NV values over the threads of a row's group; every thread gets the result.  For a CTA
// one barrier per call: the caller alternates buffers, so that a buffer is only written again
// behind the barrier of the call in between.
template <int NV, bool WARP>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*red)[4], int warps) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], s);
    }
    if (WARP) return;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) red[threadIdx.x >> 5][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = 0.f;
    for (int w = 0; w < warps; ++w) {                                    // fixed order
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] += red[w][i];
    }
}

// N values (one 16-byte piece of activations) of a vector of type W, from column `col` on.
template <typename W, int N>
__device__ __forceinline__ void load_cols(const void* p, int col, float* f) {
    constexpr int M = Vec16<W>::N;
    const W* w = static_cast<const W*>(p) + col;
    if (M <= N) {
#pragma unroll
        for (int i = 0; i < N; i += M) {
            const Vec16<W> v = *reinterpret_cast<const Vec16<W>*>(w + i);
            float t[M];
            v.unpack(t);
#pragma unroll
            for (int k = 0; k < M; ++k) f[(i + k) % N] = t[k];
        }
    } else {                                       // 4 f32 columns of a bf16 vector: 8 bytes
        const uint2 v = *reinterpret_cast<const uint2*>(w);
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float2 t = __bfloat1622float2(h[i]);
            f[2 * i] = t.x;
            f[2 * i + 1] = t.y;
        }
    }
}
template <typename T> __device__ __forceinline__ void store_piece(void* p, size_t at, const float* f) {
    Vec16<T> o;
    o.pack(f);
    *reinterpret_cast<Vec16<T>*>(static_cast<T*>(p) + at) = o;
}

template <typename T, typename W, int P, bool WARP, int S>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_kernel(const NormArgs a) {
    constexpr int N = Vec16<T>::N;
    extern __shared__ uint4 ring_all[];            // [S][2 P][threads]
    __shared__ float s_red[2][kNormMaxThreads / 32][4];
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, group = WARP ? 32 : blockDim.x;
    const int warps = blockDim.x >> 5;
    const int stride = WARP ? gridDim.x * warps : gridDim.x;
    const int row0 = WARP ? blockIdx.x * warps + (threadIdx.x >> 5) : blockIdx.x;
    const float inv_d = 1.f / (float)a.d;
    uint4* ring = ring_all + threadIdx.x;
    auto slot = [&](int stage, int q) { return ring + (size_t)(stage * 2 * P + q) * blockDim.x; };
    auto fetch = [&](int row, int stage) {
        if (row < a.T) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int col = (p * group + tid) * N;
                if (col >= a.d) continue;
                const size_t at = (size_t)row * a.d + col;
                copy_ahead(slot(stage, 2 * p), static_cast<const T*>(a.x) + at);
                if (a.y) copy_ahead(slot(stage, 2 * p + 1), static_cast<const T*>(a.y) + at);
            }
        }
        copy_commit();                             // one group per row, empty ones behind the last
    };
#pragma unroll
    for (int s = 0; s < S; ++s) fetch(row0 + s * stride, s);
    int stage = 0;
    for (int row = row0; row < a.T; row += stride) {
        const size_t base = (size_t)row * a.d;
        copy_wait<S - 1>();
        float x[P][N], y[P][N];
        float s[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const bool in = (p * group + tid) * N < a.d;
#pragma unroll
            for (int i = 0; i < N; ++i) x[p][i] = y[p][i] = 0.f;
            if (in) {
                reinterpret_cast<const Vec16<T>*>(slot(stage, 2 * p))->unpack(x[p]);
                if (a.y) reinterpret_cast<const Vec16<T>*>(slot(stage, 2 * p + 1))->unpack(y[p]);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) s[0] = fmaf(y[p][i], y[p][i], s[0]);
        }
        fetch(row + S * stride, stage);
        stage = stage + 1 == S ? 0 : stage + 1;
        float r = 1.f;
        if (a.w_post) {
            row_sum<1, WARP>(s, s_red[0], warps);
            r = rsqrtf(s[0] * inv_d + a.eps);
        }
        if (a.y) {
            float k = a.branch;
            if (a.gate_kind == R3_GATE_TOKEN) k *= static_cast<const float*>(a.gate)[row];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int col = (p * group + tid) * N;
                if (col >= a.d) continue;
                float g[N], w[N];
#pragma unroll
                for (int i = 0; i < N; ++i) g[i] = w[i] = 1.f;
                if (a.w_post) load_cols<W, N>(a.w_post, col, w);
                if (a.gate_kind == R3_GATE_CHANNEL) load_cols<W, N>(a.gate, col, g);
                if (a.gate_kind == R3_GATE_FULL)
                    load_cols<T, N>(static_cast<const T*>(a.gate) + base, col, g);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[p][i] = a.res * x[p][i] + k * (g[i] * (y[p][i] * r * w[i]));
                store_piece<T>(a.out0, base + col, x[p]);
            }
        }
        if (a.w_pre) {
            s[0] = 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < N; ++i) s[0] = fmaf(x[p][i], x[p][i], s[0]);
            row_sum<1, WARP>(s, s_red[1], warps);
            r = rsqrtf(s[0] * inv_d + a.eps);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int col = (p * group + tid) * N;
                if (col >= a.d) continue;
                float w[N];
                load_cols<W, N>(a.w_pre, col, w);
#pragma unroll
                for (int i = 0; i < N; ++i) w[i] *= x[p][i] * r;
                store_piece<T>(a.out1, base + col, w);
            }
        }
        // with one reduction per row its buffer comes around without a barrier in between
        if (!WARP && (!a.w_post || !a.w_pre)) __syncthreads();
    }
    copy_wait<0>();
}

// Backward.  With x = x_out, m = x r the pre-normalised row (r = rsqrt(mean(x^2) + eps)),
// u = dh w_pre and c = mean(u m):
//   g  = dx_out + r (u - m c);      dw_pre += dh m;      dx = residual_scale g
// and with q = branch_scale g, t = q gate, n = y s (s = rsqrt(mean(y^2) + eps)), e = mean(t w_post n):
//   dw_post += t n;    dgate = q n w_post (summed over what the gate is broadcast along);
//   dy = s (t w_post - n e)
// e and a token's dgate need g, so a row takes two reductions.
template <typename T, typename W, int P, bool WARP, int S>
__global__ void __launch_bounds__(kNormMaxThreads) norm_bwd_kernel(const NormArgs a) {
    constexpr int N = Vec16<T>::N;
    extern __shared__ uint4 ring_all[];            // [S][4 P][threads]
    __shared__ float s_red[2][kNormMaxThreads / 32][4];
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, group = WARP ? 32 : blockDim.x;
    const int warps = blockDim.x >> 5;
    const int stride = WARP ? gridDim.x * warps : gridDim.x;
    const int row0 = WARP ? blockIdx.x * warps + (threadIdx.x >> 5) : blockIdx.x;
    const float inv_d = 1.f / (float)a.d;
    uint4* ring = ring_all + threadIdx.x;
    auto slot = [&](int stage, int q) { return ring + (size_t)(stage * 4 * P + q) * blockDim.x; };
    auto fetch = [&](int row, int stage) {
        if (row < a.T) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int col = (p * group + tid) * N;
                if (col >= a.d) continue;
                const size_t at = (size_t)row * a.d + col;
                if (a.w_pre) {
                    copy_ahead(slot(stage, 4 * p), static_cast<const T*>(a.x) + at);
                    copy_ahead(slot(stage, 4 * p + 1), static_cast<const T*>(a.dh) + at);
                }
                if (a.dx_out) copy_ahead(slot(stage, 4 * p + 2), static_cast<const T*>(a.dx_out) + at);
                if (a.y) copy_ahead(slot(stage, 4 * p + 3), static_cast<const T*>(a.y) + at);
            }
        }
        copy_commit();
    };
    float acc_pre[P][N], acc_post[P][N], acc_gate[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < N; ++i) acc_pre[p][i] = acc_post[p][i] = acc_gate[p][i] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) fetch(row0 + s * stride, s);
    int stage = 0;
    for (int row = row0; row < a.T; row += stride) {
        const size_t base = (size_t)row * a.d;
        copy_wait<S - 1>();
        Vec16<T> xv[P], hv[P], yv[P];
        float g[P][N];
        float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * group + tid) * N;
            float w[N], f[N];
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = w[i] = g[p][i] = 0.f;
            xv[p].pack(f);
            hv[p].pack(f);
            yv[p].pack(f);
            if (col >= a.d) continue;
            if (a.w_pre) {
                xv[p] = *reinterpret_cast<const Vec16<T>*>(slot(stage, 4 * p));
                hv[p] = *reinterpret_cast<const Vec16<T>*>(slot(stage, 4 * p + 1));
                load_cols<W, N>(a.w_pre, col, w);
                float h[N];
                xv[p].unpack(f);
                hv[p].unpack(h);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    s[0] = fmaf(f[i], f[i], s[0]);
                    s[1] = fmaf(h[i] * w[i], f[i], s[1]);
                }
            }
            if (a.dx_out) reinterpret_cast<const Vec16<T>*>(slot(stage, 4 * p + 2))->unpack(g[p]);
            if (a.y) {
                yv[p] = *reinterpret_cast<const Vec16<T>*>(slot(stage, 4 * p + 3));
                yv[p].unpack(f);
#pragma unroll
                for (int i = 0; i < N; ++i) s[2] = fmaf(f[i], f[i], s[2]);
            }
        }
        fetch(row + S * stride, stage);
        stage = stage + 1 == S ? 0 : stage + 1;
        row_sum<3, WARP>(s, s_red[0], warps);
        const float r = rsqrtf(s[0] * inv_d + a.eps);
        const float c = s[1] * r * inv_d;                       // mean(u m)
        const float sy = a.w_post ? rsqrtf(s[2] * inv_d + a.eps) : 1.f;
        const float token =
            a.gate_kind == R3_GATE_TOKEN ? static_cast<const float*>(a.gate)[row] : 1.f;
        float z[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * group + tid) * N;
            if (col >= a.d) continue;
            float w[N], f[N];
            if (a.w_pre) {
                float h[N];
                load_cols<W, N>(a.w_pre, col, w);
                xv[p].unpack(f);
                hv[p].unpack(h);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float m = f[i] * r;
                    acc_pre[p][i] = fmaf(h[i], m, acc_pre[p][i]);
                    g[p][i] += r * (h[i] * w[i] - m * c);
                }
            }
            const float res = a.y ? a.res : 1.f;
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = res * g[p][i];
            store_piece<T>(a.out0, base + col, f);
            if (!a.y) continue;
            float gate[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                w[i] = 1.f;
                gate[i] = token;
            }
            if (a.w_post) load_cols<W, N>(a.w_post, col, w);
            if (a.gate_kind == R3_GATE_CHANNEL) load_cols<W, N>(a.gate, col, gate);
            if (a.gate_kind == R3_GATE_FULL)
                load_cols<T, N>(static_cast<const T*>(a.gate) + base, col, gate);
            yv[p].unpack(f);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float q = a.branch * g[p][i], n = f[i] * sy, t = q * gate[i];
                f[i] = q * n * w[i];                            // dgate of this element
                acc_post[p][i] = fmaf(t, n, acc_post[p][i]);
                g[p][i] = t * w[i];
                z[0] = fmaf(g[p][i], n, z[0]);
                z[1] += f[i];
            }
            if (a.gate_kind == R3_GATE_CHANNEL) {
#pragma unroll
                for (int i = 0; i < N; ++i) acc_gate[p][i] += f[i];
            }
            if (a.gate_kind == R3_GATE_FULL) store_piece<T>(a.dgate, base + col, f);
        }
        if (a.y) {
            row_sum<2, WARP>(z, s_red[1], warps);
            const float e = a.w_post ? z[0] * inv_d * sy : 0.f;
            if (a.gate_kind == R3_GATE_TOKEN && tid == 0) static_cast<float*>(a.dgate)[row] = z[1];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int col = (p * group + tid) * N;
                if (col >= a.d) continue;
                float f[N];
                yv[p].unpack(f);
#pragma unroll
                for (int i = 0; i < N; ++i) f[i] = sy * (g[p][i] - f[i] * e);
                store_piece<T>(a.out1, base + col, f);
            }
        } else if (!WARP) {
            __syncthreads();                                    // see the forward kernel
        }
    }
    copy_wait<0>();
    if (!a.part) return;
    // One row of partial sums per CTA.  In the one-warp form the warps add theirs up in order first.
    const size_t plane = (size_t)gridDim.x * a.d;
    float* mine = a.part + (size_t)blockIdx.x * a.d;
    const bool wanted[3] = {a.w_pre != nullptr, a.w_post != nullptr, a.gate_kind == R3_GATE_CHANNEL};
    float* sums = reinterpret_cast<float*>(ring_all);           // [warps][P N 32], the ring is idle
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (!wanted[k]) continue;
        float(&acc)[P][N] = k == 0 ? acc_pre : k == 1 ? acc_post : acc_gate;
        if (WARP) {
            __syncthreads();
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sums[((threadIdx.x >> 5) * P * N + p * N + i) * 32 + tid] = acc[p][i];
            __syncthreads();
            if (threadIdx.x >= 32) continue;
            for (int w = 1; w < warps; ++w)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[p][i] += sums[(w * P * N + p * N + i) * 32 + tid];
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int col = (p * group + tid) * N;
            if (col >= a.d) continue;
#pragma unroll
            for (int i = 0; i < N; i += 4)
                *reinterpret_cast<float4*>(mine + k * plane + col + i) =
                    make_float4(acc[p][i], acc[p][i + 1], acc[p][i + 2], acc[p][i + 3]);
        }
    }
}

// Column sums of the partial rows, in order: out[k][c] = sum_b part[k][b][c].
struct NormSumArgs {
    const float* part;
    float* out[3];
    int parts, d;
};
__global__ void __launch_bounds__(256) norm_sum_kernel(const NormSumArgs a) {
    __shared__ float s[8][32];
    float* out = a.out[blockIdx.y];
    if (!out) return;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    const float* p = a.part + (size_t)blockIdx.y * a.parts * a.d;
    float v = 0.f;
    if (col < a.d)
        for (int b = w; b < a.parts; b += 8) v += p[(size_t)b * a.d + col];
    s[w][lane] = v;
    __syncthreads();
    if (w == 0 && col < a.d) {
        v = s[0][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) v += s[k][lane];
        out[col] = v;
    }
}

// ---- host side ------------------------------------------------------------------------------------
constexpr int kNormMaxPieces = 4;
constexpr int kNormRingBytes = 200 * 1024;   // of an SM's shared memory, for the rings of its CTAs
constexpr int kNormMaxRows = 0x7f000000;     // row numbers a few strides ahead stay in 32 bits

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

struct NormPlan {
    int pieces, threads, grid, stages;
    bool warp;
    size_t smem;
};
// Rows of up to 32 kWarpPieces pieces go to one warp each.  Longer ones take a CTA with the
// least number of pieces per thread (1, 2 or 4) that leaves at most kNormMaxThreads threads.
static bool plan_norm(const r3_norm* s, bool bwd, NormPlan* p) {
    const int n = s->act_dtype == R3_BF16 ? 8 : 4, vecs = s->d / n;
    p->warp = vecs <= 32 * kWarpPieces;
    if (p->warp) {
        p->pieces = kWarpPieces;
        p->threads = 32 * kWarpRows;
    } else {
        for (p->pieces = 1; (vecs + p->pieces - 1) / p->pieces > kNormMaxThreads; p->pieces *= 2) {}
        if (p->pieces > kNormMaxPieces) return false;
        p->threads = ((vecs + p->pieces - 1) / p->pieces + 31) / 32 * 32;
    }
    p->stages = p->pieces == 4 ? 1 : 3;
    p->smem = (size_t)p->stages * (bwd ? 4 : 2) * p->pieces * p->threads * 16;
    // resident CTAs: what the registers allow (64 to 128 a thread), at most what the ring allows
    int per_sm = (bwd ? 640 : 1280) / p->threads;
    const int by_smem = (int)(kNormRingBytes / p->smem);
    if (per_sm > by_smem) per_sm = by_smem;
    if (per_sm < 1) per_sm = 1;
    const int rows = p->warp ? kWarpRows : 1;
    const int want = (s->T + rows - 1) / rows, most = sm_count() * per_sm;
    p->grid = want < most ? want : most;
    return true;
}

template <void (*KERN)(const NormArgs)>
static r3_status launch_norm_kernel(const NormArgs& a, const NormPlan& p, cudaStream_t cs) {
    static PerDevice ready;
    if (p.smem > 40 * 1024 && !ready.done()) {
        if (cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kNormRingBytes) != cudaSuccess)
            return R3_ERR_CUDA;
        ready.mark();
    }
    KERN<<<p.grid, p.threads, p.smem, cs>>>(a);
    return launch_status();
}
template <typename T, typename W, int P, bool WARP, int S>
static r3_status launch_norm(const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs) {
    return bwd ? launch_norm_kernel<norm_bwd_kernel<T, W, P, WARP, S>>(a, p, cs)
               : launch_norm_kernel<norm_fwd_kernel<T, W, P, WARP, S>>(a, p, cs);
}
template <typename T, typename W>
static r3_status launch_norm_pieces(const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs) {
    if (p.warp) return launch_norm<T, W, kWarpPieces, true, 3>(a, p, bwd, cs);
    if (p.pieces == 1) return launch_norm<T, W, 1, false, 3>(a, p, bwd, cs);
    if (p.pieces == 2) return launch_norm<T, W, 2, false, 3>(a, p, bwd, cs);
    return launch_norm<T, W, 4, false, 1>(a, p, bwd, cs);
}
static r3_status launch_norm_types(const r3_norm* s, const NormArgs& a, const NormPlan& p, bool bwd,
                                   cudaStream_t cs) {
    if (s->act_dtype == R3_BF16)
        return s->w_dtype == R3_BF16
                   ? launch_norm_pieces<__nv_bfloat16, __nv_bfloat16>(a, p, bwd, cs)
                   : launch_norm_pieces<__nv_bfloat16, float>(a, p, bwd, cs);
    return s->w_dtype == R3_BF16 ? launch_norm_pieces<float, __nv_bfloat16>(a, p, bwd, cs)
                                 : launch_norm_pieces<float, float>(a, p, bwd, cs);
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
    return r3::round_up((size_t)3 * plan.grid * shape->d * sizeof(float), 256);
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
        sum.d = shape->d;
        r3::norm_sum_kernel<<<dim3((shape->d + 31) / 32, 3), 256, 0, cs>>>(sum);
    }
    return r3::launch_status();
}
