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
// reductions.  A row belongs to a group of threads: one warp for up to 64 pieces of 16 bytes (no
// barrier then), else a CTA.  A thread owns two pieces of the row (four in the longest rows) and
// walks over the rows with a stride; one piece a thread left the kernels bound by instruction
// issue, because the reductions and addresses of a row cost a thread the same whatever it holds.
// The columns' weights and the sums of the weight gradients stay in its registers.  What hides the
// memory latency is a ring in shared memory that is private to the thread: it copies its own pieces
// of the rows to come there (cp.async), S rows ahead, so no barrier or wait between threads belongs
// to the copies (65536 x 2048 bf16: forward 176 us = 93% of the measured copy bandwidth, backward 258 to
// 274 us by GPU = 95 to 90%; 16384 x 2048: 50 and 76 us, of which the second
// kernel, which adds up the CTAs' sums of the weight gradients, takes 5; backward 8192 x 4096, two rows at a
// time, 83 us of 62; 4096 x 8192 and 2048 x 16384, the wide form, 106 and 180 of 62: it lacks registers).  A
// warp's pieces are neighbours
// (piece p of lane l is piece 32 p + l of the warp's share), so that all of a thread's addresses of a row
// are one base and constant offsets.
#pragma once

#include <type_traits>

#include "r3_common.cuh"
#include "r3_internal.h"
#include "r3_tc.cuh"

namespace r3 {

constexpr int kNormMaxThreads = 512;   // per row
constexpr int kNormBwdThreads = 384;   // backward: per SM, at up to 168 registers a thread
constexpr int kNormBwdThreadsF32 = 512;   // ... float32 rows (half the columns), at up to 128
constexpr int kNormPairThreads = 256;  // ... two rows at a time, at up to 255
constexpr int kNormFwdThreads = 640;   // forward: per SM, at up to 102
constexpr int kNormPieces = 2;         // pieces per thread; twice as many where these do not reach
constexpr int kWarpRows = 4;           // forward, one-warp form: rows per CTA

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
    float* part;            // backward: [2][grid][d] sums over a CTA's rows of dh x r and of g n
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

// The values of a 16-byte piece as float32.
__device__ __forceinline__ void widen(const Vec16<float>& v, float* f) { v.unpack(f); }
__device__ __forceinline__ void widen(const Vec16<__nv_bfloat16>& v, float* f) {
    const uint32_t w[4] = {v.v.x, v.v.y, v.v.z, v.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = bf16_pair(w[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
}

// Sum of NV values over the threads of a row; every thread gets the result.  One barrier per call: the
// caller alternates buffers, so that a buffer is only written again behind the barrier of the call in
// between.  The wide form's up to 16 warps are added as a tree over the lanes (a loop costs a thread three
// times the instructions: 4096 x 8192 bf16 backward 133 against 106 us), fewer one after the other (the
// tree beside the loop costs registers: 65536 x 2048 bf16 backward 267 against 258 us).
template <int NV, bool WARP, bool WIDE, int M>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*red)[M], int warps) {
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
    if (WIDE) {                                     // up to 16 warps: a tree over the lanes
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = lane < warps ? red[lane & 15][i] : 0.f;
#pragma unroll
        for (int s = 8; s > 0; s >>= 1) {
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], s);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = __shfl_sync(0xffffffffu, v[i], 0);
        return;
    }
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
            widen(v, t);
#pragma unroll
            for (int k = 0; k < M; ++k) f[(i + k) % N] = t[k];
        }
    } else {                                       // 4 f32 columns of a bf16 vector: 8 bytes
        const uint2 v = *reinterpret_cast<const uint2*>(w);
        const float2 lo = bf16_pair(v.x), hi = bf16_pair(v.y);
        f[0] = lo.x; f[1] = lo.y; f[2] = hi.x; f[3] = hi.y;
    }
}
template <typename T> __device__ __forceinline__ void store_piece(T* p, const float* f) {
    Vec16<T> o;
    o.pack(f);
    *reinterpret_cast<Vec16<T>*>(p) = o;
}

// What a call has, as far as a kernel of its own knows it: y, the norms, (backward) a gradient from above,
// a gate per token or per element.  What it lacks costs no instructions and no registers there (32714 x 2048
// bf16 backward without w_pre: 150 -> 98 us, without w_post: 164 -> 148, with a gate per element: 270 ->
// 190).  In the open form all but a gate per element is decided at run time; the forward kernel, which has
// registers left, knows the most usual calls only.
enum { kHasY = 1, kHasPost = 2, kHasPre = 4, kHasUp = 8, kTokenGate = 16, kFullGate = 32, kOpen = 64 };

// The weights of a thread's columns: with KEEP in registers for all its rows, else (the wide form's longer
// rows, which have no room) read again from L1 for each.  A column's factor is the vector's element
// (1 without a vector) times `times` (likewise) times `scale`.
template <typename W, int N, int P, bool KEEP> struct Weights {
    float w[KEEP ? P : 1][KEEP ? N : 1];
    const void *src, *times;
    float scale;
    __device__ __forceinline__ void read(int col, float* f) const {
        float b[N];
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = b[i] = 1.f;
        if (src) load_cols<W, N>(src, col, f);
        if (times) load_cols<W, N>(times, col, b);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] *= b[i] * scale;
    }
    __device__ __forceinline__ void init(const void* s, const void* t, float k, int col, const bool (&in)[P]) {
        src = s;
        times = t;
        scale = k;
        if constexpr (KEEP) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (in[p]) read(col + p * 32 * N, w[p]);
            }
        }
    }
    __device__ __forceinline__ void get(int p, int col, float* f) const {
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = w[p][i];
        } else {
            read(col + p * 32 * N, f);
        }
    }
};

// A thread's place: its first column (the further pieces follow at 32 N columns' distance), its rows,
// and its ring: stage s, array q, lane at ((s Q + q) 32 + lane) of the warp's part.
struct NormPlace {
    int lane, warps, col, row, stride;
    uint4* ring;
};
template <int N, int P, bool WARP, int Q, int S>
__device__ __forceinline__ NormPlace norm_place(uint4* ring) {
    NormPlace t;
    const int warp = threadIdx.x >> 5;
    t.lane = threadIdx.x & 31;
    t.warps = blockDim.x >> 5;
    t.col = ((WARP ? 0 : warp * 32 * P) + t.lane) * N;
    t.row = blockIdx.x + (WARP ? gridDim.x * warp : 0);        // few rows: spread over the SMs
    t.stride = gridDim.x * (WARP ? t.warps : 1);
    t.ring = ring + warp * (S * Q * 32) + t.lane;
    return t;
}

// A row's gate per element, loaded a row ahead.
template <typename T, int P, int FORM> struct RowGate {
    Vec16<T> full[FORM & kFullGate ? P : 1];
    __device__ __forceinline__ void load(const NormArgs& a, int row, int col, const bool (&in)[P]) {
        if constexpr ((FORM & kFullGate) != 0) {
            constexpr int HOP = 32 * Vec16<T>::N;
            if (row >= a.T) return;
            const T* g = static_cast<const T*>(a.gate) + (size_t)row * a.d + col;
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (in[p]) full[p] = *reinterpret_cast<const Vec16<T>*>(g + p * HOP);
        }
    }
};
// The gates of a group's tokens: lane l holds that of the l-th of its next 32 rows, and the 32 behind them
// are on their way.
struct TokenGates {
    const float* gate;
    long long row, step;                            // the lane's row among the 32 after `next`
    float mine, next;
    int rows, at;
    __device__ __forceinline__ float fetch() {
        const float g = row < rows ? gate[row] : 1.f;
        row += step;
        return g;
    }
    __device__ __forceinline__ void init(const NormArgs& a, const NormPlace& me) {
        gate = static_cast<const float*>(a.gate);
        rows = a.T;
        row = me.row + (long long)me.lane * me.stride;
        step = 32LL * me.stride;
        at = 0;
        mine = fetch();
        next = fetch();
    }
    __device__ __forceinline__ float take() {
        const float g = __shfl_sync(0xffffffffu, mine, at);
        if (++at == 32) {
            at = 0;
            mine = next;
            next = fetch();
        }
        return g;
    }
};

template <typename T, typename W, int P, bool WARP, bool WIDE, int S, int FORM>
__global__ void __launch_bounds__(WARP ? 32 * kWarpRows : kNormMaxThreads)
norm_fwd_kernel(const NormArgs a) {
    constexpr int N = Vec16<T>::N, Q = 2 * P, HOP = 32 * N;
    // the wide form has registers enough for 16 columns (8178 x 8192 bf16: 165 -> 84 us)
    constexpr bool KEEP = P * N <= 16;
    typedef const Vec16<T>* Ptr;
    extern __shared__ uint4 ring_all[];
    __shared__ float s_red[2][kNormMaxThreads / 32][4];   // up to three values per warp of the CTA
    constexpr bool OPEN = (FORM & kOpen) != 0, full = (FORM & kFullGate) != 0;
    const bool has_y = OPEN ? a.y != nullptr : (FORM & kHasY) != 0;
    const bool has_post = OPEN ? a.w_post != nullptr : (FORM & kHasPost) != 0;
    const bool has_pre = OPEN ? a.w_pre != nullptr : (FORM & kHasPre) != 0;
    const bool token = OPEN && !full ? a.gate_kind == R3_GATE_TOKEN : (FORM & kTokenGate) != 0;
    const NormPlace me = norm_place<N, P, WARP, Q, S>(ring_all);
    const float inv_d = 1.f / (float)a.d, eps = a.eps, res = a.res;
    const size_t start = (size_t)me.row * a.d + me.col, step = (size_t)me.stride * a.d;
    bool in[P];
#pragma unroll
    for (int p = 0; p < P; ++p) in[p] = me.col + p * HOP < a.d;
    // the ring's next row, and where it comes from
    const T* fx = static_cast<const T*>(a.x) + start;
    const T* fy = static_cast<const T*>(a.y) + start;
    int frow = me.row;
    auto fetch = [&](uint4* to) {
        if (frow < a.T) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (!in[p]) continue;
                copy_ahead(to + (2 * p) * 32, fx + p * HOP);
                if (has_y) copy_ahead(to + (2 * p + 1) * 32, fy + p * HOP);
            }
        }
        copy_commit();                             // one group per row, empty ones behind the last
        frow += me.stride;
        fx += step;
        fy += step;
    };
#pragma unroll
    for (int s = 0; s < S; ++s) fetch(me.ring + s * Q * 32);
    Weights<W, N, P, KEEP> post, pre;
    const void* channel =
        !(FORM & (kTokenGate | kFullGate)) && a.gate_kind == R3_GATE_CHANNEL ? a.gate : nullptr;
    if (has_y) post.init(a.w_post, channel, a.branch, me.col, in);
    if (has_pre) pre.init(a.w_pre, nullptr, 1.f, me.col, in);
    RowGate<T, P, FORM> gate, ahead;
    ahead.load(a, me.row, me.col, in);
    TokenGates gates;
    if (token) gates.init(a, me);
    T* x_out = static_cast<T*>(a.out0) + start;
    T* h_out = static_cast<T*>(a.out1) + start;
    int stage = 0;
    for (int row = me.row; row < a.T; row += me.stride, x_out += step, h_out += step) {
        uint4* slot = me.ring + stage * Q * 32;
        copy_wait<S - 1>();
        float x[P][N];
        Vec16<T> yv[P];
        float s[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[p][i] = 0.f;
            if (!in[p]) continue;
            widen(*reinterpret_cast<Ptr>(slot + (2 * p) * 32), x[p]);
            if (!has_y) continue;
            yv[p] = *reinterpret_cast<Ptr>(slot + (2 * p + 1) * 32);
            float y[N];
            widen(yv[p], y);
#pragma unroll
            for (int i = 0; i < N; ++i) s[0] = fmaf(y[i], y[i], s[0]);
        }
        fetch(slot);
        stage = stage + 1 == S ? 0 : stage + 1;
        gate = ahead;
        ahead.load(a, row + me.stride, me.col, in);
        float r = 1.f;
        if (has_post) {
            row_sum<1, WARP, WIDE>(s, s_red[0], me.warps);
            r = rsqrtf(s[0] * inv_d + eps);
        }
        if (has_y) {
            if (token) r *= gates.take();
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (!in[p]) continue;
                float w[N], y[N];
                post.get(p, me.col, w);
                widen(yv[p], y);
                if (full) {
                    float g[N];
                    widen(gate.full[full ? p : 0], g);
#pragma unroll
                    for (int i = 0; i < N; ++i) y[i] *= g[i];
                }
#pragma unroll
                for (int i = 0; i < N; ++i) x[p][i] = fmaf(y[i] * r, w[i], res * x[p][i]);
                store_piece<T>(x_out + p * HOP, x[p]);
            }
        }
        if (has_pre) {
            s[0] = 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < N; ++i) s[0] = fmaf(x[p][i], x[p][i], s[0]);
            row_sum<1, WARP, WIDE>(s, s_red[1], me.warps);
            r = rsqrtf(s[0] * inv_d + eps);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (!in[p]) continue;
                float w[N];
                pre.get(p, me.col, w);
#pragma unroll
                for (int i = 0; i < N; ++i) w[i] *= x[p][i] * r;
                store_piece<T>(h_out + p * HOP, w);
            }
        }
        // with one reduction per row its buffer comes around without a barrier in between
        if (!WARP && (!has_post || !has_pre)) __syncthreads();
    }
    copy_wait<0>();
}

// Threads per SM that the backward kernel is compiled for.  (An SM's registers are four files of 16384:
// 15 warps at 134 registers do not fit although 15 x 32 x 134 < 65536.)
__host__ __device__ constexpr int norm_bwd_threads(bool wide, bool f32, bool full, int rows) {
    return rows > 1       ? kNormPairThreads
           : wide         ? kNormMaxThreads
           : f32 && !full ? kNormBwdThreadsF32
                          : kNormBwdThreads;
}

// Backward.  With x = x_out, r = rsqrt(mean(x^2) + eps), u = dh w_pre and c = mean(u x) r:
//   g  = dx_out + r u - x r^2 c;      dw_pre += dh x r;      dx = residual_scale g
// and with n = y s (s = rsqrt(mean(y^2) + eps)), v = branch_scale gate w_post g, e = mean(v n):
//   dy = s (v - n e)
// dw_post and the gate's gradient both come from g n: per column, where the gate is one factor per
// column (or there is none), A = sum g n gives dw_post = branch_scale gate A and dgate =
// branch_scale w_post A; a token's gate is taken out of v, so that its gradient is the sum that e
// is formed from.  A row takes two reductions, of three values and of one.  A group of threads works on R
// rows at a time.
template <typename T, typename W, int P, bool WARP, bool WIDE, int S, int R, int FORM>
__global__ void __launch_bounds__(norm_bwd_threads(WIDE, sizeof(T) == 4, (FORM & kFullGate) != 0, R))
norm_bwd_kernel(const NormArgs a) {
    constexpr int N = Vec16<T>::N, Q = 4 * P * R, HOP = 32 * N;
    // the wide form has registers for the weights of 8 columns, of 16 where there is one vector of them (8178
    // x 4096 float32: 180 -> 148 us; 8178 x 8192 bf16 without w_pre 140 -> 94, without y 116 -> 81)
    constexpr bool ONE = !(FORM & kOpen) && (!(FORM & kHasPre) || !(FORM & kHasY));
    constexpr bool KEEP = !WIDE || P * N <= (ONE ? 16 : 8);
    typedef const Vec16<T>* Ptr;
    extern __shared__ uint4 ring_all[];
    __shared__ float s_red[2][kNormMaxThreads / 32][3 * R + R % 2];   // up to 3 R values per warp of the CTA
    constexpr bool OPEN = (FORM & kOpen) != 0, full = (FORM & kFullGate) != 0;
    const bool has_y = OPEN ? a.y != nullptr : (FORM & kHasY) != 0;
    const bool has_post = OPEN ? a.w_post != nullptr : (FORM & kHasPost) != 0;
    const bool has_pre = OPEN ? a.w_pre != nullptr : (FORM & kHasPre) != 0;
    const bool has_up = OPEN ? a.dx_out != nullptr : (FORM & kHasUp) != 0;
    const bool token = OPEN && !full ? a.gate_kind == R3_GATE_TOKEN : (FORM & kTokenGate) != 0;
    const NormPlace me = norm_place<N, P, WARP, Q, S>(ring_all);
    const float inv_d = 1.f / (float)a.d, eps = a.eps, res = has_y ? a.res : 1.f;
    const size_t start = (size_t)me.row * a.d + me.col, step = (size_t)me.stride * a.d;
    bool in[P];
#pragma unroll
    for (int p = 0; p < P; ++p) in[p] = me.col + p * HOP < a.d;
    const T* fx = static_cast<const T*>(a.x) + start;
    const T* fh = static_cast<const T*>(a.dh) + start;
    const T* fg = static_cast<const T*>(a.dx_out) + start;
    const T* fy = static_cast<const T*>(a.y) + start;
    int frow = me.row;
    auto fetch = [&](uint4* to) {
#pragma unroll
        for (int r = 0; r < R; ++r, to += 4 * P * 32) {
            if (frow < a.T) {
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if (!in[p]) continue;
                    if (has_pre) {
                        copy_ahead(to + (4 * p) * 32, fx + p * HOP);
                        copy_ahead(to + (4 * p + 1) * 32, fh + p * HOP);
                    }
                    if (has_up) copy_ahead(to + (4 * p + 2) * 32, fg + p * HOP);
                    if (has_y) copy_ahead(to + (4 * p + 3) * 32, fy + p * HOP);
                }
            }
            frow += me.stride;
            fx += step;
            fh += step;
            fg += step;
            fy += step;
        }
        copy_commit();
    };
#pragma unroll
    for (int s = 0; s < S; ++s) fetch(me.ring + s * Q * 32);
    const void* channel =
        !(FORM & (kTokenGate | kFullGate)) && a.gate_kind == R3_GATE_CHANNEL ? a.gate : nullptr;
    Weights<W, N, P, KEEP> post, pre;
    if (has_y) post.init(a.w_post, channel, a.branch, me.col, in);
    if (has_pre) pre.init(a.w_pre, nullptr, 1.f, me.col, in);
    float acc_pre[P][N], acc_post[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < N; ++i) acc_pre[p][i] = acc_post[p][i] = 0.f;
    RowGate<T, P, FORM> row_gate[R], ahead[R];
#pragma unroll
    for (int r = 0; r < R; ++r) ahead[r].load(a, me.row + r * me.stride, me.col, in);
    TokenGates gates;
    if (token) gates.init(a, me);
    T* dx = static_cast<T*>(a.out0) + start;
    T* dy = static_cast<T*>(a.out1) + start;
    int stage = 0;
    for (int row = me.row; row < a.T; row += R * me.stride, dx += R * step, dy += R * step) {
        uint4* slot = me.ring + stage * Q * 32;
        copy_wait<S - 1>();
        Vec16<T> xv[R][P], hv[R][P], yv[R][P], gv[R][P];
        float s[3 * R];
        bool live[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            live[r] = r == 0 || row + r * me.stride < a.T;
            s[3 * r] = s[3 * r + 1] = s[3 * r + 2] = 0.f;
            if (!live[r]) continue;
            const uint4* from = slot + 4 * P * 32 * r;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (!in[p]) continue;
                float f[N];
                if (has_pre) {
                    float h[N], w[N];
                    xv[r][p] = *reinterpret_cast<Ptr>(from + (4 * p) * 32);
                    hv[r][p] = *reinterpret_cast<Ptr>(from + (4 * p + 1) * 32);
                    pre.get(p, me.col, w);
                    widen(xv[r][p], f);
                    widen(hv[r][p], h);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        s[3 * r] = fmaf(f[i], f[i], s[3 * r]);
                        s[3 * r + 1] = fmaf(h[i] * w[i], f[i], s[3 * r + 1]);
                    }
                }
                if (has_up) gv[r][p] = *reinterpret_cast<Ptr>(from + (4 * p + 2) * 32);
                if (has_y) {
                    yv[r][p] = *reinterpret_cast<Ptr>(from + (4 * p + 3) * 32);
                    widen(yv[r][p], f);
#pragma unroll
                    for (int i = 0; i < N; ++i) s[3 * r + 2] = fmaf(f[i], f[i], s[3 * r + 2]);
                }
            }
        }
        fetch(slot);
        stage = stage + 1 == S ? 0 : stage + 1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            row_gate[r] = ahead[r];
            ahead[r].load(a, row + (R + r) * me.stride, me.col, in);
        }
        if (has_pre || has_post) row_sum<3 * R, WARP, WIDE>(s, s_red[0], me.warps);
        // wide rows: n is formed again, no room
        float v[R][P][N], n[R][WIDE ? 1 : P][N], z[R], sy[R], gate_t[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            z[r] = 0.f;
            const float rx = rsqrtf(s[3 * r] * inv_d + eps);
            const float rrc = s[3 * r + 1] * inv_d * rx * rx * rx;      // r^2 c
            sy[r] = has_post ? rsqrtf(s[3 * r + 2] * inv_d + eps) : 1.f;
            gate_t[r] = token ? gates.take() : 1.f;
            if (!live[r]) continue;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (!in[p]) continue;
                float f[N], g[N];
#pragma unroll
                for (int i = 0; i < N; ++i) g[i] = 0.f;
                if (has_up) widen(gv[r][p], g);
                if (has_pre) {
                    float h[N], w[N];
                    pre.get(p, me.col, w);
                    widen(xv[r][p], f);
                    widen(hv[r][p], h);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        acc_pre[p][i] = fmaf(h[i] * f[i], rx, acc_pre[p][i]);
                        g[i] = fmaf(h[i] * w[i], rx, g[i]);
                        g[i] = fmaf(f[i], -rrc, g[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < N; ++i) f[i] = res * g[i];
                store_piece<T>(dx + r * step + p * HOP, f);
                if (!has_y) continue;
                float w[N];
                post.get(p, me.col, w);
                float(&np)[N] = n[r][WIDE ? 0 : p];
                widen(yv[r][p], np);
#pragma unroll
                for (int i = 0; i < N; ++i) np[i] *= sy[r];
                if (full) {
                    float gate[N], dg[N];
                    widen(row_gate[r].full[full ? p : 0], gate);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        dg[i] = g[i] * w[i] * np[i];
                        g[i] *= gate[i];
                    }
                    T* to = static_cast<T*>(a.dgate) + (size_t)(row + r * me.stride) * a.d;
                    store_piece<T>(to + me.col + p * HOP, dg);
                }
                if (token) {
#pragma unroll
                    for (int i = 0; i < N; ++i) acc_post[p][i] = fmaf(gate_t[r] * g[i], np[i], acc_post[p][i]);
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) acc_post[p][i] = fmaf(g[i], np[i], acc_post[p][i]);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    v[r][p][i] = g[i] * w[i];
                    z[r] = fmaf(v[r][p][i], np[i], z[r]);
                }
            }
        }
        if (has_y) {
            if (has_post || token) row_sum<R, WARP, WIDE>(z, s_red[1], me.warps);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (!live[r]) continue;
                const float k = gate_t[r] * sy[r];
                const float e = has_post ? -z[r] * inv_d : 0.f;
                if (token && me.col == 0)
                    static_cast<float*>(a.dgate)[row + r * me.stride] = z[r];
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if (!in[p]) continue;
                    float(&np)[N] = n[r][WIDE ? 0 : p];
                    if (WIDE) {
                        widen(yv[r][p], np);
#pragma unroll
                        for (int i = 0; i < N; ++i) np[i] *= sy[r];
                    }
#pragma unroll
                    for (int i = 0; i < N; ++i) v[r][p][i] = k * fmaf(np[i], e, v[r][p][i]);
                    store_piece<T>(dy + r * step + p * HOP, v[r][p]);
                }
            }
        }
        // with one reduction per row its buffer comes around without a barrier in between
        if (!WARP && (has_pre || has_post) != (has_y && (has_post || token))) __syncthreads();
    }
    copy_wait<0>();
    if (!a.part) return;
    // the kernel that adds up the CTAs' sums may be set up meanwhile
    tc::grid_launch_dependents();
    // One row of partial sums per CTA.  In the one-warp form the warps' are added up in order first.
    const size_t plane = (size_t)gridDim.x * a.d;
    float* mine = a.part + (size_t)blockIdx.x * a.d + me.col;
    float* sums = reinterpret_cast<float*>(ring_all);           // [P N][threads], the ring is idle
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (!(k == 0 ? has_pre : has_post || channel != nullptr)) continue;
        float(&acc)[P][N] = k == 0 ? acc_pre : acc_post;
        if (WARP) {
            __syncthreads();
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < N; ++i) sums[(p * N + i) * blockDim.x + threadIdx.x] = acc[p][i];
            __syncthreads();
            if (threadIdx.x >= 32) continue;
            for (int g = 1; g < me.warps; ++g)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        acc[p][i] += sums[(p * N + i) * blockDim.x + 32 * g + threadIdx.x];
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (!in[p]) continue;
#pragma unroll
            for (int i = 0; i < N; i += 4)
                *reinterpret_cast<float4*>(mine + k * plane + p * HOP + i) =
                    make_float4(acc[p][i], acc[p][i + 1], acc[p][i + 2], acc[p][i + 3]);
        }
    }
}

// ---- launch ---------------------------------------------------------------------------------------
constexpr int kNormRingBytes = 200 * 1024;   // of an SM's shared memory, for the rings of its CTAs
// Rows in a thread's ring.  Three fit everywhere but in the backward of the longest rows, where 288 threads or
// more with four pieces of four arrays each need 72 KB and more for one.
__host__ __device__ constexpr int norm_stages(int pieces, bool bwd) { return bwd && pieces > kNormPieces ? 1 : 3; }
__host__ __device__ constexpr int norm_ring_bytes(int pieces, bool bwd, int threads) {      // one row's
    return (bwd ? 4 : 2) * pieces * threads * 16;
}
static_assert(3 * norm_ring_bytes(2 * kNormPieces, false, kNormMaxThreads) <= kNormRingBytes, "");
static_assert(3 * norm_ring_bytes(kNormPieces, true, kNormMaxThreads) <= kNormRingBytes, "");
static_assert(3 * norm_ring_bytes(kNormPieces, true, 2 * kNormPairThreads) <= kNormRingBytes, "");
static_assert(norm_ring_bytes(2 * kNormPieces, true, kNormMaxThreads) <= kNormRingBytes, "");

struct NormPlan {
    int pieces, threads, grid;
    bool warp, wide, pair;
    size_t smem;
};

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
template <typename T, typename W, int P, bool WARP, bool WIDE, int R>
static r3_status launch_norm(const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs) {
    const bool full = a.gate_kind == R3_GATE_FULL, token = a.gate_kind == R3_GATE_TOKEN;
    if constexpr (R == 1) {
        if (!bwd) {
            auto run = [&](auto form) {
                constexpr int F = decltype(form)::value;
                return launch_norm_kernel<norm_fwd_kernel<T, W, P, WARP, WIDE, norm_stages(P, false), F>>(a, p, cs);
            };
            constexpr int BOTH = kHasY | kHasPost | kHasPre;
            if (!a.y) return run(std::integral_constant<int, kHasPre>());
            if (full) return run(std::integral_constant<int, kOpen | kFullGate>());
            if (!a.w_post || !a.w_pre) return run(std::integral_constant<int, kOpen>());
            return token ? run(std::integral_constant<int, BOTH | kTokenGate>())
                         : run(std::integral_constant<int, BOTH>());
        }
    }
    auto run = [&](auto form) {
        constexpr int F = decltype(form)::value;
        return launch_norm_kernel<norm_bwd_kernel<T, W, P, WARP, WIDE, norm_stages(P, true), R, F>>(a, p, cs);
    };
    auto gated = [&](auto form) {
        constexpr int F = decltype(form)::value | kHasY | kHasUp;
        return full    ? run(std::integral_constant<int, F | kFullGate>())
               : token ? run(std::integral_constant<int, F | kTokenGate>())
                       : run(std::integral_constant<int, F>());
    };
    if (!a.y)
        return a.dx_out ? run(std::integral_constant<int, kHasPre | kHasUp>())
                        : run(std::integral_constant<int, kHasPre>());
    if (a.dx_out && a.w_post && a.w_pre) return gated(std::integral_constant<int, kHasPost | kHasPre>());
    if (a.dx_out && a.w_post) return gated(std::integral_constant<int, kHasPost>());
    if (a.dx_out && a.w_pre) return gated(std::integral_constant<int, kHasPre>());
    return full ? run(std::integral_constant<int, kOpen | kFullGate>())
                : run(std::integral_constant<int, kOpen>());
}
template <typename T, typename W>
static r3_status launch_norm_size(const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs) {
    constexpr int P = kNormPieces;
    if (p.warp) return launch_norm<T, W, P, true, false, 1>(a, p, bwd, cs);
    if (!p.wide)
        return p.pair ? launch_norm<T, W, P, false, false, 2>(a, p, bwd, cs)
                      : launch_norm<T, W, P, false, false, 1>(a, p, bwd, cs);
    return p.pieces == P ? launch_norm<T, W, P, false, true, 1>(a, p, bwd, cs)
                         : launch_norm<T, W, 2 * P, false, true, 1>(a, p, bwd, cs);
}

// By the rows' type, in a file each (they compile side by side).
r3_status launch_norm_bf16(bool w_bf16, const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs);
r3_status launch_norm_f32(bool w_bf16, const NormArgs& a, const NormPlan& p, bool bwd, cudaStream_t cs);

}  // namespace r3
