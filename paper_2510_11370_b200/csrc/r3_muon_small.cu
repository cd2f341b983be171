// The orthogonalised update of matrices whose smaller side is at most 128, in one launch: gradient and
// momentum are read, the whole iteration runs on the chip, the weights are written.  (r3_muon.cu holds the
// method, its numbers and the form for larger matrices, whose iterates go through memory between products.)
//
// With m <= 128 the smaller side, X [m, n] lies across the CTAs of a cluster, up to 256 columns each, as two fp16
// planes in shared memory.  The same tiles (64 columns to a 128-byte row, swizzled) are the K-major operands of
// X X^T and the MN-major operand of B X, so nothing is ever laid out again, and every product's epilogue
// replaces its operand in place.  A is m x m: with more than one CTA the parts X_s X_s^T are added up through
// distributed shared memory, each CTA a share of A's columns, which it then hands to all; b A + c A^2 is small
// and every CTA forms it for itself.  Bound by latency: fifteen products with their barriers one after
// the other.
#include "r3_muon.cuh"

namespace r3 {
namespace ns {

constexpr int SM_THREADS = 256;
constexpr int SM_BLOCK = 128 * 128;           // bytes of 128 rows x 64 columns of fp16
constexpr int SM_MISC = 512;

__device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void fence_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ void store_remote(uint32_t at, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};"
                 ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void store_remote(uint32_t at, uint2 v) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(v.x), "r"(v.y) : "memory");
}
__device__ __forceinline__ void store_remote(uint32_t at, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(v) : "memory");
}
// Byte of element (row, column) within a plane; the eight columns from a multiple of 8 on are 16 bytes.
__device__ __forceinline__ uint32_t tile_at(int row, int col) {
    return (uint32_t)((col >> 6) * SM_BLOCK + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4) + (col & 7) * 2);
}
__device__ __forceinline__ void split8(const float (&x)[8], uint4* hi, uint4* lo) {
    __half2* h = reinterpret_cast<__half2*>(hi);
    __half2* l = reinterpret_cast<__half2*>(lo);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
        const float2 f = __half22float2(h[i]);
        l[i] = __floats2half2_rn(x[2 * i] - f.x, x[2 * i + 1] - f.y);
    }
}
__device__ __forceinline__ void add8(const uint4& v, float (&x)[8]) {
    const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(h[i]);
        x[2 * i] += f.x;
        x[2 * i + 1] += f.y;
    }
}

// Eight elements, `step` apart, of which `valid` exist (the others read as 0); together where `wide`.
template <typename T>
__device__ __forceinline__ void get8(const T* p, bool wide, long long step, int valid, float (&f)[8]) {
    if (wide) {
        load8(p, f);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = k < valid ? to_f32(p[k * step]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void put8(T* p, bool wide, long long step, int valid, const float (&f)[8]) {
    if (wide) {
        store8(p, f);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < valid) p[k * step] = from_f32<T>(f[k]);
    }
}
__device__ __forceinline__ void get8(const void* p, int dtype, long long at, bool wide, long long step, int valid,
                                     float (&f)[8]) {
    if (dtype == R3_BF16) get8(static_cast<const __nv_bfloat16*>(p) + at, wide, step, valid, f);
    else get8(static_cast<const float*>(p) + at, wide, step, valid, f);
}

template <int TERMS>
__global__ void __launch_bounds__(SM_THREADS, 2) small_kernel(const __grid_constant__ SmallArgs a) {
    constexpr int PL = TERMS > 1 ? 2 : 1;                // planes of A and B
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* bp = smem_raw + (base - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int C = a.cluster;
    const uint32_t rank = C > 1 ? cluster_ctarank() : 0;
    const uint32_t x_plane = (uint32_t)a.x_blocks * SM_BLOCK, a_plane = (uint32_t)a.a_blocks * SM_BLOCK;
    const uint32_t a0 = 2 * x_plane;                     // the A region, behind X's two planes
    uint8_t* misc = bp + a0 + a.a_bytes;
    const uint32_t bar = base + a0 + a.a_bytes;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc + 16);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 20);
    double* s_sum = reinterpret_cast<double*>(misc + 64);           // [8] warps
    double* s_norm = reinterpret_cast<double*>(misc + 128);         // [16] CTAs
    const uint32_t norm_at = base + a0 + a.a_bytes + 128;

    const int matrix = blockIdx.x / C;
    int z = matrix, si = 0;
    for (int step = MAX_STACKS / 2; step > 0; step >>= 1)
        if (si + step < a.stacks && a.stack[si + step].first <= matrix) si += step;
    const SmallStack& st = a.stack[si];
    z -= st.first;
    const bool tall = st.rows > st.cols;
    const int m = min(st.rows, st.cols), n = max(st.rows, st.cols);
    const int m16 = (m + 15) & ~15;
    const int W = ((n + C - 1) / C + 15) & ~15;          // columns of X in this CTA, those that exist
    const int j0 = (int)rank * W, jn = max(0, min(W, n - j0));
    const int octets = W >> 3;

    if (threadIdx.x == 0) {
        mbar_init(bar, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), a.tmem_cols);
    tc_fence_before();
    __syncthreads();
    if (C > 1) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_launch_dependents();
    grid_dependency_wait();

    float gs;
    const bool go = scale_of(a.grad_scale, &gs);         // the same in every CTA
    if (go) {
        // ---- u = the direction, its norm; the momentum's update ------------------------------------
        const long long size = (long long)st.rows * st.cols, at0 = (long long)z * size;
        const long long row = st.cols;                   // elements of a row in memory
        const bool wide = !tall && (st.cols & 7) == 0;
        float* mom = st.momentum ? st.momentum + at0 : nullptr;
        const long long hop = tall ? row : 1;            // between the elements of an octet of X's columns
        auto offset = [&](int i, int o) {
            return tall ? (long long)(j0 + 8 * o) * row + i : (long long)i * row + j0 + 8 * o;
        };
        double sum = 0.0;
        const int live = (jn + 7) >> 3;                  // octets with elements
        for (int u = threadIdx.x; u < m * live; u += SM_THREADS) {
            const int i = tall ? u % m : u / live, o = tall ? u / m : u % live;
            const int valid = min(8, jn - 8 * o);
            const long long at = offset(i, o);
            float g[8], v[8];
            get8(st.grad, a.grad_dtype, at0 + at, wide, hop, valid, g);
            if (mom) {
                get8(mom + at, wide, hop, valid, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __fadd_rn(__fmul_rn(a.momentum, v[k]), __fmul_rn(g[k], gs));
                put8(mom + at, wide, hop, valid, v);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double x = (double)direction(a.nesterov, a.momentum, mom != nullptr, __fmul_rn(g[k], gs), v[k]);
                sum += x * x;
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_sum[warp] = sum;
        __syncthreads();
        if (threadIdx.x < C) {
            sum = 0.0;
            for (int i = 0; i < SM_THREADS / 32; ++i) sum += s_sum[i];
            if (C > 1) store_remote(mapa_shared(norm_at + 8u * rank, threadIdx.x), sum);
            else s_norm[0] = sum;
        }
        if (C > 1) {
            __syncwarp();
            cluster_sync_all();
        } else {
            __syncthreads();
        }
        sum = 0.0;
        for (int i = 0; i < C; ++i) sum += s_norm[i];
        const float inv = start_scale(sum, a.eps);
        // ---- X = u / (|u| + eps) into the planes, zeros around it (its reads meet in L2) -----------
        for (int u = threadIdx.x; u < 128 * octets; u += SM_THREADS) {
            const int i = tall ? u & 127 : u / octets, o = tall ? u >> 7 : u % octets;
            const int valid = i < m ? min(8, jn - 8 * o) : 0;
            float g[8], v[8];
            if (valid > 0) {
                const long long at = offset(i, o);
                get8(st.grad, a.grad_dtype, at0 + at, wide, hop, valid, g);
                if (mom) get8(mom + at, wide, hop, valid, v);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    g[k] = k < valid ? direction(a.nesterov, a.momentum, mom != nullptr, __fmul_rn(g[k], gs), v[k]) * inv
                                     : 0.f;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) g[k] = 0.f;
            }
            uint4 hi, lo;
            split8(g, &hi, &lo);
            const uint32_t t = tile_at(i, 8 * o);
            *reinterpret_cast<uint4*>(bp + t) = hi;
            *reinterpret_cast<uint4*>(bp + x_plane + t) = lo;
        }
        fence_async();
        __syncthreads();

        // ---- the iteration ---------------------------------------------------------------------------
        const int q = warp & 3, half = warp >> 2, r = q * 32 + lane;      // this thread's row of every product
        const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16);
        uint32_t phase = 0;
        bool alive = true;
        // D = P Q over k16 steps of 16 along k; plane choice by term, small products first
        auto multiply = [&](uint32_t p0, uint32_t p_plane, uint32_t q0, uint32_t q_plane, bool q_mn, int N, int k16) {
            if (warp == 0) {
                tc_fence_after();
                if (alive && elect_one()) {
                    const uint32_t idesc = (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24) |
                                           (q_mn ? 1u << 16 : 0u);
                    for (int term = 0; term < TERMS; ++term) {
                        const uint32_t p = base + p0 + (TERMS > 1 && term == 1 ? p_plane : 0u);
                        const uint32_t qq = base + q0 + (TERMS > 1 && term == 0 ? q_plane : 0u);
                        for (int k = 0; k < k16; ++k) {
                            const uint32_t in_row = (uint32_t)((k >> 2) * SM_BLOCK + (k & 3) * 32);
                            const uint64_t dq = q_mn ? smem_desc_mn_sw128(qq + (uint32_t)k * 2048u, SM_BLOCK)
                                                     : smem_desc_sw128(qq + in_row);
                            tc_mma_bf16(tmem, smem_desc_sw128(p + in_row), dq, idesc, (term | k) != 0 ? 1u : 0u);
                        }
                    }
                    tc_commit(bar);
                }
                __syncwarp();
            }
            if (alive) {
                const bool ok = mbar_wait(bar, phase, abort_flag, a.dev_status);
                alive = __all_sync(0xffffffffu, ok);
            }
            phase ^= 1u;
            tc_fence_after();
        };
        // the next product may read what this one's epilogue wrote
        auto written = [&]() {
            fence_async();
            tc_fence_before();
            __syncthreads();
        };
        for (int s = 0; s < a.steps; ++s) {
            const float ca = a.coefs[s][0], cb = a.coefs[s][1], cc = a.coefs[s][2];
            // A = X X^T
            multiply(0, x_plane, 0, x_plane, false, m16, W >> 4);
            if (C == 1) {
#pragma unroll 1
                for (int c = half * 64; c < min(m16, half * 64 + 64); c += 32) {
                    if (!alive) break;
                    float v[32];
                    tc_ld32(trow + c, v);
                    tc_wait_ld();
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] = v[8 * j + k] * (1.f / SCALE);
                        uint4 hi, lo;
                        split8(x, &hi, &lo);
                        const uint32_t t = a0 + tile_at(r, c + 8 * j);
                        if (c + 8 * j < m16) {
                            *reinterpret_cast<uint4*>(bp + t) = hi;
                            if (PL > 1) *reinterpret_cast<uint4*>(bp + a_plane + t) = lo;
                        }
                    }
                }
                written();
            } else {
                // parts to the owners of their columns: [source][4 columns][row], in the A region, once every
                // CTA has its last product with B behind it
                if (s > 0) cluster_wait();
                const int share = 128 / C;               // columns per owner
#pragma unroll 1
                for (int c = half * 64; c < min(m16, half * 64 + 64); c += 32) {
                    if (!alive) break;
                    float v[32];
                    tc_ld32(trow + c, v);
                    tc_wait_ld();
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int col = c + 4 * j;
                        const uint32_t to = base + a0 + rank * (uint32_t)(128 * share * 4) +
                                            (uint32_t)((((col % share) >> 2) * 128 + r) * 16);
                        if (col < m16)
                            store_remote(mapa_shared(to, (uint32_t)(col / share)),
                                         make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
                    }
                }
                tc_fence_before();
                __syncwarp();
                cluster_sync_all();
                uint2 hi[8], lo[8];                      // 128 * share / 4 / 256 of them, 8 at most
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int u = threadIdx.x + e * SM_THREADS;
                    if (u >= 32 * share) break;
                    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
                    if ((int)rank * share + 4 * (u >> 7) < m16)
                        for (int src = 0; src < C; ++src) {
                            const float4 p = *reinterpret_cast<const float4*>(
                                bp + a0 + (uint32_t)src * (uint32_t)(128 * share * 4) + (uint32_t)u * 16u);
                            t.x += p.x;
                            t.y += p.y;
                            t.z += p.z;
                            t.w += p.w;
                        }
                    const __half2 h0 = __floats2half2_rn(t.x * (1.f / SCALE), t.y * (1.f / SCALE));
                    const __half2 h1 = __floats2half2_rn(t.z * (1.f / SCALE), t.w * (1.f / SCALE));
                    const float2 f0 = __half22float2(h0), f1 = __half22float2(h1);
                    const __half2 l0 = __floats2half2_rn(t.x * (1.f / SCALE) - f0.x, t.y * (1.f / SCALE) - f0.y);
                    const __half2 l1 = __floats2half2_rn(t.z * (1.f / SCALE) - f1.x, t.w * (1.f / SCALE) - f1.y);
                    hi[e] = make_uint2(*reinterpret_cast<const uint32_t*>(&h0), *reinterpret_cast<const uint32_t*>(&h1));
                    lo[e] = make_uint2(*reinterpret_cast<const uint32_t*>(&l0), *reinterpret_cast<const uint32_t*>(&l1));
                }
                __syncwarp();
                cluster_sync_all();                      // every CTA has read its parts: A may stand there now
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int u = threadIdx.x + e * SM_THREADS;
                    const int col = (int)rank * share + 4 * (u >> 7);
                    if (u >= 32 * share || col >= m16) break;          // (behind m16 the planes may end)
                    const uint32_t t = base + a0 + tile_at(u & 127, col);
                    for (int to = 0; to < C; ++to) {
                        store_remote(mapa_shared(t, (uint32_t)to), hi[e]);
                        if (PL > 1) store_remote(mapa_shared(t + a_plane, (uint32_t)to), lo[e]);
                    }
                }
                fence_async_all();
                __syncwarp();
                cluster_sync_all();
                fence_async_all();
                tc_fence_before();
                __syncthreads();
            }
            // B = b A + c A^2, in A's place
            multiply(a0, a_plane, a0, a_plane, false, m16, m16 >> 4);
#pragma unroll 1
            for (int c = half * 64; c < min(m16, half * 64 + 64); c += 32) {
                if (!alive) break;
                float v[32];
                tc_ld32(trow + c, v);
                tc_wait_ld();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c + 8 * j >= m16) break;
                    const uint32_t t = a0 + tile_at(r, c + 8 * j);
                    float x[8] = {};
                    add8(*reinterpret_cast<const uint4*>(bp + t), x);
                    if (PL > 1) add8(*reinterpret_cast<const uint4*>(bp + a_plane + t), x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = fmaf(cb, x[k], (cc / SCALE) * v[8 * j + k]);
                    uint4 hi, lo;
                    split8(x, &hi, &lo);
                    *reinterpret_cast<uint4*>(bp + t) = hi;
                    if (PL > 1) *reinterpret_cast<uint4*>(bp + a_plane + t) = lo;
                }
            }
            written();
            // X = a X + B X, in X's place
            multiply(a0, a_plane, 0, x_plane, true, W, m16 >> 4);
            if (C > 1 && s + 1 < a.steps) {
                __syncwarp();
                cluster_arrive();                        // B is read: the next parts may come
            }
#pragma unroll 1
            for (int c = half * 128; c < min(W, half * 128 + 128); c += 32) {
                if (!alive) break;
                float v[32];
                tc_ld32(trow + c, v);
                tc_wait_ld();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c + 8 * j >= W) break;
                    const uint32_t t = tile_at(r, c + 8 * j);
                    float x[8] = {};
                    add8(*reinterpret_cast<const uint4*>(bp + t), x);
                    add8(*reinterpret_cast<const uint4*>(bp + x_plane + t), x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = fmaf(ca, x[k], (1.f / SCALE) * v[8 * j + k]);
                    uint4 hi, lo;
                    split8(x, &hi, &lo);
                    *reinterpret_cast<uint4*>(bp + t) = hi;
                    *reinterpret_cast<uint4*>(bp + x_plane + t) = lo;
                }
            }
            written();
        }

        // ---- the result, or the weights' update -------------------------------------------------------
        const float lr = a.lr_now ? *a.lr_now : a.lr;
        const float keep = 1.f - lr * st.decay, rate = a.step ? lr * st.scale * (1.f / SCALE) : -(1.f / SCALE);
        float* master = st.master ? st.master + at0 : nullptr;
        for (int u = threadIdx.x; u < m * live; u += SM_THREADS) {
            const int i = tall ? u % m : u / live, o = tall ? u / m : u % live;
            const int valid = min(8, jn - 8 * o);
            const long long at = offset(i, o);
            const uint32_t t = tile_at(i, 8 * o);
            float x[8] = {}, w[8];
            add8(*reinterpret_cast<const uint4*>(bp + t), x);
            add8(*reinterpret_cast<const uint4*>(bp + x_plane + t), x);
            if (a.step) {
                if (master) get8(master + at, wide, hop, valid, w);
                else get8(st.param, a.param_dtype, at0 + at, wide, hop, valid, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = w[k] * keep - rate * x[k];
                if (master) put8(master + at, wide, hop, valid, w);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = -rate * x[k];
            }
            if (a.param_dtype == R3_BF16) put8(static_cast<__nv_bfloat16*>(st.param) + at0 + at, wide, hop, valid, w);
            else put8(static_cast<float*>(st.param) + at0 + at, wide, hop, valid, w);
        }
    }

    // ---- teardown -------------------------------------------------------------------------------------
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);      // products may still be in flight
        __syncthreads();
    }
    if (C > 1) cluster_sync_all();                             // no CTA leaves while a peer may write to it
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tmem, a.tmem_cols);
    }
}

int small_cluster(int rows, int cols) {
    const int m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (m > SMALL_SIDE) return 0;
    for (int c = 1; c <= SMALL_CTAS; c *= 2)
        if (n <= c * SMALL_SLAB) return c;
    return 0;
}

template <int TERMS> static r3_status launch_small(SmallArgs& a, int matrices, cudaStream_t cs) {
    // shared memory for the largest of the stacks
    int slab = 16, side = 16;
    for (int i = 0; i < a.stacks; ++i) {
        const int m = a.stack[i].rows < a.stack[i].cols ? a.stack[i].rows : a.stack[i].cols;
        const int n = a.stack[i].rows < a.stack[i].cols ? a.stack[i].cols : a.stack[i].rows;
        const int w = ((n + a.cluster - 1) / a.cluster + 15) & ~15;
        slab = w > slab ? w : slab;
        side = m > side ? m : side;
    }
    a.x_blocks = (slab + 63) / 64;
    a.a_blocks = (side + 63) / 64;
    a.a_bytes = a.cluster > 1 ? 4 * SM_BLOCK : (TERMS > 1 ? 2 : 1) * a.a_blocks * SM_BLOCK;
    a.tmem_cols = 32;
    while (a.tmem_cols < slab || a.tmem_cols < side) a.tmem_cols *= 2;
    const size_t smem = 1024 + 2 * (size_t)a.x_blocks * SM_BLOCK + a.a_bytes + SM_MISC;
    static PerDevice ready;
    if (!ready.done()) {
        if (cudaFuncSetAttribute(small_kernel<TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 1024 + 12 * SM_BLOCK + SM_MISC) != cudaSuccess)
            return R3_ERR_CUDA;
        ready.mark();
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)matrices * (unsigned)a.cluster);
    cfg.blockDim = dim3(SM_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = cs;
    cfg.attrs = attr;
    cfg.numAttrs = a.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, small_kernel<TERMS>, a) == cudaSuccess ? R3_OK : R3_ERR_CUDA;
}

r3_status run_small(SmallArgs& a, int terms, int matrices, cudaStream_t cs) {
    return terms > 1 ? launch_small<3>(a, matrices, cs) : launch_small<1>(a, matrices, cs);
}

}  // namespace ns
}  // namespace r3
