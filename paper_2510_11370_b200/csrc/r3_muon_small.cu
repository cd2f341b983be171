// The orthogonalised update of matrices whose smaller side is at most 128, in one launch: gradient and
// momentum are read, the whole iteration runs on the chip, the weights are written.  (r3_muon.cu holds the
// method, its numbers and the form for larger matrices, whose iterates go through memory between products.)
//
// With m <= 128 the smaller side, X [m, n] lies across the CTAs of a cluster, up to 256 columns each, as two fp16
// planes in shared memory.  The same tiles (64 columns to a 128-byte row, swizzled) are the K-major operands of
// X X^T and the MN-major operand of B X, so nothing is ever laid out again, and every product's epilogue
// replaces its operand in place.  A is m x m: with more than one CTA the parts X_s X_s^T are added up through
// distributed shared memory, each CTA a share of A's rows, which it then copies to all (whole rows: they lie
// together, a copy takes 128 / C of them; as stores of single columns this took 14 us of a step's 26);
// a I + b A + c A^2 is small and every CTA forms it for itself.
// Bound by latency, fifteen products with their epilogues one after the other: of a step of 128 x 256 with three
// products, 17000 clocks, the tensor pipe of the one SM has 8900 (7700 at its rate), the epilogues the others.
// 24 matrices of 256 x 128 f32 with their momentum 70 us, 128 x 2048 f32 over eight CTAs 83, of which the parts'
// exchange takes 20.
#include "r3_muon.cuh"

namespace r3 {
namespace ns {

constexpr int SM_THREADS = 512;
constexpr int SM_WARPS = SM_THREADS / 32;
constexpr int SM_UNITS = 128 * SMALL_SLAB / 8 / SM_THREADS;      // octets of X per thread
constexpr int SM_BLOCK = 128 * 128;           // bytes of 128 rows x 64 columns of fp16
constexpr int SM_MISC = 512;

__device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_remote(uint32_t at, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};"
                 ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
// Shared memory of this CTA to that of another (or this) one; the bytes are counted on a barrier there.
__device__ __forceinline__ void copy_remote(uint32_t to, uint32_t from, uint32_t bytes, uint32_t to_bar) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(to), "r"(from), "r"(bytes), "r"(to_bar) : "memory");
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
        l[i] = __floats2half2_rn((x[2 * i] - f.x) * LO, (x[2 * i + 1] - f.y) * LO);
    }
}
// x += v, or v / LO where it is of a lo plane.
template <bool LOW> __device__ __forceinline__ void add8(const uint4& v, float (&x)[8]) {
    const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(h[i]);
        x[2 * i] = fmaf(f.x, LOW ? 1.f / LO : 1.f, x[2 * i]);
        x[2 * i + 1] = fmaf(f.y, LOW ? 1.f / LO : 1.f, x[2 * i + 1]);
    }
}

// Eight elements: together (VEC), or `step` apart, of which `valid` exist (the others read as 0).
template <bool VEC, typename T>
__device__ __forceinline__ void get8(const T* p, int step, int valid, float (&f)[8]) {
    if (VEC) {
        load8(p, f);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = k < valid ? to_f32(p[(long long)k * step]) : 0.f;
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void put8(T* p, int step, int valid, const float (&f)[8]) {
    if (VEC) {
        store8(p, f);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < valid) p[(long long)k * step] = from_f32<T>(f[k]);
    }
}
// A thread's octets of X: numbers threadIdx.x + SM_THREADS e of 128 rows x `octets`, rows fastest where the
// matrix in memory is tall.
struct Octets {
    int octets, m, jn, row;               // rows of X, columns in this CTA, elements of a row in memory
    long long first;                      // elements before this CTA's first column
    bool tall;
    int i, o, hop_i, hop_o;
    __device__ __forceinline__ void begin() {
        const int u = threadIdx.x;
        i = tall ? u & 127 : u / octets;
        o = tall ? u >> 7 : u - i * octets;
        hop_i = tall ? 0 : SM_THREADS / octets;
        hop_o = tall ? SM_THREADS >> 7 : SM_THREADS - hop_i * octets;
    }
    __device__ __forceinline__ void next() {
        i += hop_i;
        o += hop_o;
        if (!tall && o >= octets) {
            o -= octets;
            ++i;
        }
    }
    __device__ __forceinline__ bool within() const { return i < 128 && o < octets; }
    __device__ __forceinline__ int valid() const { return within() && i < m ? max(0, min(8, jn - 8 * o)) : 0; }
    __device__ __forceinline__ long long at() const {
        return tall ? first + (long long)(8 * o) * row + i : first + (long long)i * row + 8 * o;
    }
};
// Reads them, updates the momentum, leaves u; returns the sum of u^2.  Two octets at a time are under way.
template <bool VEC, typename G>
__device__ __forceinline__ double read_octets(const SmallArgs& a, Octets w, const G* grad, float* mom, float gs,
                                              float (&u)[SM_UNITS][8]) {
    double sum = 0.0;
    const int hop = w.tall ? w.row : 1;
    w.begin();
#pragma unroll
    for (int e0 = 0; e0 < SM_UNITS; e0 += 2) {
        int valid[2];
        long long at[2];
        float v[2][8];
#pragma unroll
        for (int e = 0; e < 2; ++e, w.next()) {
            valid[e] = w.valid();
            at[e] = w.at();
#pragma unroll
            for (int k = 0; k < 8; ++k) u[e0 + e][k] = v[e][k] = 0.f;
            if (valid[e] > 0) {
                get8<VEC>(grad + at[e], hop, valid[e], u[e0 + e]);
                if (mom) get8<VEC>(mom + at[e], hop, valid[e], v[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (mom) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    v[e][k] = __fadd_rn(__fmul_rn(a.momentum, v[e][k]), __fmul_rn(u[e0 + e][k], gs));
                if (valid[e] > 0) put8<VEC>(mom + at[e], hop, valid[e], v[e]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float x =
                    direction(a.nesterov, a.momentum, mom != nullptr, __fmul_rn(u[e0 + e][k], gs), v[e][k]);
                u[e0 + e][k] = x;
                sum += (double)x * (double)x;
            }
        }
    }
    return sum;
}
// The result, or the weights' update, from the planes.
template <bool VEC, typename P>
__device__ __forceinline__ void write_octets(const SmallArgs& a, Octets w, const uint8_t* planes, uint32_t plane,
                                             P* param, float* master, float keep, float rate) {
    const int hop = w.tall ? w.row : 1;
    w.begin();
#pragma unroll
    for (int e0 = 0; e0 < SM_UNITS; e0 += 4) {
        int valid[4];
        long long at[4];
        uint32_t t[4];
        float old[4][8];
#pragma unroll
        for (int e = 0; e < 4; ++e, w.next()) {
            valid[e] = w.valid();
            at[e] = w.at();
            t[e] = tile_at(w.i, 8 * w.o);
            if (a.step && valid[e] > 0) {
                if (master) get8<VEC>(master + at[e], hop, valid[e], old[e]);
                else get8<VEC>(param + at[e], hop, valid[e], old[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (valid[e] == 0) continue;
            float x[8] = {};
            add8<false>(*reinterpret_cast<const uint4*>(planes + t[e]), x);
            add8<true>(*reinterpret_cast<const uint4*>(planes + plane + t[e]), x);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = a.step ? old[e][k] * keep - rate * x[k] : -rate * x[k];
            if (master) put8<VEC>(master + at[e], hop, valid[e], x);
            put8<VEC>(param + at[e], hop, valid[e], x);
        }
    }
}

template <int TERMS>
__global__ void __launch_bounds__(SM_THREADS, 1) small_kernel(const __grid_constant__ SmallArgs a) {
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
    const uint32_t bar = base + a0 + a.a_bytes, a_bar = bar + 8, bar2 = bar + 24;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc + 16);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 20);
    double* s_sum = reinterpret_cast<double*>(misc + 64);           // [SM_WARPS]
    double* s_norm = reinterpret_cast<double*>(misc + 192);         // [SMALL_CTAS]
    const uint32_t norm_at = base + a0 + a.a_bytes + 192;

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
        mbar_init(a_bar, 1);
        mbar_init(bar2, 1);
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
        const long long at0 = (long long)z * st.rows * st.cols;
        const bool vec = !tall && (st.cols & 7) == 0;
        float* mom = st.momentum ? st.momentum + at0 : nullptr;
        Octets mine;
        mine.octets = octets;
        mine.m = m;
        mine.jn = jn;
        mine.row = st.cols;
        mine.first = tall ? (long long)j0 * st.cols : j0;
        mine.tall = tall;
        float u[SM_UNITS][8];
        double sum;
        if (a.grad_dtype == R3_BF16) {
            const __nv_bfloat16* grad = static_cast<const __nv_bfloat16*>(st.grad) + at0;
            sum = vec ? read_octets<true>(a, mine, grad, mom, gs, u) : read_octets<false>(a, mine, grad, mom, gs, u);
        } else {
            const float* grad = static_cast<const float*>(st.grad) + at0;
            sum = vec ? read_octets<true>(a, mine, grad, mom, gs, u) : read_octets<false>(a, mine, grad, mom, gs, u);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_sum[warp] = sum;
        __syncthreads();
        if (threadIdx.x < C) {
            sum = 0.0;
            for (int i = 0; i < SM_WARPS; ++i) sum += s_sum[i];
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
        const float inv = start_scale(sum, a.eps), up = a.scale / LEAST_SCALE, unscale = 1.f / a.scale;
        // ---- X = u / (|u| + eps) into the planes, zeros around it ----------------------------------
        Octets w = mine;
        w.begin();
#pragma unroll
        for (int e = 0; e < SM_UNITS; ++e, w.next()) {
            if (!w.within()) break;
            // (a product of zero and an infinite or undefined scale would leave NaN around the matrix)
            const int valid = w.valid();
#pragma unroll
            for (int k = 0; k < 8; ++k) u[e][k] = k < valid ? u[e][k] * inv * up : 0.f;
            uint4 hi, lo;
            split8(u[e], &hi, &lo);
            const uint32_t t = tile_at(w.i, 8 * w.o);
            *reinterpret_cast<uint4*>(bp + t) = hi;
            *reinterpret_cast<uint4*>(bp + x_plane + t) = lo;
        }
        fence_async();
        __syncthreads();

        // ---- the iteration ---------------------------------------------------------------------------
        const int q = warp & 3, quarter = warp >> 2, r = q * 32 + lane;   // this thread's row of every product
        const int m32 = (m16 + 31) & ~31, w32 = (W + 31) & ~31;
        const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16);
        uint32_t phase = 0, phase2 = 0, a_phase = 0;
        bool alive = true;
        // D = P Q over the steps of 16 along k from `k0` to `k1`, columns c0 to c0 + N of D; plane choice by term,
        // small products first, onto 2^-11 of whose sum
        // (they hold a lo plane) comes the large one.  Three products: every 64 of k have an accumulator of their own, `apart` columns
        // further on, and the epilogue adds them up (an addition in tensor memory drops what lies below the
        // running sum's last place).
        auto issue = [&](uint32_t p0, uint32_t p_plane, uint32_t q0, uint32_t q_plane, bool q_mn, int c0, int N,
                         int apart, int k0, int k1, uint32_t done) {
            if (warp == 0) {
                tc_fence_after();
                if (alive && elect_one()) {
                    const uint32_t idesc = (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24) |
                                           (q_mn ? 1u << 16 : 0u);
                    const uint64_t q_step = q_mn ? 2048 >> 4 : 2;          // (a descriptor counts 16 bytes)
                    for (int seg = k0; seg < k1; seg += 4) {
                        const uint32_t d = tmem + (uint32_t)(c0 + (TERMS > 1 ? (seg >> 2) * apart : 0));
                        const uint32_t block = (uint32_t)((seg >> 2) * SM_BLOCK);
                        const uint32_t p = base + p0 + block;
                        const uint32_t qq = base + q0 + (q_mn ? (uint32_t)(c0 >> 6) * SM_BLOCK + (uint32_t)seg * 2048u : block);
#pragma unroll
                        for (int term = 0; term < TERMS; ++term) {
                            const uint32_t tq = qq + (TERMS > 1 && term == 0 ? q_plane : 0u);
                            const uint64_t dp = smem_desc_sw128(p + (TERMS > 1 && term == 1 ? p_plane : 0u));
                            const uint64_t dq = q_mn ? smem_desc_mn_sw128(tq, SM_BLOCK) : smem_desc_sw128(tq);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (seg + j >= k1) continue;
                                if (term == 2 && j == 0)
                                    tc_mma_bf16_onto_scaled<LO_SHIFT>(d, dp, dq, idesc);
                                else
                                    tc_mma_bf16(d, dp + 2 * j, dq + q_step * j, idesc,
                                                (term | j) != 0 || (TERMS == 1 && seg != k0) ? 1u : 0u);
                            }
                        }
                    }
                    tc_commit(done);
                }
                __syncwarp();
            }
        };
        auto wait = [&](uint32_t done, uint32_t& phase) {
            if (alive) {
                const bool ok = mbar_wait(done, phase, abort_flag, a.dev_status);
                alive = __all_sync(0xffffffffu, ok);
            }
            phase ^= 1u;
            tc_fence_after();
        };
        // 32 columns of this thread's row, the accumulators of k16 steps `apart` columns apart added up
        auto take = [&](int c, int apart, int k16, float (&v)[32]) {
            tc_ld32(trow + c, v);
            tc_wait_ld();
            if (TERMS > 1) {
#pragma unroll 1
                for (int seg = 4; seg < k16; seg += 4) {
                    float more[32];
                    tc_ld32(trow + c + (seg >> 2) * apart, more);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] += more[k];
                }
            }
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
            issue(0, x_plane, 0, x_plane, false, 0, m16, m32, 0, W >> 4, bar);
            wait(bar, phase);
            if (C == 1) {
                const int c = quarter * 32;
                if (alive && c < m16) {
                    float v[32];
                    take(c, m32, W >> 4, v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] = v[8 * j + k] * unscale;
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
                // parts to the owners of their rows: [source][4 columns][row], in the A region, once every
                // CTA has its last product with B behind it
                if (s > 0) cluster_wait();
                const int share = 128 / C;               // rows per owner
                const int c = quarter * 32;
                if (alive && c < m16) {
                    float v[32];
                    take(c, m32, W >> 4, v);
                    const uint32_t to = mapa_shared(base + a0 + rank * (uint32_t)(share * 512), (uint32_t)(r / share));
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + 4 * j < m16)
                            store_remote(to + (uint32_t)(((c / 4 + j) * share + r % share) * 16),
                                         make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
                }
                tc_fence_before();
                __syncwarp();
                cluster_sync_all();
                // the sums, as rows of the planes, to a place of their own: [plane][block][row]
                const uint32_t rows_bytes = (uint32_t)share * 128u, staged = a0 + (uint32_t)(4 * SM_BLOCK);
                for (int u = threadIdx.x; u < share * (m16 >> 3); u += SM_THREADS) {
                    const int rr = u % share, o = u / share;
                    float x[8] = {};
                    for (int src = 0; src < C; ++src) {
                        const float4* p = reinterpret_cast<const float4*>(bp + a0 + (uint32_t)(src * share * 512)) +
                                          2 * o * share + rr;
                        const float4 f = p[0], h = p[share];
                        x[0] += f.x; x[1] += f.y; x[2] += f.z; x[3] += f.w;
                        x[4] += h.x; x[5] += h.y; x[6] += h.z; x[7] += h.w;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] *= unscale;
                    uint4 hi, lo;
                    split8(x, &hi, &lo);
                    const uint32_t t = staged + (uint32_t)(o >> 3) * rows_bytes + (uint32_t)(rr * 128) +
                                       (uint32_t)(((o & 7) ^ (rr & 7)) << 4);
                    *reinterpret_cast<uint4*>(bp + t) = hi;
                    if (PL > 1) *reinterpret_cast<uint4*>(bp + t + (uint32_t)a.a_blocks * rows_bytes) = lo;
                }
                fence_async();
                __syncwarp();
                cluster_sync_all();                      // every CTA has read its parts: A may stand there now
                if (warp == 0) {
                    const int pieces = PL * a.a_blocks;  // times C copies: 32 at most
                    if (lane == 0) mbar_expect_tx(a_bar, (uint32_t)(pieces * SM_BLOCK));
                    if (lane < pieces * C) {
                        const uint32_t to = (uint32_t)(lane % C), piece = (uint32_t)(lane / C);
                        copy_remote(mapa_shared(base + a0 + piece * SM_BLOCK + rank * rows_bytes, to),
                                    base + staged + piece * rows_bytes, rows_bytes, mapa_shared(a_bar, to));
                    }
                    __syncwarp();
                }
                if (alive) {
                    const bool ok = mbar_wait(a_bar, a_phase, abort_flag, a.dev_status);
                    alive = __all_sync(0xffffffffu, ok);
                }
                a_phase ^= 1u;
            }
            // B = a I + b A + c A^2, in A's place (three products: without a I, a X is added in float32)
            issue(a0, a_plane, a0, a_plane, false, 0, m16, m32, 0, m16 >> 4, bar);
            wait(bar, phase);
            const int c_square = quarter * 32;
            if (alive && c_square < m16) {
                const int c = c_square;
                float v[32];
                take(c, m32, m16 >> 4, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c + 8 * j >= m16) continue;
                    const uint32_t t = a0 + tile_at(r, c + 8 * j);
                    float x[8] = {};
                    add8<false>(*reinterpret_cast<const uint4*>(bp + t), x);
                    if (PL > 1) add8<true>(*reinterpret_cast<const uint4*>(bp + a_plane + t), x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        x[k] = fmaf(cb, x[k], cc * unscale * v[8 * j + k]);
                        if (TERMS == 1 && c + 8 * j + k == r) x[k] += ca * a.scale;
                    }
                    uint4 hi, lo;
                    split8(x, &hi, &lo);
                    *reinterpret_cast<uint4*>(bp + t) = hi;
                    if (PL > 1) *reinterpret_cast<uint4*>(bp + a_plane + t) = lo;
                }
            }
            written();
            // X = B X, in X's place (one product: + a times the lo plane, which is no operand then; three: + a X)
            // the second half of X's columns is multiplied while the first half's sums are taken
            issue(a0, a_plane, 0, x_plane, true, 0, min(W, 128), w32, 0, m16 >> 4, bar);
            if (W > 128) issue(a0, a_plane, 0, x_plane, true, 128, W - 128, w32, 0, m16 >> 4, bar2);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (half == 0) wait(bar, phase);
                else if (W > 128) wait(bar2, phase2);
                if (C > 1 && s + 1 < a.steps && half == (W > 128 ? 1 : 0)) {
                    __syncwarp();
                    cluster_arrive();                    // B is read: the next parts may come
                }
                const int c = half * 128 + quarter * 32;
                if (!alive || c >= W) continue;
                float v[32];
                take(c, w32, m16 >> 4, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c + 8 * j >= W) continue;
                    const uint32_t t = tile_at(r, c + 8 * j);
                    float x[8] = {};
                    if (TERMS > 1) add8<false>(*reinterpret_cast<const uint4*>(bp + t), x);
                    add8<true>(*reinterpret_cast<const uint4*>(bp + x_plane + t), x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = fmaf(ca, x[k], unscale * v[8 * j + k]);
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
        const float keep = 1.f - lr * st.decay, rate = a.step ? lr * st.scale * unscale : -unscale;
        float* master = st.master ? st.master + at0 : nullptr;
        if (a.param_dtype == R3_BF16) {
            __nv_bfloat16* param = static_cast<__nv_bfloat16*>(st.param) + at0;
            if (vec) write_octets<true>(a, mine, bp, x_plane, param, master, keep, rate);
            else write_octets<false>(a, mine, bp, x_plane, param, master, keep, rate);
        } else {
            float* param = static_cast<float*>(st.param) + at0;
            if (vec) write_octets<true>(a, mine, bp, x_plane, param, master, keep, rate);
            else write_octets<false>(a, mine, bp, x_plane, param, master, keep, rate);
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
    // (several CTAs: the parts, 128 x 128 float32, and the sums of this CTA's rows)
    a.a_bytes = a.cluster > 1 ? 4 * SM_BLOCK + (TERMS > 1 ? 2 : 1) * a.a_blocks * (SM_BLOCK / a.cluster)
                              : (TERMS > 1 ? 2 : 1) * a.a_blocks * SM_BLOCK;
    // accumulators of up to 128 or 256 columns, one per 64 of k with three products: 512 columns at most
    const int side32 = (side + 31) & ~31, slab32 = (slab + 31) & ~31;
    const int by_slab = TERMS > 1 ? (slab + 63) / 64 : 1, by_side = TERMS > 1 ? (side32 + 63) / 64 : 1;
    int cols = by_slab * side32;
    if (by_side * side32 > cols) cols = by_side * side32;
    if (by_side * slab32 > cols) cols = by_side * slab32;
    a.tmem_cols = 32;
    while (a.tmem_cols < cols) a.tmem_cols *= 2;
    const size_t smem = 1024 + 2 * (size_t)a.x_blocks * SM_BLOCK + a.a_bytes + SM_MISC;
    static PerDevice ready;
    if (!ready.done()) {
        if (cudaFuncSetAttribute(small_kernel<TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 1024 + 14 * SM_BLOCK + SM_MISC) != cudaSuccess)
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
