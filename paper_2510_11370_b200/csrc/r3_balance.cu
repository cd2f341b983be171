// Balance loss and z loss of the routers of L blocks, the counts per expert, and the gradient to the
// router logits.  Per block, over N tokens, with p the softmax of a token's logits over ALL experts and
// counts the choices of the record,
//   f_i = E counts_i / sum_j counts_j      balance = sum_i f_i mean_t p_ti
//   z   = mean_t (log sum_i exp s_ti)^2
//   ds_ti = balance_coef p_ti (f_i - sum_j f_j p_tj) / N  +  2 z_coef lse_t p_ti / N
// The counts do not depend on the logits, so they come first, from the record alone (K bytes a token),
// and the logits are then read once: the pass that forms the probabilities has f and N in hand and
// writes the gradient at once.  Bound by HBM: 8 E + K bytes a token and block.
//
// Counting: a cluster per part of a block's tokens, counters in shared memory, added up over the cluster.
// Main pass: a token's logits lie across G lanes, 8 each where the experts are many (a shuffle then serves
// 32 / G tokens), so that its maximum, its sum and its product with f are shuffles; a lane keeps the f of its
// experts and the sums of their probabilities in registers, and the next tokens' logits are under way while
// these are worked on.  The first logits come into L2 while the choices are still counted.  All resident CTAs take
// equal shares of the L T tokens, across the borders of blocks where need be (grids of whole parts per block left
// a second wave of 32 CTAs for 48 blocks: 285 us against 150).  A CTA's sums end in one number, counts times
// probabilities, and the last CTA of a block to arrive adds these up, in an order that depends on the shape alone
// (rows of sums per CTA, added up by the last one: 26 us instead of 22 for 65536 tokens).
// 48 blocks of 16384 tokens, 128 experts: 147 us, 5.5 TB/s of the 812 MB that have to move; one block of 65536
// tokens: 22 us, of which the counting pass and the main pass's start are 9, the logits 10, the losses 3.  Above 512
// experts a lane's 32 logits, sums and shares of the counts do not fit its 128 registers (the compiler leaves 500 to
// 600 bytes of them in local memory): 8 blocks of 8192 tokens, 1024 experts 126 us against 83 for their bytes.
#include <cfloat>
#include <cmath>

#include "r3_common.cuh"
#include "r3_internal.h"
#include "r3_tc.cuh"

namespace r3 {
namespace bal {

constexpr int MAX_EXPERTS = 1024;
constexpr int MAX_TOKENS = 1 << 30;       // of a block: a CTA's hop beyond them is still a 32-bit number
constexpr int COUNT_THREADS = 256;
constexpr int COUNT_TOKENS = 1024;        // tokens of a CTA of the counting pass
constexpr int COUNT_CTAS = 8;             // CTAs of its clusters
constexpr int THREADS = 512;
constexpr int WARPS = THREADS / 32;
constexpr int CTAS_PER_SM = 2;
constexpr int EARLY_BYTES = 32 << 20;     // of logits that all CTAs fetch ahead: a part of L2
constexpr int ALONE = 8192;               // logits of a block that one CTA takes with its choices
constexpr int FOLD = 64;                  // tokens of a lane that are added up in float32
constexpr float FAR = 1e6f;               // logits beyond: 0.05 and more of rounding in their product with log2(e)
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Args {
    int T, E, K, L;
    int count_parts, count_ctas;          // clusters per block in the counting pass, CTAs of each
    int grid;                             // CTAs of the main pass
    int alone, idx_bytes;                 // one CTA per block, which counts its choices itself
    int accumulate, given;
    float balance_coef, z_coef;
    const float* logits;
    const void* idx;
    const uint8_t* mask;
    int32_t* counts;                      // given, or written (may be null)
    float* loss;                          // [L, 2]
    float* dlogits;                       // or null
    int32_t* part_counts;                 // [L, count_parts, E + 1]: per expert, then the tokens
    double2* part;                        // [grid + L]: the sums of a CTA and a block that it has tokens of
    unsigned* ticket;                     // [L]
    int32_t* dev_status;
};
// The hardware's approximations: 2^x and 1 / x within 2^-22 of the value, log2(x) within 2^-22 above 2.
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_inverse(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_log2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The tokens of a CTA, as numbers of the L T; block l's first CTA and the number of its CTAs follow.
__device__ __forceinline__ long long first_token(const Args& a, int cta) {
    return (long long)a.L * a.T * cta / a.grid;
}
__device__ __forceinline__ int cta_of(const Args& a, long long token) {
    int c = (int)(token * a.grid / ((long long)a.L * a.T));
    while (c + 1 < a.grid && first_token(a, c + 1) <= token) ++c;
    while (c > 0 && first_token(a, c) > token) --c;
    return c;
}

// ---- counting pass: grid (count_parts * count_ctas, L), clusters of count_ctas -------------------
template <typename IdxT>
__global__ void __launch_bounds__(COUNT_THREADS) count_kernel(const __grid_constant__ Args a) {
    extern __shared__ int s_count[];
    const int l = blockIdx.y, E = a.E, K = a.K;
    for (int e = threadIdx.x; e <= E; e += COUNT_THREADS) s_count[e] = 0;
    __syncthreads();
    // the main pass may start once everything in front of this one is done: until this one is too it only brings its
    // first logits into L2
    tc::grid_dependency_wait();
    tc::grid_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x == 0) a.ticket[l] = 0;
    const int t0 = (int)min((long long)a.T, (long long)blockIdx.x * COUNT_TOKENS), t1 = min(a.T, t0 + COUNT_TOKENS);
    if (a.mask) {
        int n = 0;
        for (int t = t0 + threadIdx.x; t < t1; t += COUNT_THREADS) n += a.mask[t] != 0;
        n = __reduce_add_sync(0xffffffffu, n);
        if ((threadIdx.x & 31) == 0 && n) atomicAdd(&s_count[E], n);
    } else if (threadIdx.x == 0) {
        s_count[E] = t1 - t0;
    }
    if (!a.given) {
        const IdxT* idx = static_cast<const IdxT*>(a.idx) + ((size_t)l * a.T + t0) * K;
        const int n = (t1 - t0) * K;
        auto take = [&](int i, int e) {
            if (a.mask && !a.mask[t0 + i / K]) return;
            if (e < 0 || e >= E) {
                report(a.dev_status, R3_DEV_BAD_INDEX);
                return;
            }
            atomicAdd(&s_count[e], 1);
        };
        constexpr int VEC = 16 / (int)sizeof(IdxT);
        // the record's base is aligned to 16 bytes, a CTA's first choice need not be
        const int skip = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(idx) & 15)) & 15) / (int)sizeof(IdxT));
        const int vecs = (n - skip) / VEC;
        for (int i = threadIdx.x; i < skip; i += COUNT_THREADS) take(i, idx_to_int(idx[i]));
        for (int v = threadIdx.x; v < vecs; v += COUNT_THREADS) {
            const int4 w = *reinterpret_cast<const int4*>(idx + skip + v * VEC);
            const IdxT* x = reinterpret_cast<const IdxT*>(&w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) take(skip + v * VEC + j, idx_to_int(x[j]));
        }
        for (int i = skip + vecs * VEC + threadIdx.x; i < n; i += COUNT_THREADS) take(i, idx_to_int(idx[i]));
    }
    const int ctas = a.count_ctas;
    const int part = ctas > 1 ? blockIdx.x / ctas : blockIdx.x;
    int32_t* out = a.part_counts + ((size_t)l * a.count_parts + part) * (E + 1);
    if (ctas == 1) {
        __syncthreads();
        for (int e = threadIdx.x; e <= E; e += COUNT_THREADS) out[e] = s_count[e];
        return;
    }
    __syncwarp();
    tc::cluster_sync_all();
    const int rank = (int)tc::cluster_ctarank();
    for (int e = threadIdx.x * ctas + rank; e <= E; e += COUNT_THREADS * ctas) {
        int n = 0;
        int v[COUNT_CTAS];                               // (all of them under way at once)
#pragma unroll
        for (int c = 0; c < COUNT_CTAS; ++c)
            asm volatile("ld.shared::cluster.s32 %0, [%1];"
                         : "=r"(v[c])
                         : "r"(tc::mapa_shared(tc::smem_u32(s_count + e), (uint32_t)min(c, ctas - 1))) : "memory");
#pragma unroll
        for (int c = 0; c < COUNT_CTAS; ++c) n += c < ctas ? v[c] : 0;
        out[e] = n;
    }
    __syncwarp();
    tc::cluster_sync_all();                              // no CTA leaves while another reads its counters
}

// ---- main pass ------------------------------------------------------------------------------------
// G lanes per token, V logits per lane.  WIDE: E is a multiple of 4, a lane's logits come in fours
// (columns 4 (lane + G q) ..); otherwise one by one (columns lane + G q).
template <int G, int V, bool WIDE> struct Row {
    static __device__ __forceinline__ int column(int sub, int j) {
        return WIDE ? 4 * (sub + G * (j / 4)) + j % 4 : sub + G * j;
    }
    static __device__ __forceinline__ void load(const float* p, int E, int sub, float (&v)[V], float none) {
        if constexpr (WIDE) {
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                const int c = 4 * (sub + G * q);
                const float4 f = c < E ? *reinterpret_cast<const float4*>(p + c)
                                       : make_float4(none, none, none, none);
                v[4 * q] = f.x;
                v[4 * q + 1] = f.y;
                v[4 * q + 2] = f.z;
                v[4 * q + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = sub + G * j < E ? p[sub + G * j] : none;
        }
    }
    static __device__ __forceinline__ void store(float* p, int E, int sub, const float (&v)[V]) {
        if constexpr (WIDE) {
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                const int c = 4 * (sub + G * q);
                if (c < E) *reinterpret_cast<float4*>(p + c) =
                    make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (sub + G * j < E) p[sub + G * j] = v[j];
        }
    }
};

template <int G, int V, bool WIDE>
__global__ void __launch_bounds__(THREADS, V <= 8 ? CTAS_PER_SM : 1) balance_kernel(const __grid_constant__ Args a) {
    using R = Row<G, V, WIDE>;
    constexpr int ROWS = 32 / G;                       // tokens of a warp at a time
    extern __shared__ float s_n[];                     // [E] counts, then [WARPS][E] sums of probabilities in 64 bits
    double* s_col = reinterpret_cast<double*>(s_n + ((a.E + 3) & ~3));
    __shared__ long long s_sum[WARPS];
    __shared__ double s_z[WARPS], s_b[WARPS];
    __shared__ int s_tokens;
    __shared__ bool s_last;
    const int E = a.E, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane % G, row = lane / G;
    tc::grid_launch_dependents();
    const long long begin = first_token(a, blockIdx.x), end = first_token(a, blockIdx.x + 1);
    {
        // while the choices are counted, this CTA's first logits come into L2
        const char* from = reinterpret_cast<const char*>(a.logits + (size_t)begin * E);
        const long long bytes = min((end - begin) * E * 4, (long long)(EARLY_BYTES / gridDim.x));
        for (long long at = threadIdx.x * 128LL; at < bytes; at += THREADS * 128LL)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(from + at));
    }
    tc::grid_dependency_wait();
    // an empty batch: CTA 0 still writes the losses of every block
    const int l_first = a.T > 0 ? (int)(begin / a.T) : 0;
    const int l_past = a.T > 0 ? (end > begin ? (int)((end - 1) / a.T) + 1 : l_first) : a.L;
    for (int l = l_first; l < l_past; ++l) {
        const long long block0 = (long long)l * a.T;
        const int t0 = (int)(max(begin, block0) - block0), t1 = (int)(min(end, block0 + a.T) - block0);
        const float* logits = a.logits + (size_t)block0 * E;
        float* dlogits = a.dlogits ? a.dlogits + (size_t)block0 * E : nullptr;
        const int hop = WARPS * ROWS;
        // the first tokens' logits are under way while the counts are added up
        float next[V];
        bool next_on = false;
        auto fetch = [&](int t) {
            const int at = t + row;
            next_on = at < t1 && (!a.mask || a.mask[at]);
            if (at < t1) {                             // (not behind the mask's arrival)
                R::load(logits + (size_t)at * E, E, sub, next, -INFINITY);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) next[j] = -INFINITY;
            }
        };
        fetch(t0 + warp * ROWS);
        int* s_count = reinterpret_cast<int*>(s_col);  // [E + 1], until the sums of probabilities take the place
        if (a.alone) {
            for (int e = threadIdx.x; e <= E; e += THREADS) s_count[e] = 0;
            __syncthreads();
            for (int t = threadIdx.x; t < a.T; t += THREADS)
                if (!a.mask || a.mask[t]) atomicAdd(s_count + E, 1);
            const size_t from = (size_t)block0 * a.K;
            for (int i = threadIdx.x; !a.given && i < a.T * a.K; i += THREADS) {
                if (a.mask && !a.mask[i / a.K]) continue;
                const int e = a.idx_bytes == 1 ? static_cast<const uint8_t*>(a.idx)[from + i]
                                               : static_cast<const int16_t*>(a.idx)[from + i];
                if (e < 0 || e >= E) report(a.dev_status, R3_DEV_BAD_INDEX);
                else atomicAdd(s_count + e, 1);
            }
            __syncthreads();
        }
        // the block's counts, the number of its choices and of its tokens
        long long mine = 0;
        for (int e = threadIdx.x; e <= E; e += THREADS) {
            int n = 0;
            if (e < E && a.given) {
                n = a.counts[(size_t)l * E + e];
            } else if (a.alone) {
                n = s_count[e];
            } else {
                const int32_t* p = a.part_counts + (size_t)l * a.count_parts * (E + 1) + e;
#pragma unroll 8
                for (int q = 0; q < a.count_parts; ++q) n += p[(size_t)q * (E + 1)];
            }
            if (e == E) {
                s_tokens = n;
            } else {
                s_n[e] = (float)n;                     // below 2^24, or off by a rounding
                mine += n;
                if (!a.given && a.counts && t0 == 0) a.counts[(size_t)l * E + e] = n;
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        if (lane == 0) s_sum[warp] = mine;
        __syncthreads();
        long long choices = 0;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) choices += s_sum[i];
        const int tokens = s_tokens;
        const float per_choice = choices > 0 ? (float)E / (float)choices : 0.f;
        const float per_token = tokens > 0 ? 1.f / (float)tokens : 0.f;
        const float gb = a.balance_coef * per_token, gz = 2.f * a.z_coef * per_token;
        float f[V], sum[V];                            // f: balance_coef f_i / N
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = R::column(sub, j);
            f[j] = c < E ? gb * (s_n[c] * per_choice) : 0.f;
            sum[j] = 0.f;
        }
        float z = 0.f;
        // float32 sums of FOLD tokens a lane at most, those then added up in 64 bits: what they are off by does not
        // grow with the batch
        int t = t0 + warp * ROWS;
        for (bool more = false;; more = true) {
            const int stop = min(t1, t + FOLD * hop);
#pragma unroll 2
            for (; t < stop; t += hop) {
                float v[V];
                const bool on = next_on;
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = next[j];
                if (a.mask && !on) {
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] = -INFINITY;
                }
                if (t + hop < t1) fetch(t + hop);
                const int at = t + row;
                float top = v[0];
#pragma unroll
                for (int j = 1; j < V; ++j) top = fmaxf(top, v[j]);
#pragma unroll
                for (int o = G / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                // 2^(s log2(e) - from): from's own rounding is the same for all of a token's logits, but it stands in
                // the exponent (2^7 of it at a top of 2e9, beyond float32), so a large top is taken off first, be it a
                // mask's -1e30 or the type's lowest.  Where all of them are -inf every one gives 0
                const float least = fmaxf(top, -FLT_MAX), off = fabsf(least) > FAR ? least : 0.f;
                const float from = (least - off) * LOG2E;
                float whole = 0.f, along = 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    v[j] = fast_exp2(fmaf(v[j] - off, LOG2E, -from));
                    whole += v[j];
                    along = fmaf(v[j], f[j], along);
                }
#pragma unroll
                for (int o = G / 2; o > 0; o >>= 1) {
                    whole += __shfl_xor_sync(0xffffffffu, whole, o);
                    along += __shfl_xor_sync(0xffffffffu, along, o);
                }
                const float inv = whole != 0.f ? fast_inverse(whole) : 0.f;
                const float lse = whole != 0.f ? fmaf(LN2, from + fast_log2(whole), off) : 0.f;
                z = fmaf(lse, lse, z);                     // 0 where the token does not count
                const float shift = fmaf(gz, lse, -along * inv);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float p = v[j] * inv;
                    sum[j] += p;
                    v[j] = p * (f[j] + shift);
                }
                if (dlogits && at < t1) {
                    float* out = dlogits + (size_t)at * E;
                    if (a.accumulate) {
                        if (on) {
                            float old[V];
                            R::load(out, E, sub, old, 0.f);
#pragma unroll
                            for (int j = 0; j < V; ++j) old[j] += v[j];
                            R::store(out, E, sub, old);
                        }
                    } else {
                        R::store(out, E, sub, v);
                    }
                }
            }
            // lanes that hold the same experts, then the warp's own places
#pragma unroll
            for (int j = 0; j < V; ++j) {
#pragma unroll
                for (int o = G; o < 32; o <<= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
                const int c = R::column(sub, j);
                if (row == 0 && c < E) s_col[warp * E + c] = (more ? s_col[warp * E + c] : 0.0) + (double)sum[j];
                sum[j] = 0.f;
            }
#pragma unroll
            for (int o = G; o < 32; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            if (lane == 0) s_z[warp] = (more ? s_z[warp] : 0.0) + (double)z;
            z = 0.f;
            if (t >= t1) break;
        }
        __syncthreads();
        // this CTA's part of sum_i counts_i sum_t p_ti: the warps in their order
        double balance = 0.0, zz = 0.0;
        for (int c = threadIdx.x; c < E; c += THREADS) {
            double all = 0.0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) all += s_col[w * E + c];
            balance += all * (double)s_n[c];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) balance += __shfl_xor_sync(0xffffffffu, balance, o);
        if (lane == 0) s_b[warp] = balance;
        __syncthreads();
        const int c_first = a.T > 0 ? cta_of(a, block0) : 0, c_last = a.T > 0 ? cta_of(a, block0 + a.T - 1) : 0;
        const int parts = c_last - c_first + 1;
        if (threadIdx.x == 0) {
            balance = 0.0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                balance += s_b[w];
                zz += s_z[w];
            }
            // a place of its own per CTA and block: CTAs that cross a border have two or more
            a.part[blockIdx.x + l] = make_double2(balance, zz);
            __threadfence();
            s_last = a.alone || atomicAdd(a.ticket + l, 1u) == (unsigned)parts - 1u;
        }
        __syncthreads();
        if (!s_last) continue;
        __threadfence();
        balance = zz = 0.0;
        for (int q = threadIdx.x; q < parts; q += THREADS) {
            const double2 part = __ldcg(a.part + (size_t)c_first + l + q);
            balance += part.x;
            zz += part.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            balance += __shfl_xor_sync(0xffffffffu, balance, o);
            zz += __shfl_xor_sync(0xffffffffu, zz, o);
        }
        if (lane == 0) {
            s_b[warp] = balance;
            s_z[warp] = zz;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            balance = zz = 0.0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                balance += s_b[w];
                zz += s_z[w];
            }
            const double n = tokens > 0 ? (double)tokens : 1.0;
            a.loss[2 * l] = choices > 0 ? (float)(balance * (double)E / ((double)choices * n)) : 0.f;
            a.loss[2 * l + 1] = (float)(zz / n);
        }
        __syncthreads();                               // the next block's sums go to the same places
    }
}

struct Plan {
    int count_parts, count_ctas, grid;
    bool alone;
};
// Main pass: every resident CTA, unless a warp's share falls below two tokens or so.  Blocks of few logits: a CTA
// each, without a counting pass (a launch less; 512 tokens of 8 experts 8.8 -> 7.2 us in a graph, 48 blocks of it
// 11.3 -> 8.0; with twice the logits one block would take 9.9 instead of 8.6).
static Plan plan(int T, int L, int E) {
    Plan p;
    const int ctas = T > 0 ? (T + COUNT_TOKENS - 1) / COUNT_TOKENS : 1;
    p.count_ctas = 1;
    while (p.count_ctas < COUNT_CTAS && p.count_ctas < ctas) p.count_ctas *= 2;
    p.count_parts = (ctas + p.count_ctas - 1) / p.count_ctas;
    long long grid = ((long long)T * L + 2 * WARPS - 1) / (2 * WARPS);
    const int most = (E > 256 ? 1 : CTAS_PER_SM) * sm_count();
    if (grid > most) grid = most;
    // whole CTAs per block where that leaves at most a 32nd of them idle: one that crosses a border adds up two
    // blocks' counts and sums (3 blocks of 4097 tokens, 301 experts: 20.1 us instead of 23.8; 48 of 16384: 147, 149)
    if (grid / L * L * 32 >= grid * 31) grid = grid / L * L;
    p.grid = grid < 1 || T == 0 ? 1 : (int)grid;
    p.alone = T > 0 && (long long)T * E <= ALONE;
    if (p.alone) p.grid = L;
    return p;
}
static r3_status check(const r3_shape* s, int32_t L, const r3_balance* c) {
    if (!s || !c || L < 0 || L > 65535) return R3_ERR_INVALID_ARG;
    const r3_status st = check_shape(s);
    if (st != R3_OK) return st;
    if (!(std::fabs(c->balance_coef) < 1e30) || !(std::fabs(c->z_coef) < 1e30)) return R3_ERR_INVALID_ARG;
    return s->E > MAX_EXPERTS || s->T > MAX_TOKENS ? R3_ERR_UNSUPPORTED : R3_OK;
}
struct Layout {
    size_t counts, part, ticket, total;
};
static Layout layout(const r3_shape* s, int32_t L, const Plan& p) {
    Layout w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    w.counts = take((size_t)L * p.count_parts * (s->E + 1) * 4);
    w.part = take(((size_t)p.grid + L) * sizeof(double2));
    w.ticket = take((size_t)L * 4);
    w.total = at;
    return w;
}

template <int G, int V, bool WIDE>
static r3_status launch(const Args& a, cudaStream_t cs) {
    const size_t smem = ((size_t)a.E + 3) / 4 * 4 * sizeof(float) + (size_t)a.E * WARPS * sizeof(double);
    if (smem > 32 * 1024) {                            // above what every kernel may have, with its static part
        static PerDevice ready;
        if (!ready.done()) {
            if (cudaFuncSetAttribute(balance_kernel<G, V, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     MAX_EXPERTS * (WARPS * (int)sizeof(double) + (int)sizeof(float))) != cudaSuccess)
                return R3_ERR_CUDA;
            ready.mark();
        }
    }
    return tc::launch_dependent(balance_kernel<G, V, WIDE>, dim3(a.grid), dim3(THREADS), smem, cs, a) == cudaSuccess
               ? R3_OK : R3_ERR_CUDA;
}
template <bool WIDE>
static r3_status launch(const Args& a, cudaStream_t cs) {
    if (a.E <= 16) return launch<4, 4, WIDE>(a, cs);
    if (a.E <= 64) return launch<8, 8, WIDE>(a, cs);
    if (a.E <= 128) return launch<16, 8, WIDE>(a, cs);
    if (a.E <= 256) return launch<32, 8, WIDE>(a, cs);
    if (a.E <= 512) return launch<32, 16, WIDE>(a, cs);
    return launch<32, 32, WIDE>(a, cs);
}

static bool launch_count(const r3_shape* s, int32_t L, const Plan& p, const Args& a, cudaStream_t cs) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.count_ctas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(p.count_parts * p.count_ctas), (unsigned)L);
    cfg.blockDim = dim3(COUNT_THREADS);
    cfg.dynamicSmemBytes = (size_t)(s->E + 1) * sizeof(int);
    cfg.stream = cs;
    cfg.attrs = attr;
    cfg.numAttrs = p.count_ctas > 1 ? 2 : 1;
    cudaError_t err = cudaSuccess;
    R3_DISPATCH_IDX(s, IdxT, err = cudaLaunchKernelEx(&cfg, count_kernel<IdxT>, a));
    return err == cudaSuccess;
}

}  // namespace bal
}  // namespace r3

extern "C" size_t r3_balance_loss_workspace_bytes(const r3_shape* s, int32_t L) {
    using namespace r3::bal;
    const r3_balance none = {};
    if (check(s, L, &none) != R3_OK || L == 0) return 0;
    return layout(s, L, plan(s->T, L, s->E)).total;
}

extern "C" r3_status r3_balance_loss(const r3_shape* s, int32_t L, const r3_balance* config,
                                     const float* logits, const void* idx, const uint8_t* mask,
                                     int32_t* counts, float* loss, float* dlogits, void* workspace,
                                     size_t ws_bytes, int32_t* dev_status, void* stream) {
    using namespace r3;
    using namespace r3::bal;
    const r3_status st = check(s, L, config);
    if (st != R3_OK) return st;
    if (L == 0) return R3_OK;
    const bool given = config->counts_given != 0;
    if (!loss || (s->T > 0 && (!logits || (!given && !idx))) || (given && !counts)) return R3_ERR_INVALID_ARG;
    if (config->accumulate && !dlogits) return R3_ERR_INVALID_ARG;
    const void* wide[] = {logits, idx, dlogits};
    for (const void* p : wide)
        if (!aligned(p, 16)) return R3_ERR_INVALID_ARG;
    const void* words[] = {counts, loss, dev_status};
    for (const void* p : words)
        if (!aligned(p, 4)) return R3_ERR_INVALID_ARG;
    const Plan p = plan(s->T, L, s->E);
    const Layout w = layout(s, L, p);
    if (!workspace || !aligned(workspace, 256) || ws_bytes < w.total) return R3_ERR_WORKSPACE;
    Args a = {};
    a.T = s->T;
    a.E = s->E;
    a.K = s->K;
    a.L = L;
    a.count_parts = p.count_parts;
    a.count_ctas = p.count_ctas;
    a.grid = p.grid;
    a.accumulate = config->accumulate != 0;
    a.alone = p.alone;
    a.idx_bytes = s->idx_type == R3_IDX_U8 ? 1 : 2;
    a.given = given;
    a.balance_coef = (float)config->balance_coef;
    a.z_coef = (float)config->z_coef;
    a.logits = logits;
    a.idx = idx;
    a.mask = mask;
    a.counts = counts;
    a.loss = loss;
    a.dlogits = dlogits;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.part_counts = reinterpret_cast<int32_t*>(ws + w.counts);
    a.part = reinterpret_cast<double2*>(ws + w.part);
    a.ticket = reinterpret_cast<unsigned*>(ws + w.ticket);
    a.dev_status = dev_status;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (!p.alone && !launch_count(s, L, p, a, cs)) return R3_ERR_CUDA;
    return s->E % 4 == 0 ? launch<true>(a, cs) : launch<false>(a, cs);
}
