// Log probabilities of given tokens from rows of logits, with the entropy and the best
// alternatives of each row, and the gradient to the logits: where the p_train and p_infer of
// Eq. (kl) and Eq. (etdf) come from, and what carries a loss on them back.
//
// One pass over the logits.  With c = log2(e) / temperature every thread keeps an integer
// reference M and the sums
//   S = sum 2^(c x - M),   U = sum 2^(c x - M) (c x - M)
// over its share of the row.  M is a whole number near the running maximum of c x, so that c x - M
// is one fused multiply-add with a single rounding and moving M multiplies S by an exact power of
// two.  M only moves when a value exceeds it by more than 8 (float32 holds 2^8 times the count of
// any row), which is rare after a thread's first values.  With top = max x and S, U taken
// relative to it, log sum exp((x - top) / temperature) = ln S and the entropy is ln S - ln2 U / S,
// two numbers of the size of the result: nothing cancels for large logits.
//
// Bound by HBM as long as the SMs keep up: an element costs one exponential (16 a clock and SM) and, with
// the entropy, 6.2 instructions (10 before the rounds without bounds checks, the widening by shift and
// mask and the sums in two lanes).  8192 x 151936 bf16 with entropy, a tenth of the rows skipped: 342 us =
// the measured copy bandwidth; launched back to back for seconds the power cap takes the SM clock to 1.55
// GHz and the exponentials alone need 290 of 354 to 380 us.  One row per CTA and many CTAs: CTAs that walked
// over rows, the next row's first pieces on their way early, took 444 us where this form took 383.
// Few rows: up to eight CTAs of a cluster share one (16 x 131072 bf16: 4.4 us, with 20 alternatives 9.5,
// of which the alternatives' four barriers, second look at the row and exchange take 5).
#include <math_constants.h>

#include <initializer_list>

#include "r3_common.cuh"
#include "r3_internal.h"
#include "r3_tc.cuh"

namespace r3 {

// CTAs of a given size per SM (64 to 80 registers a thread)
__host__ __device__ constexpr int logprob_ctas(int threads) {
    return threads == 256 ? 4 : threads == 128 ? 8 : 24;
}
constexpr int kMaxTop = 32;            // alternatives per row
constexpr int kMaxSplit = 8;           // CTAs per row
constexpr int kMaxCandidates = 256;
constexpr int kSlots = 16;             // runs of rounds whose maxima a thread keeps
constexpr int kMaxSelected = 512;      // runs that are read again
constexpr float kMoveRef = 8.f;
constexpr float kLowRef = -4194304.f;  // -2^22: the least reference
constexpr float kPlainTop = 1048576.f; // |c top| up to which the reference is exact enough
constexpr float kLeastExp = -200.f;    // 2^-200 is 0 in float32, and 0 * -200 is 0, not NaN

struct LogprobArgs {
    const void* logits;
    const void* ids;
    long long ld;
    int T, V, id64, n_top, split;
    float c, inv_t;
    float* logp;
    float* entropy;
    float* stats;
    int32_t* top_ids;
    float* top_logp;
    int32_t* dev_status;
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN stays one
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// A value and its column as one number: larger values first, then lower columns.  The largest key
// of a set is the first of its largest values; both zeros are the same value.
typedef unsigned long long Key;
__device__ __forceinline__ Key make_key(float v, int column) {
    const uint32_t b = __float_as_uint(v + 0.f);
    const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((Key)o << 32) | (uint32_t)~column;
}
__device__ __forceinline__ float key_value(Key k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o ^ 0x80000000u) : ~o);
}
__device__ __forceinline__ int key_column(Key k) { return (int)~(uint32_t)k; }

// 32 keys, one per lane, into descending order (a bitonic network).
__device__ __forceinline__ Key warp_sort(Key k, int lane) {
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
        for (int j = size >> 1; j > 0; j >>= 1) {
            const Key o = __shfl_xor_sync(0xffffffffu, k, j);
            const bool larger = ((lane & j) == 0) == ((lane & size) == 0);
            k = (k > o) == larger ? k : o;
        }
    }
    return k;
}
// The 32 largest of two descending lists, descending.
__device__ __forceinline__ Key warp_merge(Key a, Key b, int lane) {
    const Key r = __shfl_sync(0xffffffffu, b, 31 - lane);
    Key k = a > r ? a : r;
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) {
        const Key o = __shfl_xor_sync(0xffffffffu, k, j);
        k = (k > o) == ((lane & j) == 0) ? k : o;
    }
    return k;
}

__device__ __forceinline__ long long load_id(const void* ids, int id64, int row) {
    return id64 ? static_cast<const long long*>(ids)[row]
                : (long long)static_cast<const int32_t*>(ids)[row];
}

// How a row of V elements at p splits into single elements up to a 16-byte boundary, whole
// 16-byte pieces, and single elements behind them (rows of an odd V start anywhere).
struct RowSplit {
    int head, vecs, tail;
};
template <typename T> __device__ __forceinline__ RowSplit split_row(const T* p, int V) {
    constexpr int N = Vec16<T>::N;
    RowSplit r;
    const int off = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
    r.head = off ? N - off : 0;
    if (r.head > V) r.head = V;
    r.vecs = (V - r.head) / N;
    r.tail = V - r.head - r.vecs * N;
    return r;
}

// Two float32 values in a register pair, one instruction for both: the sums of a thread run in two lanes.
typedef unsigned long long F2;
__device__ __forceinline__ F2 pair(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(F2 v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// A 16-byte piece of a row in the form the sums take: its largest value, and its values two by two.
// With FINITE every value is raised to at least -2^100 (c x stays finite: a term 0 times its exponent
// is 0, not NaN); a NaN stays one.
template <typename T> struct Piece;
template <> struct Piece<__nv_bfloat16> {
    static constexpr int PAIRS = 4;
    uint4 v;
    __device__ __forceinline__ void fill() { v = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    __device__ __forceinline__ float largest() const {
        uint32_t a, b;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
        const float2 m = bf16_pair(a);
        return fmaxf(m.x, m.y);
    }
    // the largest value of four pieces
    static __device__ __forceinline__ float largest(const Piece (&x)[4]) {
        uint32_t m = x[0].v.x;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t w[4] = {x[u].v.x, x[u].v.y, x[u].v.z, x[u].v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(m), "r"(w[i]));
        }
        const float2 f = bf16_pair(m);
        return fmaxf(f.x, f.y);
    }
    template <bool FINITE> __device__ __forceinline__ float2 get(int i) const {
        uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
        if (FINITE)                                     // 0xf180: -2^100
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(w) : "r"(w), "r"(0xf180f180u));
        return bf16_pair(w);
    }
};
template <> struct Piece<float> {
    static constexpr int PAIRS = 2;
    float4 v;
    __device__ __forceinline__ void fill() {
        v.x = v.y = v.z = v.w = -CUDART_INF_F;
    }
    __device__ __forceinline__ float largest() const { return fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)); }
    static __device__ __forceinline__ float largest(const Piece (&x)[4]) {
        return fmaxf(fmaxf(x[0].largest(), x[1].largest()), fmaxf(x[2].largest(), x[3].largest()));
    }
    template <bool FINITE> __device__ __forceinline__ float2 get(int i) const {
        const float a = i ? v.z : v.x, b = i ? v.w : v.y;
        return FINITE ? make_float2(max_nan(a, -1.2676506e30f), max_nan(b, -1.2676506e30f))
                      : make_float2(a, b);
    }
};

struct RowSums {
    float M, top;
    F2 S, U;
};
// Moves the reference up to hold a value of c x = t.
__device__ __forceinline__ void move_ref(RowSums& a, float t) {
    const float m = rintf(t), d = a.M - m, f = ex2(d);
    float s0, s1, u0, u1;
    split(a.S, s0, s1);
    split(a.U, u0, u1);
    a.U = pair(f * (u0 + d * s0), f * (u1 + d * s1));
    a.S = pair(f * s0, f * s1);
    a.M = m;
}
template <bool ENT> __device__ __forceinline__ void add_terms(RowSums& a, F2 u) {
    float lo, hi;
    split(u, lo, hi);
    const F2 e = pair(ex2(lo), ex2(hi));
    a.S = add2(a.S, e);
    if (ENT) a.U = fma2(e, u, a.U);
}

// What the CTAs of one row leave in the first of them.
struct SplitPart {
    float top, S, U;
};

// One row per cluster of `split` CTAs (1 for a large batch); NT threads each.
template <typename T, bool ENT, bool TOP, int NT>
__global__ void __launch_bounds__(NT, logprob_ctas(NT))
logprob_kernel(const LogprobArgs a) {
    constexpr int N = Vec16<T>::N, W = NT / 32, UNROLL = 4;
    __shared__ float s_red[W][4];
    __shared__ SplitPart s_part[kMaxSplit];
    __shared__ Key s_keys[TOP ? W : 1][32];                    // a thread's bound; fallback: lists
    __shared__ Key s_cand[TOP ? kMaxCandidates : 1];
    __shared__ Key s_gather[TOP ? kMaxSplit * kMaxTop : 1];    // the CTAs' lists, in the first one
    __shared__ Key s_list[kMaxTop];
    __shared__ float s_slot[TOP ? kSlots * NT : 1];             // a thread's maxima over its rounds
    __shared__ uint32_t s_sel[TOP ? kMaxSelected : 1];          // slot and thread
    __shared__ int s_nsel, s_ncand;
    __shared__ Key s_bound;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / a.split, rank = blockIdx.x - row * a.split;

    const long long id = a.ids ? load_id(a.ids, a.id64, row) : 0;
    if (id < 0 || id >= a.V) {                          // the same decision in the whole cluster
        if (rank == 0) {
            if (tid == 0) {
                if (id >= a.V) report(a.dev_status, R3_DEV_BAD_INDEX);
                if (a.logp) a.logp[row] = 0.f;
                if (ENT) a.entropy[row] = 0.f;
                if (a.stats) a.stats[2 * (size_t)row] = a.stats[2 * (size_t)row + 1] = 0.f;
            }
            if (TOP && tid < a.n_top) {
                a.top_ids[(size_t)row * a.n_top + tid] = -1;
                a.top_logp[(size_t)row * a.n_top + tid] = 0.f;
            }
        }
        return;
    }
    // the CTAs of a cluster write to the first one's shared memory at the end: it has to be running
    if (a.split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");

    const T* p = static_cast<const T*>(a.logits) + (size_t)row * a.ld;
    const RowSplit rs = split_row(p, a.V);
    const Piece<T>* pv = reinterpret_cast<const Piece<T>*>(p + rs.head);
    const int per_cta = (rs.vecs + a.split - 1) / a.split;
    const int v0 = min(rs.vecs, rank * per_cta), v1 = min(rs.vecs, v0 + per_cta);
    const float c = a.c;

    RowSums r = {kLowRef, -CUDART_INF_F, 0, 0};
    int best_vec = v0 + tid < v1 ? v0 + tid : -1;       // the first piece that holds the top so far
    // UNROLL pieces per thread and round; the next round's are on their way while these are summed.  In
    // the last, ragged round the pieces behind the end read as -inf: they change neither the top nor the
    // sums, and a warp skips those that all of its lanes lack.
    const int rounds = (v1 - v0) / (UNROLL * NT);
    const int all_rounds = (v1 - v0 + UNROLL * NT - 1) / (UNROLL * NT);
    const int slot_rounds = max(1, (all_rounds + kSlots - 1) / kSlots);
    int slot = 0, in_slot = 0;
    float slot_top = -CUDART_INF_F;
    Piece<T> b[UNROLL];
    auto fetch = [&](int j) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) b[u] = pv[j + u * NT];
    };
    auto fetch_last = [&](int j) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (j + u * NT < v1) b[u] = pv[j + u * NT];
            else b[u].fill();
        }
    };
    auto sum = [&](const Piece<T>(&x)[UNROLL], int j, bool last) {
        float m = -CUDART_INF_F;
        if (TOP) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const float q = x[u].largest();
                if (q > fmaxf(r.top, m)) best_vec = j + u * NT;
                m = fmaxf(m, q);
            }
            slot_top = fmaxf(slot_top, m);
            if (++in_slot == slot_rounds || last) {
                s_slot[slot * NT + tid] = slot_top;
                ++slot;
                in_slot = 0;
                slot_top = -CUDART_INF_F;
            }
        } else {
            m = Piece<T>::largest(x);
        }
        r.top = fmaxf(r.top, m);
        if (m * c - r.M > kMoveRef) move_ref(r, m * c);
        const F2 c2 = pair(c, c), ref = pair(-r.M, -r.M);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (last && j - lane + u * NT >= v1) break;
#pragma unroll
            for (int i = 0; i < Piece<T>::PAIRS; ++i) {
                const float2 f = x[u].template get<ENT>(i);
                add_terms<ENT>(r, fma2(pair(f.x, f.y), c2, ref));
            }
        }
    };
    int j = v0 + tid;
    if (rounds > 0) fetch(j);
    else fetch_last(j);
    for (int k = 0; k < rounds; ++k) {
        Piece<T> x[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) x[u] = b[u];
        if (k + 1 < rounds) fetch(j + UNROLL * NT);
        else fetch_last(j + UNROLL * NT);
        sum(x, j, false);
        j += UNROLL * NT;
    }
    if (j - tid < v1) sum(b, j, true);
    if (TOP && in_slot > 0) s_slot[slot++ * NT + tid] = slot_top;
    // the single elements in front of the first and behind the last whole piece
    const bool has_head = rank == 0, has_tail = rank == a.split - 1;
    const int tail0 = rs.head + rs.vecs * N;
    auto take_one = [&](float x) {
        r.top = fmaxf(r.top, x);
        if (x * c - r.M > kMoveRef) move_ref(r, x * c);
        // a term 0 beside it (2^-3e38 and 0 times that)
        add_terms<ENT>(r, pair(fmaf(max_nan(x, -1.2676506e30f), c, -r.M), -3e38f));
    };
    const float vec_top = r.top;                        // of the whole pieces alone
    if (has_head && tid < rs.head) take_one(to_f32(p[tid]));
    if (has_tail && tid < rs.tail) take_one(to_f32(p[tail0 + tid]));

    // ---- the CTA's maximum and sums, relative to its own top -------------------------------
    float m = r.M, top = r.top;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    }
    if (lane == 0) {
        s_red[warp][0] = m;
        s_red[warp][1] = top;
    }
    const int first = rs.head + best_vec * N;           // first column of the thread's best piece
    if (TOP) {
        s_keys[warp][lane] = best_vec >= 0 ? make_key(vec_top, first + N - 1) : 0;
        if (tid == 0) s_nsel = s_ncand = 0;
        if (tid < kMaxTop) s_list[tid] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
        m = fmaxf(m, s_red[w][0]);
        top = fmaxf(top, s_red[w][1]);
    }
    float tS, tU;                                       // this thread's sums
    {
        float s0, s1, u0, u1;
        split(r.S, s0, s1);
        split(r.U, u0, u1);
        tS = s0 + s1;
        tU = u0 + u1;
    }
    // A top whose c x is beyond 2^20 (masks of the type's lowest value in a whole row, say) leaves
    // the reference no room: the share is summed again with the differences to the known top.
    const bool again = fabsf(top * c) > kPlainTop && fabsf(top) < CUDART_INF_F;
    if (again) {
        tS = tU = 0.f;
        auto term = [&](float x) {                      // x - top keeps a NaN
            const float u = max_nan((x - top) * c, kLeastExp), e = ex2(u);
            tS += e;
            tU = fmaf(e, u, tU);
        };
        const Vec16<T>* px = reinterpret_cast<const Vec16<T>*>(pv);
        for (int q = v0 + tid; q < v1; q += NT) {
            float x[N];
            px[q].unpack(x);
#pragma unroll
            for (int i = 0; i < N; ++i) term(x[i]);
        }
        if (has_head && tid < rs.head) term(to_f32(p[tid]));
        if (has_tail && tid < rs.tail) term(to_f32(p[tail0 + tid]));
    } else {
        const float d = r.M - m, f = ex2(d);
        tU = f * (tU + d * tS);
        tS *= f;
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
        tS += __shfl_xor_sync(0xffffffffu, tS, s);
        tU += __shfl_xor_sync(0xffffffffu, tU, s);
    }
    if (lane == 0) {
        s_red[warp][2] = tS;
        s_red[warp][3] = tU;
    }

    // ---- the largest keys of the CTA's share ---------------------------------------------------
    // Every thread knows its largest value and the 16-byte piece where that stood first, so (value,
    // last column of the piece) bounds its largest key from below.  The n-th largest of the 32
    // maxima of such bounds over equal lanes is reached by n keys of the share, so none of the n
    // largest lies under it; only threads whose piece reaches it (value, first column) hold keys
    // above it, and only their pieces are read again, from L2.  What reaches the bound are a few
    // more than n keys; each one's rank is the number of larger ones.  A thread keeps the maxima of runs of
    // its rounds in shared memory, so that of its pieces only the runs that reach the bound are read.
    Key list = 0;
    if (TOP) {
        if (warp == 0) {                                // alone: all warps at it cost more than the barrier
            Key g = s_keys[0][lane];
#pragma unroll
            for (int w = 1; w < W; ++w) g = s_keys[w][lane] > g ? s_keys[w][lane] : g;
            s_keys[0][lane] = g;
            __syncwarp();
            int larger = 0;
#pragma unroll
            for (int k = 0; k < 32; ++k) larger += s_keys[0][k] > g ? 1 : 0;
            const unsigned nth = __ballot_sync(0xffffffffu, larger == a.n_top - 1);
            // none: fewer than n threads have pieces, and everything is a candidate
            const Key n_th = __shfl_sync(0xffffffffu, g, nth ? __ffs(nth) - 1 : 0);
            if (lane == 0) s_bound = nth ? n_th : 0;
        }
        __syncthreads();
        const Key bound = s_bound;
        if (best_vec >= 0 && make_key(vec_top, first) >= bound) {
            const float least = bound ? key_value(bound) : -CUDART_INF_F;
            float tops[kSlots];
#pragma unroll
            for (int k = 0; k < kSlots; ++k) tops[k] = k < slot ? s_slot[k * NT + tid] : 0.f;
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                if (k >= slot || !(tops[k] >= least)) continue;
                const int at = atomicAdd(&s_nsel, 1);
                if (at < kMaxSelected) s_sel[at] = (uint32_t)(k << 16 | tid);
            }
        }
        __syncthreads();
        const Vec16<T>* px = reinterpret_cast<const Vec16<T>*>(pv);
        // the q-th piece of the selected runs (of all, where they are too many to list); v1: none
        const bool listed = s_nsel <= kMaxSelected;
        const int run = slot_rounds * UNROLL, total = listed ? s_nsel * run : v1 - v0;
        auto piece_at = [&](int q) {
            if (q >= total) return v1;
            if (!listed) return v0 + q;
            const int s = q / run, r = q - s * run;
            const uint32_t e = s_sel[s];
            return min(v1, v0 + (int)(e & 0xffffu) + ((int)(e >> 16) * run + r) * NT);
        };
        auto offer = [&](float x, int col) {            // any order: ranks do not depend on it
            const Key k = make_key(x, col);
            if (k < bound) return;
            const int at = atomicAdd(&s_ncand, 1);
            if (at < kMaxCandidates) s_cand[at] = k;
        };
        for (int q0 = tid; q0 < total; q0 += 4 * NT) {
            Vec16<T> piece[4];
            int at[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {               // four loads on their way at once
                at[u] = piece_at(q0 + u * NT);
                if (at[u] < v1) piece[u] = px[at[u]];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (at[u] >= v1) continue;
                float x[N];
                piece[u].unpack(x);
#pragma unroll
                for (int i = 0; i < N; ++i) offer(x[i], rs.head + at[u] * N + i);
            }
        }
        if (has_head && tid < rs.head) offer(to_f32(p[tid]), tid);
        if (has_tail && tid < rs.tail) offer(to_f32(p[tail0 + tid]), tail0 + tid);
        __syncthreads();
        const int found = s_ncand;
        if (found <= kMaxCandidates) {
            for (int i = tid; i < found; i += NT) {
                const Key k = s_cand[i];
                int above = 0;
#pragma unroll 8
                for (int q = 0; q < found; ++q) above += s_cand[q] > k ? 1 : 0;
                if (above < kMaxTop) s_list[above] = k;
            }
        } else {
            // many large values in the pieces of few threads: every warp keeps the 32 largest of the
            // keys it meets, and the warps' lists are merged
            for (int q0 = warp * 32; q0 < total; q0 += NT) {
                const int vec = piece_at(q0 + lane);
                float x[N];
                if (vec < v1) px[vec].unpack(x);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    Key k = vec < v1 ? make_key(x[i], rs.head + vec * N + i) : 0;
                    if (k < bound) k = 0;
                    if (__any_sync(0xffffffffu, k != 0)) list = warp_merge(list, warp_sort(k, lane), lane);
                }
            }
            if (warp == 0) {
                int col = -1;
                if (has_head && lane < rs.head) col = lane;
                if (has_tail && lane >= 16 && lane - 16 < rs.tail) col = tail0 + lane - 16;
                const Key k = col >= 0 ? make_key(to_f32(p[col]), col) : 0;
                list = warp_merge(list, warp_sort(k, lane), lane);
            }
            s_keys[warp][lane] = list;
#pragma unroll
            for (int half = W / 2; half > 0; half >>= 1) {
                __syncthreads();
                if (warp < half) {
                    list = warp_merge(list, s_keys[warp + half][lane], lane);
                    s_keys[warp][lane] = list;
                }
            }
            if (warp == 0) s_list[lane] = list;
        }
    }
    __syncthreads();                                    // s_red, s_list

    float S = 0.f, U = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {                                        // fixed order
        S += s_red[w][2];
        U += s_red[w][3];
    }
    if (!again && top > -CUDART_INF_F) {
        const float ut = fmaf(top, c, -m), k = ex2(-ut);
        U = k * (U - ut * S);
        S *= k;
    }
    if (TOP) list = s_list[lane];

    // ---- the CTAs of a row meet in the first of them ------------------------------------------
    if (a.split > 1) {
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (warp == 0) {
            if (lane < 3) {
                const uint32_t at = tc::mapa_shared(tc::smem_u32(&s_part[rank]), 0) + 4 * lane;
                const float v = lane == 0 ? top : lane == 1 ? S : U;
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
            }
            if (TOP && lane < a.n_top) {
                const uint32_t at = tc::mapa_shared(tc::smem_u32(&s_gather[TOP ? rank * a.n_top + lane : 0]), 0);
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(list) : "memory");
            }
        }
        tc::cluster_sync_all();
        if (rank != 0) return;                          // nobody reads this CTA's memory
        if (TOP) {
            const int found = a.split * a.n_top;        // zeros where a share has fewer keys
            for (int i = tid; i < found; i += NT) {
                const Key k = s_gather[i];
                int above = 0;
#pragma unroll 8
                for (int q = 0; q < found; ++q) above += s_gather[q] > k ? 1 : 0;
                if (k != 0 && above < kMaxTop) s_list[above] = k;
            }
            __syncthreads();
            list = s_list[lane];
        }
        if (warp != 0) return;
        float t = -CUDART_INF_F, ts = 0.f, tu = 0.f;
        if (lane < a.split) {
            t = s_part[lane].top;
            ts = s_part[lane].S;
            tu = s_part[lane].U;
        }
        top = t;
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        // a share of -inf alone has S = 0 (or NaN, which stays)
        const float d = t > -CUDART_INF_F ? max_nan((t - top) * c, -1e30f) : 0.f;
        const float f = ex2(d);
        U = f * (tu + d * ts);
        S = f * ts;
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) {
            S += __shfl_xor_sync(0xffffffffu, S, s);
            U += __shfl_xor_sync(0xffffffffu, U, s);
        }
    }
    if (warp != 0) return;

    const bool bad = !(S < CUDART_INF_F);                       // NaN or +inf among the logits
    const bool none = !bad && top == -CUDART_INF_F;             // every logit -inf
    float ln_s = none ? 0.f : logf(S);
    if (ln_s < 0.f) ln_s = 0.f;                                 // S holds the top's own term, 1
    if (bad) top = ln_s = CUDART_NAN_F;
    auto logp_of = [&](float x) { return none ? -CUDART_INF_F : (x - top) * a.inv_t - ln_s; };
    if (lane == 0) {
        if (a.logp) a.logp[row] = logp_of(to_f32(p[id]));
        if (ENT) {
            const float h = none ? 0.f : bad ? CUDART_NAN_F : ln_s - CUDART_LN2_F * (U / S);
            a.entropy[row] = h < 0.f ? 0.f : h;
        }
        if (a.stats) {
            a.stats[2 * (size_t)row] = top;
            a.stats[2 * (size_t)row + 1] = ln_s;
        }
    }
    if (TOP && lane < a.n_top) {
        a.top_ids[(size_t)row * a.n_top + lane] = bad ? -1 : key_column(list);
        a.top_logp[(size_t)row * a.n_top + lane] = logp_of(key_value(list));
    }
}

// ---- gradient to the logits ----------------------------------------------------------------------
struct LogprobBwdArgs {
    const void* logits;
    const void* ids;
    const float* stats;
    const float* entropy;
    const float* dlogp;
    const float* dentropy;
    void* dlogits;
    long long ld, ld_out;
    int T, V, id64, chunks;
    float c, inv_t;
    int32_t* dev_status;
};

constexpr int kBwdThreads = 256;
constexpr int kBwdVecs = 4;            // 16-byte pieces per thread

// d logits[v] = (dlogp (1[v = id] - p_v) - dentropy p_v (log p_v + H)) / temperature.  Element by
// element once the row's two sums are known; logits and dlogits may be the same buffer (each thread
// reads its elements before it writes them).  Bound by HBM: every logit is read and written once
// (8192 x 151936 bf16 with a tenth of the rows skipped: 742 us = 97% of the measured copy bandwidth).  A
// CTA takes 16 KB of one row: many more CTAs than are resident, so that SMs which see the memory
// slower take fewer.
template <typename T, bool ENT>
__global__ void __launch_bounds__(kBwdThreads) logprob_bwd_kernel(const LogprobBwdArgs a) {
    constexpr int N = Vec16<T>::N, STEP = kBwdThreads * kBwdVecs;
    const long long items = (long long)a.T * a.chunks;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int row = (int)(item / a.chunks), chunk = (int)(item - (long long)row * a.chunks);
        const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.ld;
        T* dx = static_cast<T*>(a.dlogits) + (size_t)row * a.ld_out;
        const long long id = a.ids ? load_id(a.ids, a.id64, row) : 0;
        const bool skip = id < 0 || id >= a.V;
        if (id >= a.V && chunk == 0 && threadIdx.x == 0) report(a.dev_status, R3_DEV_BAD_INDEX);
        const float top = a.stats[2 * (size_t)row], ln_s = a.stats[2 * (size_t)row + 1];
        const bool zero = skip || top == -CUDART_INF_F;
        const float g = a.dlogp ? a.dlogp[row] * a.inv_t : 0.f;
        const float ge = ENT ? a.dentropy[row] * a.inv_t : 0.f;
        const float h = ENT ? a.entropy[row] : 0.f;
        const float ls2 = ln_s * CUDART_L2E_F, c = a.c;
        const int target = a.dlogp && !skip ? (int)id : -1;
        auto grad = [&](float v, int col) {
            float u = fmaf(v - top, c, -ls2);
            float k = -g;
            if (ENT) {
                u = max_nan(u, kLeastExp);
                k -= ge * fmaf(u, CUDART_LN2_F, h);
            }
            float d = ex2(u) * k;
            if (col == target) d += g;
            return d;
        };
        const RowSplit rs = split_row(dx, a.V);
        // the wide form needs both rows to start at the same place of a 16-byte piece
        const bool wide =
            ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 15u) == 0;
        if (wide) {
            const Vec16<T>* xv = reinterpret_cast<const Vec16<T>*>(x + rs.head);
            Vec16<T>* dv = reinterpret_cast<Vec16<T>*>(dx + rs.head);
            const int first = chunk * STEP + threadIdx.x;
            Vec16<T> b[kBwdVecs];
            if (!zero) {
#pragma unroll
                for (int q = 0; q < kBwdVecs; ++q)
                    if (first + q * kBwdThreads < rs.vecs) b[q] = xv[first + q * kBwdThreads];
            }
#pragma unroll
            for (int q = 0; q < kBwdVecs; ++q) {
                const int j = first + q * kBwdThreads;
                if (j >= rs.vecs) break;
                float f[N];
                if (zero) {
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] = 0.f;
                } else {
                    b[q].unpack(f);
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] = grad(f[i], rs.head + j * N + i);
                }
                Vec16<T> o;
                o.pack(f);
                dv[j] = o;
            }
        } else {
            // Whole pieces of dx; each is made of two neighbouring pieces of x, shifted by the same
            // number of bytes throughout the row.  The row's first and last piece are read element by
            // element: their neighbours may lie outside the row.
            const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(x + rs.head) & 15u);
            const uint4* xv = reinterpret_cast<const uint4*>(
                reinterpret_cast<const char*>(x + rs.head) - off);
            Vec16<T>* dv = reinterpret_cast<Vec16<T>*>(dx + rs.head);
#pragma unroll 1
            for (int q = 0; q < kBwdVecs; ++q) {
                const int j = chunk * STEP + threadIdx.x + q * kBwdThreads;
                if (j >= rs.vecs) break;
                const int col = rs.head + j * N;
                float f[N];
                if (zero) {
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] = 0.f;
                } else {
                    if (j == 0 || j == rs.vecs - 1) {
#pragma unroll
                        for (int i = 0; i < N; ++i) f[i] = to_f32(x[col + i]);
                    } else {
                        const uint4 lo = xv[j], hi = xv[j + 1];
                        Vec16<T> v;
                        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
                        const uint32_t bits = 8u * (off & 3u);
                        auto shift = [&](uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t w4) {
                            w[0] = __funnelshift_r(w0, w1, bits);
                            w[1] = __funnelshift_r(w1, w2, bits);
                            w[2] = __funnelshift_r(w2, w3, bits);
                            w[3] = __funnelshift_r(w3, w4, bits);
                        };
                        if (off < 4) shift(lo.x, lo.y, lo.z, lo.w, hi.x);
                        else if (off < 8) shift(lo.y, lo.z, lo.w, hi.x, hi.y);
                        else if (off < 12) shift(lo.z, lo.w, hi.x, hi.y, hi.z);
                        else shift(lo.w, hi.x, hi.y, hi.z, hi.w);
                        v.unpack(f);
                    }
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] = grad(f[i], col + i);
                }
                Vec16<T> o;
                o.pack(f);
                dv[j] = o;
            }
        }
        if (chunk == 0) {
            const int tail0 = rs.head + rs.vecs * N, t = threadIdx.x;
            const int col = t < rs.head ? t : t >= 32 && t - 32 < rs.tail ? tail0 + t - 32 : -1;
            if (col >= 0) dx[col] = from_f32<T>(zero ? 0.f : grad(to_f32(x[col]), col));
        }
    }
}

// ---- host side ------------------------------------------------------------------------------------
static bool words_aligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (!aligned(p, 4)) return false;
    return true;
}
static r3_status check_logits(const r3_logits* s) {
    if (!s) return R3_ERR_INVALID_ARG;
    if (s->T < 0 || s->T > 0x7f000000 || s->V <= 0 || s->V > (1 << 30) || s->ld < s->V) return R3_ERR_INVALID_ARG;
    if (s->dtype != R3_F32 && s->dtype != R3_BF16) return R3_ERR_INVALID_ARG;
    if (s->id_bytes != 4 && s->id_bytes != 8) return R3_ERR_INVALID_ARG;
    // -2^100, which stands for -inf in the sums, times log2(e) / temperature is finite and far below any
    // exponent that counts
    if (!(s->temperature >= 1e-6 && s->temperature <= 1e20))
        return R3_ERR_INVALID_ARG;
    return R3_OK;
}

template <typename T, bool ENT, bool TOP, int NT>
static r3_status launch_logprob(const LogprobArgs& a, cudaStream_t cs) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3((unsigned)((long long)a.T * a.split));
    cfg.blockDim = dim3(NT);
    cfg.stream = cs;
    if (a.split > 1) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)a.split;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    if (cudaLaunchKernelEx(&cfg, logprob_kernel<T, ENT, TOP, NT>, a) != cudaSuccess) {
        cudaGetLastError();
        return R3_ERR_CUDA;
    }
    return R3_OK;
}

template <typename T, int NT> static r3_status dispatch_logprob(const LogprobArgs& a, cudaStream_t cs) {
    if (a.entropy)
        return a.n_top ? launch_logprob<T, true, true, NT>(a, cs)
                       : launch_logprob<T, true, false, NT>(a, cs);
    return a.n_top ? launch_logprob<T, false, true, NT>(a, cs)
                   : launch_logprob<T, false, false, NT>(a, cs);
}

}  // namespace r3

extern "C" r3_status r3_token_logprobs(const r3_logits* shape, const void* logits,
                                       const void* token_ids, float* logp, float* entropy,
                                       float* stats, int32_t n_top, int32_t* top_ids,
                                       float* top_logp, int32_t* dev_status, void* stream) {
    const r3_status st = r3::check_logits(shape);
    if (st != R3_OK) return st;
    if (n_top < 0 || n_top > shape->V) return R3_ERR_INVALID_ARG;
    if (n_top > r3::kMaxTop) return R3_ERR_UNSUPPORTED;
    if (shape->T == 0) return R3_OK;
    const size_t es = shape->dtype == R3_BF16 ? 2 : 4;
    if (!logits || !r3::aligned(logits, es) || (logp && !token_ids) ||
        (n_top > 0 && (!top_ids || !top_logp)) || (!logp && !entropy && !stats && n_top == 0) ||
        (token_ids && !r3::aligned(token_ids, (size_t)shape->id_bytes)) ||
        !r3::words_aligned({logp, entropy, stats, top_ids, top_logp, dev_status}))
        return R3_ERR_INVALID_ARG;
    r3::LogprobArgs a = {};
    a.logits = logits;
    a.ids = token_ids;
    a.ld = shape->ld;
    a.T = shape->T;
    a.V = shape->V;
    a.id64 = shape->id_bytes == 8;
    a.n_top = n_top;
    a.c = (float)(1.4426950408889634 / shape->temperature);
    a.inv_t = (float)(1.0 / shape->temperature);
    a.logp = logp;
    a.entropy = entropy;
    a.stats = stats;
    a.top_ids = top_ids;
    a.top_logp = top_logp;
    a.dev_status = dev_status;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    const long long row_bytes = (long long)shape->V * (long long)es;
    // Threads per row: with more than its pieces keep busy the reductions at a row's end cost more than
    // its loads, and many small CTAs on an SM end at different times, which keeps the loads flowing
    // (8192 rows of bf16: 6000 columns 30.8 us at 128 threads, 25.6 at 32; 12000 columns 59.4 at 256,
    // 44.3 at 128; 151936 columns with 5 alternatives 427 at 256, 418 at 128).  Long rows that are few enough
    // for whole waves to count: 256 threads where those take less of them, a wave of 128 holding twice the
    // rows and lasting twice as long (50257 columns of float32 with 5 alternatives: 300 rows 18.5 at 256,
    // 24.6 at 128; 600 rows 36.9 and 30.3; 900 41.0 and 36.8; 1200 57.4 and 59.5; 2048 82.5 and 75.6).
    auto waves = [&](int nt) {
        const int resident = r3::logprob_ctas(nt) * r3::sm_count();
        return (a.T + resident - 1) / resident;
    };
    const int threads = row_bytes <= 16384                                ? 32
                        : row_bytes <= 49152                              ? 128
                        : waves(128) <= 4 && waves(256) < 2 * waves(128) ? 256
                                                                          : 128;
    // Few rows: a cluster of CTAs shares one, as long as each has an SM of its own and a thread two pieces
    // or more.
    a.split = 1;
    while (a.split < r3::kMaxSplit && (long long)a.T * a.split <= r3::sm_count() &&
           row_bytes / (a.split * 2) >= 2LL * 16 * threads)
        a.split *= 2;
    auto launch = [&](auto type) {
        using T = decltype(type);
        return threads == 32    ? r3::dispatch_logprob<T, 32>(a, cs)
               : threads == 128 ? r3::dispatch_logprob<T, 128>(a, cs)
                                : r3::dispatch_logprob<T, 256>(a, cs);
    };
    return shape->dtype == R3_BF16 ? launch(__nv_bfloat16()) : launch(float());
}

extern "C" r3_status r3_token_logprobs_bwd(const r3_logits* shape, const void* logits,
                                           const void* token_ids, const float* stats,
                                           const float* entropy, const float* dlogp,
                                           const float* dentropy, void* dlogits, int64_t ld_out,
                                           int32_t* dev_status, void* stream) {
    const r3_status st = r3::check_logits(shape);
    if (st != R3_OK) return st;
    if (ld_out < shape->V) return R3_ERR_INVALID_ARG;
    if (shape->T == 0) return R3_OK;
    const size_t es = shape->dtype == R3_BF16 ? 2 : 4;
    if (!logits || !r3::aligned(logits, es) || !dlogits || !r3::aligned(dlogits, es) || !stats ||
        (!dlogp && !dentropy) || (dlogp && !token_ids) || (dentropy && !entropy) ||
        (dlogits == logits && ld_out != shape->ld) ||
        (token_ids && !r3::aligned(token_ids, (size_t)shape->id_bytes)) ||
        !r3::words_aligned({stats, entropy, dlogp, dentropy, dev_status}))
        return R3_ERR_INVALID_ARG;
    r3::LogprobBwdArgs a = {};
    a.logits = logits;
    a.ids = token_ids;
    a.stats = stats;
    a.entropy = entropy;
    a.dlogp = dlogp;
    a.dentropy = dentropy;
    a.dlogits = dlogits;
    a.ld = shape->ld;
    a.ld_out = ld_out;
    a.T = shape->T;
    a.V = shape->V;
    a.id64 = shape->id_bytes == 8;
    a.c = (float)(1.4426950408889634 / shape->temperature);
    a.inv_t = (float)(1.0 / shape->temperature);
    a.dev_status = dev_status;
    const int step = r3::kBwdThreads * r3::kBwdVecs * (int)(16 / es);
    a.chunks = (shape->V + step - 1) / step;
    const long long items = (long long)a.T * a.chunks;
    const unsigned grid = (unsigned)(items < 0x7fffffffLL ? items : 0x7fffffffLL);
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (shape->dtype == R3_BF16) {
        if (dentropy)
            r3::logprob_bwd_kernel<__nv_bfloat16, true><<<grid, r3::kBwdThreads, 0, cs>>>(a);
        else
            r3::logprob_bwd_kernel<__nv_bfloat16, false><<<grid, r3::kBwdThreads, 0, cs>>>(a);
    } else {
        if (dentropy) r3::logprob_bwd_kernel<float, true><<<grid, r3::kBwdThreads, 0, cs>>>(a);
        else r3::logprob_bwd_kernel<float, false><<<grid, r3::kBwdThreads, 0, cs>>>(a);
    }
    return r3::launch_status();
}
