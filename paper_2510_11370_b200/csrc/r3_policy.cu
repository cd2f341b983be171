// Clipped policy loss over packed responses, with its gradient to the log probabilities and the
// entropies: what stands between the log probabilities of given tokens and their gradient.  Per
// response token t of sequence i, all from log probabilities,
//   d     = logp - logp_old               (ratio of sequences: its mean over the sequence's tokens)
//   rho   = exp(d)       w = min(exp(logp_old - logp_infer), cap)
//   term  = -w min(rho A, clip(rho) A)    and at most w c |A| for A < 0 with a dual clip c
//   kl    = exp(x) - 1 - x,  x = logp_ref - logp
//   loss  = sum_t weight_t (term + kl_coef kl - entropy_coef entropy)
// with weight 1 / N (tokens) or 1 / (n_i S') (sequences).  Whether a ratio lies beyond a border is asked
// of its logarithm, in 64 bits (the difference of two float32 numbers is exact there), so the choice does
// not depend on how an exponential rounds; exponentials and the terms are float32, all sums 64 bits.
//
// Two passes, since a token's gradient needs its sequence's sums and the number of tokens: the first
// leaves the sums of every unit (up to U = 128 consecutive tokens of ONE sequence, more in a large batch, a
// warp each), the second adds up a sequence's units in their order and writes the gradients; its last CTA
// adds up the CTAs' parts of the loss.  With a ratio per sequence the units' sums say all about the tokens'
// terms, and where there is no KL term and no entropy the second pass reads the mask alone (1 M tokens 29 -> 22 us).  Sequence i that starts at token c takes its units from number
// i + floor(c / U) on: that leaves each one room for all of its units whatever the lengths are, and a warp of
// the first pass finds its sequence by a search in cu_seqlens, 32 probes at a time, with no table built
// before.  Batches of up to 32 units run as one CTA.
// Bound by latency throughout: 1531 tokens in one launch 6 us, 65536 tokens with every term 10 us, 1 M tokens of
// 1024 sequences 22 us, against 2.6 us for their bytes; of those 22 the first pass takes 9, the second's start (its
// counts, its sequences' sums) 3, its tokens 2, the parts of the loss 4.
#include <cmath>

#include "r3_common.cuh"
#include "r3_internal.h"
#include "r3_tc.cuh"

namespace r3 {
namespace pol {

// Tokens of a lane at a time: the second pass has too much code per token to stand there more than once (code
// comes from memory too at every launch: four tokens at a time took 13.7 us for 65536 tokens, one 10.6).
constexpr int AHEAD = 4;                  // in the first pass
constexpr int MARKS = 16, PROBES = 32;    // of the mask, where nothing else is read
constexpr int LEAST_SHIFT = 7;            // tokens of a unit, at least: 128 (256: 1531 tokens 8.1 instead of 6.1 us)
constexpr int MOST_UNITS = 2048;          // of one sequence: beyond, units grow
constexpr int LONG = 64;                  // units from which a sequence is added up in BLOCKS blocks
constexpr int BLOCKS = 8;
constexpr int WARPS = 8;                  // units of a CTA
constexpr int CTAS_PER_SM = 4;
constexpr int ONE_WARPS = 32;             // units of a batch that takes one CTA

struct Sums {                             // of one unit; of a sequence: the sum of its units'
    double d, up, down;                   // sum of d; of w A over the tokens with A > 0 and A < 0
};
struct Marks {                            // of a unit, where ratios are of sequences
    int up, down, cut, pad;               // tokens with A > 0, with A < 0, with w at the cap
};
struct Total {
    double policy, kl, entropy;
    int tokens, clipped, cut, pad;
};
struct Args {
    int T, S, units, shift;                            // 1 << shift tokens per unit
    int by_sequence, mean_of_sequences, adv_per_token, need_sums;
    double log_high, log_low, log_dual, log_cap;       // borders of d and of logp_old - logp_infer
    float high, low, dual, cap;                        // the values beyond them
    double kl_coef, entropy_coef, denominator;         // denominator 0: counted
    const float *logp, *old, *adv, *infer, *ref, *entropy, *dloss;
    const int32_t* cu;                                 // or null: one sequence
    const uint8_t* mask;
    float *loss, *dlogp, *dentropy, *metrics;
    int32_t* counts;
    Sums* sums;                                        // [units]
    Marks* marks;                                      // [units]
    int* n;                                            // [units] tokens
    int* head;                                         // [units] 1: the first unit of a sequence with tokens
    Total* totals;                                     // [CTAs]
    unsigned* ticket;
    int32_t* dev_status;
};

__device__ __forceinline__ int bound(const Args& a, int i) {       // where sequence i starts
    if (!a.cu) return i == 0 ? 0 : a.T;
    return min(max(a.cu[i], 0), a.T);
}
__device__ __forceinline__ int first_unit(const Args& a, int i) { return i + (bound(a, i) >> a.shift); }

struct Unit {
    int seq, begin, end;                  // seq = S: behind the last sequence
    int first, count;                     // units of the sequence
};
// The whole warp; the last sequence whose first unit is not behind `unit`.
__device__ __forceinline__ Unit find_unit(const Args& a, int unit) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = a.S + 1;            // first_unit(lo) <= unit always holds: unit 0 is sequence 0's
    while (len > 1) {
        const int step = (len + 31) / 32, at = lo + lane * step;
        const bool in = lane * step < len && first_unit(a, at) <= unit;
        const int k = max(__popc(__ballot_sync(0xffffffffu, in)) - 1, 0);
        lo += k * step;
        len = min(step, len - k * step);
    }
    Unit u;
    u.seq = lo;
    const int begin = bound(a, lo), end = lo < a.S ? max(bound(a, lo + 1), begin) : a.T;
    u.first = lo + (begin >> a.shift);
    u.count = (int)(((long long)end - begin + (1 << a.shift) - 1) >> a.shift);
    const long long at = begin + ((long long)(unit - u.first) << a.shift);
    u.begin = (int)min(at, (long long)end);
    u.end = (int)min((long long)u.begin + (1 << a.shift), (long long)end);
    return u;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ int warp_sum(int v) { return __reduce_add_sync(0xffffffffu, v); }

// min(exp(old - infer), cap)
__device__ __forceinline__ float infer_weight(const Args& a, float old, float infer, bool* cut) {
    const double x = (double)old - (double)infer;
    *cut = x > a.log_cap;
    return *cut ? a.cap : expf((float)x);
}

// ---- first pass: the sums of a unit ----------------------------------------------------------
__device__ __forceinline__ void unit_sums(const Args& a, const Unit& u, int unit, Sums* s, Marks* marks, int* n,
                                          int* head) {
    const int lane = threadIdx.x & 31;
    const bool live = u.seq < a.S;
    double d = 0.0, up = 0.0, down = 0.0;
    int k = 0, ups = 0, downs = 0, cuts = 0;
    if (live && !a.by_sequence && !a.mask) {
        if (lane == 0) k = u.end - u.begin;
    } else if (live) {
        const float seq_adv = a.by_sequence && !a.adv_per_token && u.begin < u.end ? a.adv[u.seq] : 0.f;
        struct Token {
            float logp, old, infer, adv;
            bool on;
        };
        auto load = [&](int t0, Token (&x)[AHEAD]) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int t = t0 + j * 32;
                x[j].on = t < u.end;
                if (a.by_sequence) {                       // (not behind the mask's arrival)
                    x[j].logp = x[j].on ? a.logp[t] : 0.f;
                    x[j].old = x[j].on ? a.old[t] : 0.f;
                    x[j].infer = x[j].on && a.infer ? a.infer[t] : 0.f;
                    x[j].adv = x[j].on ? (a.adv_per_token ? a.adv[t] : seq_adv) : 0.f;
                }
                if (a.mask && x[j].on) x[j].on = a.mask[t] != 0;
            }
        };
        Token next[AHEAD];
        load(u.begin + lane, next);
#pragma unroll 1
        for (int t0 = u.begin + lane; t0 - lane < u.end; t0 += 32 * AHEAD) {
            Token x[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) x[j] = next[j];
            load(t0 + 32 * AHEAD, next);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                k += x[j].on;
                if (!a.by_sequence || !x[j].on) continue;
                d += (double)x[j].logp - (double)x[j].old;
                bool cut = false;
                const float w = a.infer ? infer_weight(a, x[j].old, x[j].infer, &cut) : 1.f;
                const double wa = (double)(w * x[j].adv);
                if (x[j].adv > 0.f) up += wa;
                else if (x[j].adv != 0.f) down += wa;      // NaN counts here: it has to reach the loss
                ups += x[j].adv > 0.f;
                downs += x[j].adv < 0.f;
                cuts += cut;
            }
        }
    }
    k = warp_sum(k);
    int any = 0;
    if (a.mean_of_sequences && live && unit == u.first && u.count > 0) {
        // does the sequence hold a token at all: mostly its first unit says so
        any = k > 0;
        const int seq_end = bound(a, u.seq + 1);
        for (int t = u.end; !any && t < seq_end; t += 32 * PROBES) {
            int here = 0;
#pragma unroll
            for (int j = 0; j < PROBES; ++j) {
                const int at = t + j * 32 + lane;
                here |= at < seq_end && a.mask[at];        // without a mask the first unit has tokens
            }
            any = __any_sync(0xffffffffu, here);
        }
    }
    if (a.by_sequence) {
        d = warp_sum(d);
        up = warp_sum(up);
        down = warp_sum(down);
        ups = warp_sum(ups);
        downs = warp_sum(downs);
        cuts = warp_sum(cuts);
    }
    if (lane == 0) {
        *n = k;
        *head = any;
        if (a.by_sequence) {
            *s = {d, up, down};
            *marks = {ups, downs, cuts, 0};
        }
    }
}

// Sums of the units [first, first + count), by a whole warp.
struct Whole {
    Sums s;
    int tokens;
};
__device__ __forceinline__ Whole add_units(const Args& a, const Sums* sums, const int* n, int first, int count) {
    const int lane = threadIdx.x & 31;
    Whole w = {};
#pragma unroll 4
    for (int i = lane; i < count; i += 32) {
        w.tokens += n[first + i];
        if (a.by_sequence) {
            const Sums v = sums[first + i];
            w.s.d += v.d;
            w.s.up += v.up;
            w.s.down += v.down;
        }
    }
    w.tokens = warp_sum(w.tokens);
    if (a.by_sequence) w.s = {warp_sum(w.s.d), warp_sum(w.s.up), warp_sum(w.s.down)};
    return w;
}
__device__ __forceinline__ Whole add_block(const Args& a, const Sums* sums, const int* n, int first, int count,
                                           int block) {
    const int size = (count + BLOCKS - 1) / BLOCKS, from = min(count, block * size);
    return add_units(a, sums, n, first + from, min(size, count - from));
}
__device__ __forceinline__ void add(Whole& x, const Whole& y) {
    x.s.d += y.s.d;
    x.s.up += y.s.up;
    x.s.down += y.s.down;
    x.tokens += y.tokens;
}
// A sequence's sums by one warp: in the same order as by the warps of a CTA (below).
__device__ __forceinline__ Whole sequence_sums(const Args& a, const Sums* sums, const int* n, int first, int count) {
    if (count <= LONG) return add_units(a, sums, n, first, count);
    Whole w = {};
    for (int b = 0; b < BLOCKS; ++b) add(w, add_block(a, sums, n, first, count, b));
    return w;
}

// exp(x) - 1 - x without cancellation: its series up to |x| = 1 (the first term left out, 2 / 13! of
// the result, is below a rounding).
__device__ __forceinline__ float exp_less_line(float x, float em1) {
    if (!(fabsf(x) <= 1.f)) return em1 - x;
    float p = 1.f + x * (1.f / 12.f);
#pragma unroll
    for (int k = 11; k >= 3; --k) p = 1.f + x * p * (1.f / (float)k);
    return 0.5f * x * x * p;
}

// ---- second pass: one unit's part of the loss, and its gradients ------------------------------
// `s`, n_seq: of the unit's sequence; `sums`, `marks`, `n`: the unit's own, which are all that a ratio of the whole
// sequence leaves to know of the tokens' terms (they are not read again).
__device__ __forceinline__ Total unit_loss(const Args& a, const Unit& u, const Sums& s, int n_seq, double divisor,
                                           const Sums* sums, const Marks* marks, const int* n) {
    const int lane = threadIdx.x & 31;
    Total r = {};
    const bool live = u.seq < a.S;
    double weight = 0.0;
    if (live) weight = 1.0 / (a.mean_of_sequences ? divisor * (double)max(n_seq, 1) : divisor);
    const float up_to = a.dloss ? a.dloss[0] : 1.f;            // gradient of the loss itself
    const float gw = (float)(weight * (double)up_to);
    const float kl_w = (float)(a.kl_coef * weight * (double)up_to);
    const float ent_g = (float)(-a.entropy_coef * weight * (double)up_to);
    const float seq_adv = live && !a.by_sequence && !a.adv_per_token && u.begin < u.end ? a.adv[u.seq] : 0.f;
    float seq_slope = 0.f;
    if (a.by_sequence && live) {
        const double seq_d = s.d / (double)max(n_seq, 1);
        const double rho = (double)expf((float)seq_d);
        const bool high = seq_d > a.log_high, low = seq_d < a.log_low || seq_d > a.log_dual;
        // a part that is 0 takes no ratio, be it infinite
        const double part = (high ? 0.0 : s.up) + (low ? 0.0 : s.down);
        if (lane == 0) {
            const double rho_down = seq_d < a.log_low ? (double)a.low : low ? (double)a.dual : rho;
            if (sums->up != 0.0) r.policy -= sums->up * (high ? (double)a.high : rho);
            if (sums->down != 0.0) r.policy -= sums->down * rho_down;
            r.tokens = *n;
            r.clipped = (high ? marks->up : 0) + (low ? marks->down : 0);
            r.cut = marks->cut;
        }
        seq_slope = part == 0.0 ? 0.f
                                : (float)(-part * rho * weight * (double)up_to / (double)max(n_seq, 1));
    }
    const bool terms = !a.by_sequence;
    if (a.by_sequence && !a.ref && !a.entropy) {
        // the same gradient for every token that counts
        for (int t0 = u.begin + lane; a.dlogp && t0 - lane < u.end; t0 += 32 * MARKS) {
            bool on[MARKS];
#pragma unroll
            for (int j = 0; j < MARKS; ++j)
                on[j] = live && t0 + 32 * j < u.end && (!a.mask || a.mask[t0 + 32 * j]);
#pragma unroll
            for (int j = 0; j < MARKS; ++j)
                if (t0 + 32 * j < u.end) a.dlogp[t0 + 32 * j] = on[j] ? seq_slope : 0.f;
        }
        r.policy *= weight;
        return r;
    }
    struct Token {
        float logp, old, infer, ref, entropy, adv;
        bool on;
    };
    auto load = [&](int t, Token& x) {
        const bool on = live && t < u.end;
        x.logp = on && (terms || a.ref) ? a.logp[t] : 0.f;
        x.old = on && terms ? a.old[t] : 0.f;
        x.infer = on && terms && a.infer ? a.infer[t] : 0.f;
        x.ref = on && a.ref ? a.ref[t] : 0.f;
        x.entropy = on && a.entropy ? a.entropy[t] : 0.f;
        x.adv = on && terms ? (a.adv_per_token ? a.adv[t] : seq_adv) : 0.f;
        x.on = on && (!a.mask || a.mask[t]);
    };
    Token next;
    load(u.begin + lane, next);
#pragma unroll 1
    for (int t = u.begin + lane; t < u.end; t += 32) {
        const Token x = next;
        load(t + 32, next);
        float g = 0.f, ge = 0.f;
        if (x.on) {
            g = seq_slope;
            if (terms) {
                const double d = (double)x.logp - (double)x.old;
                bool cut = false;
                const float w = a.infer ? infer_weight(a, x.old, x.infer, &cut) : 1.f, wa = w * x.adv;
                const bool high = x.adv > 0.f && d > a.log_high;
                const bool low = x.adv < 0.f && d < a.log_low;
                const bool far = x.adv < 0.f && d > a.log_dual;
                const float rho = high ? a.high : low ? a.low : far ? a.dual : expf((float)d);
                const float term = x.adv == 0.f ? 0.f : -(wa * rho);
                const bool beyond = high || low || far;
                r.tokens += 1;
                r.clipped += beyond;
                r.cut += cut;
                r.policy += (double)term;
                g = beyond ? 0.f : term * gw;
            }
            if (a.ref) {
                const float y = (float)((double)x.ref - (double)x.logp);
                const float em1 = expm1f(y);
                r.kl += (double)exp_less_line(y, em1);
                if (a.kl_coef != 0.0) g -= kl_w * em1;
            }
            if (a.entropy) {
                r.entropy += (double)x.entropy;
                ge = ent_g;
            }
        }
        if (a.dlogp) a.dlogp[t] = g;
        if (a.dentropy) a.dentropy[t] = ge;
    }
    // (lane by lane: the warp's lanes are added up once, at the end)
    r.policy *= weight;
    r.kl *= weight;
    r.entropy *= weight;
    return r;
}

__device__ __forceinline__ void add(Total& x, const Total& y) {
    x.policy += y.policy;
    x.kl += y.kl;
    x.entropy += y.entropy;
    x.tokens += y.tokens;
    x.clipped += y.clipped;
    x.cut += y.cut;
}
__device__ __forceinline__ Total warp_total(const Args& a, Total r) {
    r.policy = warp_sum(r.policy);
    if (a.ref) r.kl = warp_sum(r.kl);
    if (a.entropy) r.entropy = warp_sum(r.entropy);
    r.tokens = warp_sum(r.tokens);
    r.clipped = warp_sum(r.clipped);
    if (a.infer) r.cut = warp_sum(r.cut);
    return r;
}
__device__ __forceinline__ void write_loss(const Args& a, const Total& r) {
    a.loss[0] = (float)(r.policy + (a.kl_coef != 0.0 ? a.kl_coef * r.kl : 0.0) -
                        (a.entropy_coef != 0.0 ? a.entropy_coef * r.entropy : 0.0));
    if (a.metrics) {
        a.metrics[0] = (float)r.policy;
        a.metrics[1] = (float)r.kl;
        a.metrics[2] = (float)r.entropy;
    }
    if (a.counts) {
        a.counts[0] = r.tokens;
        a.counts[1] = r.clipped;
        a.counts[2] = r.cut;
    }
}

// The number that the weights are divided by, for the whole CTA: response tokens, or sequences that hold
// one.  `n`, `head`: all units'.
template <int W>
__device__ __forceinline__ double count_divisor(const Args& a, const int* n, const int* head, int* s_warp) {
    if (a.denominator > 0.0) return a.denominator;
    // (the arrays end with zeros up to a multiple of four)
    const int4* from = reinterpret_cast<const int4*>(a.mean_of_sequences ? head : n);
    int k = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < (a.units + 3) / 4; i += 32 * W) {
        const int4 v = from[i];
        k += v.x + v.y + v.z + v.w;
    }
    k = warp_sum(k);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = k;
    __syncthreads();
    k = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) k += s_warp[i];
    return (double)max(k, 1);
}

// cu_seqlens has to ascend from 0 to at most T.
__device__ __forceinline__ void check_bounds(const Args& a, int thread, int threads) {
    if (!a.cu) return;
    for (int i = thread; i <= a.S; i += threads) {
        const int c = a.cu[i];
        if (c < 0 || c > a.T || (i == 0 && c != 0) || (i > 0 && c < a.cu[i - 1]))
            report(a.dev_status, R3_DEV_BAD_INDEX);
    }
}

__global__ void __launch_bounds__(WARPS * 32, CTAS_PER_SM) sums_kernel(const __grid_constant__ Args a) {
    // the second pass may start once everything in front of this one is done: it reads its inputs at once
    tc::grid_dependency_wait();
    tc::grid_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    check_bounds(a, blockIdx.x * WARPS * 32 + threadIdx.x, gridDim.x * WARPS * 32);
    const int padded = (a.units + 3) & ~3;
    for (int unit = blockIdx.x * WARPS + (threadIdx.x >> 5); unit < padded; unit += gridDim.x * WARPS) {
        if (unit >= a.units) {
            a.n[unit] = a.head[unit] = 0;
            continue;
        }
        const Unit u = find_unit(a, unit);
        if (a.need_sums) unit_sums(a, u, unit, a.sums + unit, a.marks + unit, a.n + unit, a.head + unit);
    }
}

__global__ void __launch_bounds__(WARPS * 32, CTAS_PER_SM) loss_kernel(const __grid_constant__ Args a) {
    __shared__ int s_count[WARPS];
    __shared__ int s_seq[2][WARPS];
    __shared__ Whole s_block[2][BLOCKS];
    __shared__ Total s_total[WARPS];
    __shared__ bool s_last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    static_assert(BLOCKS == WARPS, "a block of a long sequence per warp");
    tc::grid_launch_dependents();
    // the first unit is found, and what it reads comes into L2, while the first pass runs
    Unit u = {a.S, 0, 0, 0, 0};
    {
        const int unit = blockIdx.x * WARPS + warp;
        if (unit < a.units) u = find_unit(a, unit);
        const bool terms = !a.by_sequence;
        const float* from[] = {terms || a.ref ? a.logp : nullptr, terms ? a.old : nullptr, terms ? a.infer : nullptr,
                               a.ref, a.entropy, terms && a.adv_per_token ? a.adv : nullptr};
        for (int t = u.begin + 32 * lane; t < u.end; t += 32 * 32)
#pragma unroll
            for (int k = 0; k < 6; ++k)
                if (from[k]) asm volatile("prefetch.global.L2 [%0];" ::"l"(from[k] + t));
        if (a.mask && u.begin + 128 * lane < u.end) asm volatile("prefetch.global.L2 [%0];" ::"l"(a.mask + u.begin + 128 * lane));
    }
    tc::grid_dependency_wait();
    const double divisor = count_divisor<WARPS>(a, a.n, a.head, s_count);
    Total r = {};
    int turn = 0;
    for (int first = blockIdx.x * WARPS; first < a.units; first += gridDim.x * WARPS, turn ^= 1) {
        const int unit = first + warp;
        if (first != (int)blockIdx.x * WARPS) {
            u = {a.S, 0, 0, 0, 0};
            if (unit < a.units) u = find_unit(a, unit);
        }
        Whole w = {};
        w.tokens = 1;
        if (a.by_sequence || a.mean_of_sequences) {
            // (what stands in shared memory is exchanged every other turn: a barrier lies in between)
            if (lane == 0) s_seq[turn][warp] = unit < a.units ? u.seq : -1;
            __syncthreads();
            if (s_seq[turn][0] == s_seq[turn][WARPS - 1] && u.count > LONG) {
                // one long sequence: a block per warp
                const Whole mine = add_block(a, a.sums, a.n, u.first, u.count, warp);
                if (lane == 0) s_block[turn][warp] = mine;
                __syncthreads();
                w.tokens = 0;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) add(w, s_block[turn][b]);
            } else if (u.begin < u.end && u.seq < a.S) {
                w = sequence_sums(a, a.sums, a.n, u.first, u.count);
            }
        }
        add(r, unit_loss(a, u, w.s, w.tokens, divisor, a.sums + unit, a.marks + unit, a.n + unit));
    }
    r = warp_total(a, r);
    if (lane == 0) s_total[warp] = r;
    __syncthreads();
    if (threadIdx.x == 0) {
        Total sum = s_total[0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) add(sum, s_total[i]);
        a.totals[blockIdx.x] = sum;
        __threadfence();
        s_last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
    // the last CTA to arrive adds up all of them, in an order that depends on their number alone
    __threadfence();
    Total sum = {};
    for (int i = threadIdx.x; i < (int)gridDim.x; i += WARPS * 32) {
        const volatile Total* t = a.totals + i;
        add(sum, Total{t->policy, t->kl, t->entropy, t->tokens, t->clipped, t->cut, 0});
    }
    sum = warp_total(a, sum);
    if (lane == 0) s_total[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = s_total[0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) add(sum, s_total[i]);
        write_loss(a, sum);
    }
}

// Both passes of a batch of few units.
__global__ void __launch_bounds__(ONE_WARPS * 32) one_cta_kernel(const __grid_constant__ Args a) {
    __shared__ Sums s_sums[ONE_WARPS];
    __shared__ Marks s_marks[ONE_WARPS];
    __shared__ int s_n[ONE_WARPS], s_head[ONE_WARPS];
    __shared__ Total s_total[ONE_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    tc::grid_launch_dependents();
    tc::grid_dependency_wait();
    check_bounds(a, threadIdx.x, blockDim.x);
    Unit u = {a.S, 0, 0, 0, 0};
    if (warp < a.units) {
        u = find_unit(a, warp);
        unit_sums(a, u, warp, s_sums + warp, s_marks + warp, s_n + warp, s_head + warp);
    }
    __syncthreads();
    double divisor = a.denominator;
    if (!(divisor > 0.0)) {
        const int* from = a.mean_of_sequences ? s_head : s_n;
        divisor = (double)max(warp_sum(lane < a.units ? from[lane] : 0), 1);
    }
    Whole w = {};
    if ((a.by_sequence || a.mean_of_sequences) && u.begin < u.end && u.seq < a.S)
        w = sequence_sums(a, s_sums, s_n, u.first, u.count);
    const Total r = warp_total(a, unit_loss(a, u, w.s, w.tokens, divisor, s_sums + warp, s_marks + warp, s_n + warp));
    if (lane == 0) s_total[warp] = r;
    __syncthreads();
    if (warp == 0) {
        const Total sum = warp_total(a, lane < a.units ? s_total[lane] : Total{});
        if (lane == 0) write_loss(a, sum);
    }
}

static int unit_shift(const r3_policy* c) {
    int shift = LEAST_SHIFT;
    while ((c->T >> shift) > MOST_UNITS) ++shift;
    return shift;
}
static int unit_count(const r3_policy* c) { return c->S + 1 + (c->T >> unit_shift(c)); }

static r3_status check(const r3_policy* c) {
    if (!c || c->T < 0 || c->S < 0 || c->T > (1 << 30) || c->S > (1 << 28)) return R3_ERR_INVALID_ARG;
    if ((c->ratio != R3_RATIO_TOKEN && c->ratio != R3_RATIO_SEQUENCE) ||
        (c->reduce != R3_REDUCE_TOKEN && c->reduce != R3_REDUCE_SEQUENCE))
        return R3_ERR_INVALID_ARG;
    if (!(c->clip_low >= 0.0 && c->clip_low <= 1.0) || !(c->clip_high >= 0.0) ||
        !(c->dual_clip == 0.0 || c->dual_clip > 1.0) || !(c->infer_cap > 0.0) ||
        !(std::fabs(c->kl_coef) < 1e30) || !(std::fabs(c->entropy_coef) < 1e30) ||
        !(c->denominator >= 0.0 && c->denominator < 1e30))
        return R3_ERR_INVALID_ARG;
    return R3_OK;
}

}  // namespace pol
}  // namespace r3

extern "C" size_t r3_policy_loss_workspace_bytes(const r3_policy* c) {
    using namespace r3::pol;
    if (check(c) != R3_OK) return 0;
    const size_t units = (size_t)unit_count(c);
    return 256 + r3::round_up(units * sizeof(Sums), 256) + r3::round_up(units * sizeof(Marks), 256) + 2 * r3::round_up(units * sizeof(int), 256) +
           r3::round_up((units + WARPS - 1) / WARPS * sizeof(Total), 256);
}

extern "C" r3_status r3_policy_loss(const r3_policy* c, const float* logp, const float* logp_old,
                                    const float* advantages, const int32_t* cu_seqlens,
                                    const uint8_t* mask, const float* logp_infer, const float* logp_ref,
                                    const float* entropy, const float* dloss, float* loss, float* dlogp,
                                    float* dentropy, float* metrics, int32_t* counts, void* workspace,
                                    size_t ws_bytes, int32_t* dev_status, void* stream) {
    using namespace r3;
    using namespace r3::pol;
    const r3_status st = check(c);
    if (st != R3_OK) return st;
    if (!loss || (c->T > 0 && (!logp || !logp_old)) || (c->T > 0 && c->S > 0 && !advantages))
        return R3_ERR_INVALID_ARG;
    if (!cu_seqlens && c->S != 1) return R3_ERR_INVALID_ARG;
    if (dentropy && !entropy) return R3_ERR_INVALID_ARG;
    const void* words[] = {logp, logp_old, advantages, cu_seqlens, logp_infer, logp_ref, entropy, dloss,
                           loss, dlogp, dentropy, metrics, counts, dev_status};
    for (const void* p : words)
        if (!aligned(p, 4)) return R3_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || ws_bytes < r3_policy_loss_workspace_bytes(c))
        return R3_ERR_WORKSPACE;
    Args a = {};
    a.T = c->T;
    a.S = c->S;
    a.units = unit_count(c);
    a.shift = unit_shift(c);
    a.by_sequence = c->ratio == R3_RATIO_SEQUENCE;
    a.mean_of_sequences = c->reduce == R3_REDUCE_SEQUENCE;
    a.adv_per_token = c->adv_per_token != 0;
    a.need_sums = a.by_sequence || a.mean_of_sequences || c->denominator == 0.0;
    a.log_high = std::log1p(c->clip_high);
    a.log_low = std::log1p(-c->clip_low);
    a.log_dual = c->dual_clip > 0.0 ? std::log(c->dual_clip) : INFINITY;
    a.log_cap = std::log(c->infer_cap);
    a.high = (float)(1.0 + c->clip_high);
    a.low = (float)(1.0 - c->clip_low);
    a.dual = (float)c->dual_clip;
    a.cap = (float)c->infer_cap;
    a.kl_coef = c->kl_coef;
    a.entropy_coef = c->entropy_coef;
    a.denominator = c->denominator;
    a.logp = logp;
    a.old = logp_old;
    a.adv = advantages;
    a.infer = logp_infer;
    a.ref = logp_ref;
    a.entropy = entropy;
    a.dloss = dloss;
    a.cu = cu_seqlens;
    a.mask = mask;
    a.loss = loss;
    a.dlogp = dlogp;
    a.dentropy = dentropy;
    a.metrics = metrics;
    a.counts = counts;
    a.dev_status = dev_status;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.ticket = reinterpret_cast<unsigned*>(ws);
    ws += 256;
    a.sums = reinterpret_cast<Sums*>(ws);
    ws += round_up((size_t)a.units * sizeof(Sums), 256);
    a.marks = reinterpret_cast<Marks*>(ws);
    ws += round_up((size_t)a.units * sizeof(Marks), 256);
    a.n = reinterpret_cast<int*>(ws);
    ws += round_up((size_t)a.units * sizeof(int), 256);
    a.head = reinterpret_cast<int*>(ws);
    ws += round_up((size_t)a.units * sizeof(int), 256);
    a.totals = reinterpret_cast<Total*>(ws);
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (a.units <= ONE_WARPS)
        return tc::launch_dependent(one_cta_kernel, dim3(1), dim3(32 * a.units), 0, cs, a) == cudaSuccess
                   ? R3_OK : R3_ERR_CUDA;
    // a wave of resident CTAs at most, which go on to further units
    const int ctas = (a.units + WARPS - 1) / WARPS, most = CTAS_PER_SM * sm_count(), grid = ctas < most ? ctas : most;
    if (tc::launch_dependent(sums_kernel, dim3(grid), dim3(WARPS * 32), 0, cs, a) != cudaSuccess ||
        tc::launch_dependent(loss_kernel, dim3(grid), dim3(WARPS * 32), 0, cs, a) != cudaSuccess)
        return R3_ERR_CUDA;
    return R3_OK;
}
