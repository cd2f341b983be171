// One AdamW step over many tensors in one launch: what follows the weight gradients of the
// replayed layers.  Per element, with g the gradient times grad_scale:
//   m = beta1 m + (1 - beta1) g          v = beta2 v + (1 - beta2) g^2
//   w = w (1 - lr decay) - lr / (1 - beta1^t)  m / ( sqrt(v) / sqrt(1 - beta2^t) + eps )
//
// Bound by HBM (12.06 bytes an element for bf16 weights, float32 gradients and 8-bit states; 28 for
// float32 with 32-bit states): 604 M elements of the former 1110 us = the measured copy bandwidth (1270
// at the clock of a power-capped second, where instruction issue bounds it), 120 M bf16 elements with
// master weights, bf16 gradients and 32-bit states 522 us = 98%.  States of 8 bits are kept in blocks of 256 elements with one scale:
// e4m3 codes times the smallest power of two (at least 2^-126) that brings the block's largest
// magnitude to 448 or less, so that scaling is exact both ways and the one rounding is the code's.
// The second moment is kept as its square root, which halves the range its codes have to span; a
// root above zero is never kept as zero, because the update divides by it (the smallest code is the
// safe side: a smaller step).  Every sum and product that leads to a stored state is rounded to float32
// by itself (no fused multiply-add), and every code is that of the correctly rounded root, so that the states
// do not depend on how a compiler contracts the expressions or a GPU approximates a root.
//
// A warp takes a block, and one warp-wide maximum per state gives its scale.  With 32-bit states lane l
// holds elements 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3: every load and store of the warp covers
// consecutive bytes.  With 8-bit states it holds 8 l .. 8 l + 7 and takes them out of a ring in shared
// memory that the warp copies its blocks to ahead (16 bytes per lane and copy, so 4 or 5 copies, 6 loads
// and 3 or 4 stores a block where 4-element pieces take twice as many).  The table of tensors travels in the
// kernel's parameters: no workspace, no copy, and a captured launch keeps its own.
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>
#include <utility>
#include <vector>

#include "r3_common.cuh"
#include "r3_internal.h"

namespace r3 {

constexpr int kAdamBlock = 256;                     // elements per scale
constexpr int kAdamThreads = 256;
constexpr int kAdamWarps = kAdamThreads / 32;
constexpr int kAdamCtas = 4, kAdamCtas8 = 2;        // resident per SM at up to 64 and 128 registers a thread
constexpr int kAdamStages = 4;                      // 8-bit states: blocks in a warp's ring
constexpr int kAdamMaxPerWarp8 = 16, kAdamMaxPerWarp = 8;   // blocks per warp and chunk, 8- and 32-bit states
constexpr int kAdamSmall = 24, kAdamLarge = 400;    // tensors per launch

struct AdamTensor {
    void* param;
    float* master;
    const void* grad;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    long long n;
    float decay;
};
struct AdamScalars {
    float beta1, one_beta1, beta2, one_beta2, eps, lr, bias1, bias2, one;
    const float* grad_scale;
    const float* dynamic;                           // {lr, bias1, bias2} on the device, or null
    const int32_t* dev_status;                      // not null: no step where an error stands in it
    int tensors, per_warp;
};
template <int CAP> struct AdamTable {
    AdamScalars s;
    unsigned first[CAP];                            // first chunk of each tensor, close together for the search
    AdamTensor t[CAP];
};

// Four consecutive elements as they lie, and as float32.
template <typename T> struct Four;
template <> struct Four<float> {
    float4 v;
    __device__ __forceinline__ void unpack(float* f) const {
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    }
    __device__ __forceinline__ void pack(const float* f) { v = make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Four<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void unpack(float* f) const {
        const float2 a = bf16_pair(v.x), b = bf16_pair(v.y);
        f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
    }
    __device__ __forceinline__ void pack(const float* f) {
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
        h[0] = __floats2bfloat162_rn(f[0], f[1]);
        h[1] = __floats2bfloat162_rn(f[2], f[3]);
    }
};
template <> struct Four<uint8_t> {                  // e4m3 codes
    uint32_t v;
    __device__ __forceinline__ void unpack(float* f) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const __half2_raw h =
                __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v >> (16 * i)), __NV_E4M3);
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&h));
            f[2 * i] = t.x;
            f[2 * i + 1] = t.y;
        }
    }
    __device__ __forceinline__ void pack(const float* f) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
        v = lo | (hi << 16);
    }
};
// A lane's eight elements of a block, in two fours: 4 l .. and 128 + 4 l .., or (NEAR) 8 l .. and
// 8 l + 4 ..; `left` elements of the tensor follow from the block's first on (only looked at where FULL
// is false; what lies behind reads as 0 and is not written).
template <bool NEAR> __device__ __forceinline__ int place(int h, int lane) {
    return NEAR ? 8 * lane + 4 * h : 128 * h + 4 * lane;
}
template <bool FULL, bool NEAR, typename T>
__device__ __forceinline__ void take(const T* p, int lane, int left, Four<T> (&f)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = place<NEAR>(h, lane);
        if (FULL) {
            f[h] = *reinterpret_cast<const Four<T>*>(p + at);
        } else {
            T e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (at + i < left) e[i] = p[at + i];
                else memset(&e[i], 0, sizeof(T));
            }
            memcpy(&f[h], e, sizeof(e));
        }
    }
}
// Two neighbouring fours of less than 16 bytes are one load or store.
template <typename T> struct alignas(sizeof(T) == 4 ? 16 : 8 * sizeof(T)) Eight {
    Four<T> f[2];
};
template <bool FULL, bool NEAR, typename T>
__device__ __forceinline__ void put(T* p, int lane, int left, const Four<T> (&f)[2]) {
    if constexpr (FULL && NEAR && sizeof(T) < 4) {
        *reinterpret_cast<Eight<T>*>(p + 8 * lane) = {{f[0], f[1]}};
        return;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = place<NEAR>(h, lane);
        if (FULL) {
            *reinterpret_cast<Four<T>*>(p + at) = f[h];
        } else {
            T e[4];
            memcpy(e, &f[h], sizeof(e));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + i < left) p[at + i] = e[i];
        }
    }
}
// Two float32 values in a register pair, one instruction for both.  There is no sum among them: the
// compiler contracts a product and a sum of pairs into one fused operation, .rn or not (measured: a
// quarter of random sums of two products differ).  A sum is a fused multiply-add with a factor of 1 that
// only the launch knows, which rounds once and has nothing to be contracted with.
typedef unsigned long long F2;
__device__ __forceinline__ F2 pair(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(F2 v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float max_abs(float a, float b) {      // a NaN stays one
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
// Biased exponent of the scale 2^k for a block whose largest magnitude is f 2^e, f in [1, 2), given
// as bits: 448 = 1.75 2^8, so k = e - 8, and one more where f > 1.75 (the addition carries then); at
// least -126.
__device__ __forceinline__ uint32_t scale_exponent(uint32_t bits) {
    const uint32_t e = (bits + 0x1fffffu) >> 23;
    return e > 9u ? e - 8u : 1u;
}
// The same for the root of a second moment whose largest value is f 2^e: the root is at most 448 2^k
// exactly where the value is at most 448^2 4^k, 448^2 = 1.53125 2^17, so k = ceil((e - 17 + [f >
// 1.53125]) / 2).  Values below float32's normal range are brought into it first.
__device__ __forceinline__ uint32_t root_exponent(uint32_t bits) {
    if (bits == 0u) return 1u;
    int shift = 0;
    if (bits < 0x00800000u) {
        bits = __float_as_uint(__uint_as_float(bits) * 18446744073709551616.f);         // 2^64
        shift = 64;
    }
    const int e = (int)((bits + 0x3bffffu) >> 23) - 127 - shift;
    return (uint32_t)(((e - 16) >> 1) + 127);
}
// The largest magnitude of a block's finite values, as bits; `clean` tells whether all are.
__device__ __forceinline__ uint32_t block_top(const float (&f)[8], bool& clean) {
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max_abs(big, f[i]);
    uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(big));
    clean = top < 0x7f800000u;
    if (!clean) {
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = __float_as_uint(f[i]) & 0x7fffffffu;
            if (b < 0x7f800000u) top = max(top, b);
        }
        top = __reduce_max_sync(0xffffffffu, top);
    }
    return top;
}
__device__ __forceinline__ void mark_nan(const float (&f)[8], Four<uint8_t> (&codes)[2]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)                     // 0x7f: NaN
        if ((__float_as_uint(f[i]) & 0x7f800000u) == 0x7f800000u) codes[i >> 2].v |= 0x7fu << (8 * (i & 3));
}
// The eight codes of a lane and the scale of its block.
__device__ __forceinline__ float quantise(const float (&f)[8], Four<uint8_t> (&codes)[2]) {
    bool clean;
    const uint32_t e = scale_exponent(block_top(f, clean));
    const float inv = __uint_as_float((254u - e) << 23);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = f[4 * h + i] * inv;
        codes[h].pack(q);
    }
    if (!clean) mark_nan(f, codes);
    return __uint_as_float(e << 23);
}
// Sixteen units of 2^-24: four times what an approximate root and the product with the scale are off by.
constexpr float kRootSlack = 9.5367432e-7f;
// The same for the second moment v (least its least element), kept as its root: none above zero
// becomes code 0.  With APPROX the roots are only within 2^-22: where their codes differ between the ends of
// an interval that holds the right root (a few lanes in 10^4), the four roots are formed again to the last
// bit, so that the codes are those of correctly rounded roots in either form.
template <bool APPROX>
__device__ __forceinline__ float quantise_root(const float (&v)[8], const float (&root)[8], float least,
                                               Four<uint8_t> (&codes)[2]) {
    bool clean;
    const uint32_t e = root_exponent(block_top(v, clean));
    const float inv = __uint_as_float((254u - e) << 23);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[4];
        if constexpr (APPROX) {
            const float low = inv * (1.f - kRootSlack), high = inv * (1.f + kRootSlack);
            Four<uint8_t> other;
#pragma unroll
            for (int i = 0; i < 4; i += 2)
                split(mul2(pair(root[4 * h + i], root[4 * h + i + 1]), pair(low, low)), q[i], q[i + 1]);
            codes[h].pack(q);
#pragma unroll
            for (int i = 0; i < 4; i += 2)
                split(mul2(pair(root[4 * h + i], root[4 * h + i + 1]), pair(high, high)), q[i], q[i + 1]);
            other.pack(q);
            if (codes[h].v != other.v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = __fsqrt_rn(v[4 * h + i]) * inv;
                codes[h].pack(q);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = root[4 * h + i] * inv;
            codes[h].pack(q);
        }
        // 1 in every byte that is 0 (no code here has its top bit set, so nothing carries)
        const uint32_t zeros = (((codes[h].v + 0x7f7f7f7fu) & 0x80808080u) ^ 0x80808080u) >> 7;
        if (least > 0.f) {
            codes[h].v |= zeros;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[4 * h + i] > 0.f) codes[h].v |= zeros & (0xffu << (8 * i));
        }
    }
    if (!clean) mark_nan(v, codes);
    return __uint_as_float(e << 23);
}

struct AdamRates {                                  // what the whole launch shares
    float beta1, one_beta1, beta2, one_beta2, eps, bias2, step, keep, gs, one;
};

__device__ __forceinline__ void copy_ahead16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                 ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_ahead4(void* dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;"
                 ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

// One block's values: loaded to registers, or (8-bit states) copied ahead to a stage of the warp's ring.
// The arithmetic around the codes is long enough to leave the memory idle without the ring; with 32-bit
// states the occupancy does as well, and the registers and the shared memory are better left to it.
template <typename P, typename G, bool MASTER, bool BITS8> struct AdamBlock {
    typedef typename std::conditional<MASTER, float, P>::type Wt;
    typedef typename std::conditional<BITS8, uint8_t, float>::type St;
    // bf16 weights without masters and 8-bit states: the update's root and quotient are the hardware's
    // approximations, a unit or two of 2^-23 off beside the weight's rounding of 2^-9, and the codes are
    // secured by themselves.  At the clock of a power-capped second this form is bound by instruction issue: 604
    // M elements 1260 us, 1350 with the exact root, 1540 with the exact quotient too (1215 with approximate
    // codes); with 32-bit states the exact ones cost 0.3%.
    static constexpr bool APPROX = BITS8 && sizeof(Wt) == 2;
    Four<Wt> w[2];
    Four<G> g[2];
    Four<St> m[2], v[2];
    float ms, vs;

    struct Stage {
        alignas(16) Wt w[kAdamBlock];
        G g[kAdamBlock];
        St m[kAdamBlock], v[kAdamBlock];
        float scale[4];                             // of m, of v, unused
    };
    template <typename T> static __device__ __forceinline__ void ahead(T* to, const void* from, long long at, int lane) {
        constexpr int N = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < kAdamBlock; i += 32 * N)
            copy_ahead16(to + i + N * lane, static_cast<const T*>(from) + at + i + N * lane);
    }
    // A whole block, copied by its warp (one group of copies per lane, empty for block >= end).
    static __device__ __forceinline__ void fetch(Stage* s, const AdamTensor& t, long long block,
                                                 long long end, int lane) {
        if (block < end) {
            const long long at = block * kAdamBlock;
            ahead(s->w, MASTER ? static_cast<const void*>(t.master) : t.param, at, lane);
            ahead(s->g, t.grad, at, lane);
            // the codes of both states: 16 lanes each
            const int half = lane >> 4, i = 16 * (lane & 15);
            copy_ahead16((half ? s->v : s->m) + i, static_cast<const uint8_t*>(half ? t.v : t.m) + at + i);
            if (lane < 2) copy_ahead4(&s->scale[lane], (lane == 0 ? t.m_scale : t.v_scale) + block);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    template <typename T> static __device__ __forceinline__ void near(const T* p, int lane, Four<T> (&f)[2]) {
        const Eight<T> e = *reinterpret_cast<const Eight<T>*>(p + 8 * lane);
        f[0] = e.f[0];
        f[1] = e.f[1];
    }
    __device__ __forceinline__ void from_stage(const Stage* s, int lane) {
        near(s->w, lane, w);
        near(s->g, lane, g);
        near(s->m, lane, m);
        near(s->v, lane, v);
        const float2 both = *reinterpret_cast<const float2*>(s->scale);
        ms = both.x;
        vs = both.y;
    }

    template <bool FULL>
    __device__ __forceinline__ void load(const AdamTensor& t, long long block, int lane, int left) {
        const long long at = block * kAdamBlock;
        take<FULL, BITS8>((MASTER ? reinterpret_cast<const Wt*>(t.master) : static_cast<const Wt*>(t.param)) + at,
                   lane, left, w);
        take<FULL, BITS8>(static_cast<const G*>(t.grad) + at, lane, left, g);
        take<FULL, BITS8>(static_cast<const St*>(t.m) + at, lane, left, m);
        take<FULL, BITS8>(static_cast<const St*>(t.v) + at, lane, left, v);
        if (BITS8) {
            ms = t.m_scale[block];
            vs = t.v_scale[block];
        }
    }
    template <bool FULL>
    __device__ __forceinline__ void update(const AdamTensor& t, long long block, int lane, int left,
                                           const AdamRates& a) {
        const long long at = block * kAdamBlock;
        float fw[8], fg[8], fm[8], fv[8], root[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            w[h].unpack(fw + 4 * h);
            g[h].unpack(fg + 4 * h);
            m[h].unpack(fm + 4 * h);
            v[h].unpack(fv + 4 * h);
        }
        const F2 gs = pair(a.gs, a.gs), b1 = pair(a.beta1, a.beta1), c1 = pair(a.one_beta1, a.one_beta1);
        const F2 b2 = pair(a.beta2, a.beta2), c2 = pair(a.one_beta2, a.one_beta2), one = pair(a.one, a.one);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const F2 gi = mul2(pair(fg[i], fg[i + 1]), gs);
            F2 m0 = pair(fm[i], fm[i + 1]), v0 = pair(fv[i], fv[i + 1]);
            if (BITS8) {
                m0 = mul2(m0, pair(ms, ms));        // powers of two: exact
                v0 = mul2(v0, pair(vs, vs));
                v0 = mul2(v0, v0);
            }
            split(fma2(mul2(b1, m0), one, mul2(c1, gi)), fm[i], fm[i + 1]);
            split(fma2(mul2(b2, v0), one, mul2(c2, mul2(gi, gi))), fv[i], fv[i + 1]);
        }
        // Roots and quotients are rounded to the last bit where the weight is kept in float32, and where the
        // kernel waits for the memory anyway (32-bit states).
        float least = fv[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) least = fminf(least, fv[i]);
        if (!APPROX) {
#pragma unroll
            for (int i = 0; i < 8; ++i) root[i] = __fsqrt_rn(fv[i]);
        } else if (least >= 1.17549435e-38f) {      // below float32's normal range the longer form
#pragma unroll
            for (int i = 0; i < 8; ++i) asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root[i]) : "f"(fv[i]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) asm("sqrt.approx.f32 %0, %1;" : "=f"(root[i]) : "f"(fv[i]));
        }
        const F2 bias2 = pair(a.bias2, a.bias2), eps = pair(a.eps, a.eps);
        const F2 step = pair(-a.step, -a.step), keep = pair(a.keep, a.keep);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float lo, hi;
            split(fma2(pair(root[i], root[i + 1]), bias2, eps), lo, hi);
            F2 up;
            if (APPROX) {
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(lo) : "f"(lo));
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(hi) : "f"(hi));
                up = mul2(pair(fm[i], fm[i + 1]), pair(lo, hi));
            } else {
                up = pair(__fdiv_rn(fm[i], lo), __fdiv_rn(fm[i + 1], hi));
            }
            split(fma2(step, up, mul2(pair(fw[i], fw[i + 1]), keep)), fw[i], fw[i + 1]);
        }
        if constexpr (BITS8) {
            ms = quantise(fm, m);
            vs = quantise_root<APPROX>(fv, root, least, v);
            if (lane == 0) {
                t.m_scale[block] = ms;
                t.v_scale[block] = vs;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                m[h].pack(fm + 4 * h);
                v[h].pack(fv + 4 * h);
            }
        }
        put<FULL, BITS8>(static_cast<St*>(t.m) + at, lane, left, m);
        put<FULL, BITS8>(static_cast<St*>(t.v) + at, lane, left, v);
        Four<P> p[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) p[h].pack(fw + 4 * h);
        put<FULL, BITS8>(static_cast<P*>(t.param) + at, lane, left, p);
        if constexpr (MASTER) {
#pragma unroll
            for (int h = 0; h < 2; ++h) w[h].pack(fw + 4 * h);
            put<FULL, BITS8>(t.master + at, lane, left, w);
        }
    }
};

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
__global__ void __launch_bounds__(kAdamThreads, BITS8 ? kAdamCtas8 : kAdamCtas) adamw_kernel(const __grid_constant__ AdamTable<CAP> a) {
    extern __shared__ uint4 ring_all[];             // 8-bit states: [warps][kAdamStages] stages
    AdamRates r;
    r.gs = a.s.grad_scale ? *a.s.grad_scale : 1.f;
    const int32_t error = a.s.dev_status ? *a.s.dev_status : R3_DEV_OK;
    // NaN or infinite, or gradients that an error was reported for: the step is skipped
    if (!(fabsf(r.gs) <= 3.402823466e38f) || error != R3_DEV_OK) return;
    const float lr = a.s.dynamic ? a.s.dynamic[0] : a.s.lr;
    r.step = lr * (a.s.dynamic ? a.s.dynamic[1] : a.s.bias1);
    r.bias2 = a.s.dynamic ? a.s.dynamic[2] : a.s.bias2;
    r.beta1 = a.s.beta1;
    r.one_beta1 = a.s.one_beta1;
    r.beta2 = a.s.beta2;
    r.one_beta2 = a.s.one_beta2;
    r.eps = a.s.eps;
    r.one = a.s.one;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned chunk = blockIdx.x;
    int lo = 0, hi = a.s.tensors - 1;           // the last tensor that starts at or before it
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    const AdamTensor t = a.t[lo];
    const unsigned first = a.first[lo];
    r.keep = 1.f - lr * t.decay;
    // the warps of a CTA take the chunk's blocks in turn
    long long block = (long long)(chunk - first) * (kAdamWarps * a.s.per_warp) + warp;
    const long long whole = t.n / kAdamBlock;   // blocks without a ragged end
    const long long end = min(whole, block + (long long)kAdamWarps * a.s.per_warp);
    AdamBlock<P, G, MASTER, BITS8> b;
    if constexpr (BITS8) {
        typedef typename AdamBlock<P, G, MASTER, BITS8>::Stage Stage;
        Stage* ring = reinterpret_cast<Stage*>(ring_all) + warp * kAdamStages;
#pragma unroll
        for (int s = 0; s < kAdamStages; ++s) b.fetch(ring + s, t, block + s * kAdamWarps, end, lane);
        for (int stage = 0; block < end; block += kAdamWarps) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kAdamStages - 1) : "memory");
            __syncwarp();                       // the lanes' copies of the scales
            b.from_stage(ring + stage, lane);
            __syncwarp();                       // read by all lanes before it is written again
            b.fetch(ring + stage, t, block + kAdamStages * kAdamWarps, end, lane);
            stage = stage + 1 == kAdamStages ? 0 : stage + 1;
            b.template update<true>(t, block, lane, kAdamBlock, r);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    } else {
        for (; block < end; block += kAdamWarps) {
            b.template load<true>(t, block, lane, kAdamBlock);
            b.template update<true>(t, block, lane, kAdamBlock, r);
        }
    }
    // the warp whose turn it is takes the ragged end
    const long long past = (long long)(chunk - first + 1) * (kAdamWarps * a.s.per_warp);
    if (block == whole && block < past && t.n > whole * kAdamBlock) {
        const int left = (int)(t.n - whole * kAdamBlock);
        b.template load<false>(t, block, lane, left);
        b.template update<false>(t, block, lane, left, r);
    }
}

// ---- host side ------------------------------------------------------------------------------------
static r3_status check_adamw(const r3_adamw* c, const r3_adamw_tensor* ts, int32_t count) {
    if (!c || count < 0 || (count > 0 && !ts)) return R3_ERR_INVALID_ARG;
    if ((c->param_dtype != R3_F32 && c->param_dtype != R3_BF16) ||
        (c->grad_dtype != R3_F32 && c->grad_dtype != R3_BF16) ||
        (c->state_bits != 8 && c->state_bits != 32))
        return R3_ERR_INVALID_ARG;
    if (c->master && c->param_dtype != R3_BF16) return R3_ERR_INVALID_ARG;
    if (c->step < 1 || !(c->lr >= 0.0 && c->lr < 1e30) || !(c->beta1 >= 0.0 && c->beta1 < 1.0) ||
        !(c->beta2 >= 0.0 && c->beta2 < 1.0) || !(c->eps >= 1e-30 && c->eps < 1e30))
        return R3_ERR_INVALID_ARG;
    for (int32_t i = 0; i < count; ++i) {
        const r3_adamw_tensor& t = ts[i];
        if (t.n < 0 || t.n > (1LL << 40) || !(t.weight_decay >= 0.f && t.weight_decay < 1e30f))
            return R3_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq || (c->master != 0) != (t.master != nullptr))
            return R3_ERR_INVALID_ARG;
        if (c->state_bits == 8 && (!t.exp_avg_scale || !t.exp_avg_sq_scale)) return R3_ERR_INVALID_ARG;
        const void* ps[5] = {t.param, t.master, t.grad, t.exp_avg, t.exp_avg_sq};
        for (const void* p : ps)
            if (!aligned(p, 16)) return R3_ERR_INVALID_ARG;
        if (c->state_bits == 8 && (!aligned(t.exp_avg_scale, 4) || !aligned(t.exp_avg_sq_scale, 4)))
            return R3_ERR_INVALID_ARG;
    }
    return R3_OK;
}
// Calls f(kind, begin, end) for every buffer that the step writes.
template <typename F> static void each_written(const r3_adamw* c, const r3_adamw_tensor* ts, int32_t count, F f) {
    const int64_t size = c->param_dtype == R3_BF16 ? 2 : 4, state = c->state_bits == 8 ? 1 : 4;
    auto one = [&](int kind, const void* p, int64_t bytes) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) f(kind, at, at + (uintptr_t)bytes);
    };
    for (int32_t i = 0; i < count; ++i) {
        const r3_adamw_tensor& t = ts[i];
        if (t.n == 0) continue;
        one(0, t.param, t.n * size);
        one(1, t.master, t.n * 4);
        one(2, t.exp_avg, t.n * state);
        one(3, t.exp_avg_sq, t.n * state);
        if (c->state_bits != 8) continue;
        const int64_t scales = (t.n + kAdamBlock - 1) / kAdamBlock * 4;
        one(4, t.exp_avg_scale, scales);
        one(5, t.exp_avg_sq_scale, scales);
    }
}
// The same for every buffer that it reads alone; `grads` (3, or null) stand in for the entries' own.
template <typename F>
static void each_read(const r3_adamw* c, const r3_adamw_tensor* ts, int32_t count, const void* const* grads,
                      const float* grad_scale, const float* scalars, F f) {
    const int64_t size = c->grad_dtype == R3_BF16 ? 2 : 4;
    auto one = [&](const void* p, int64_t bytes) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) f(at, at + (uintptr_t)bytes);
    };
    for (int32_t i = 0; i < count; ++i) one(grads ? grads[i % 3] : ts[i].n ? ts[i].grad : nullptr, ts[i].n * size);
    one(grad_scale, 4);
    one(scalars, 12);
}
typedef std::pair<uintptr_t, uintptr_t> Range;
// Into ascending order: neighbouring ascending runs are merged, pair by pair, where they are few.
static void sort_runs(std::vector<Range>& v) {
    std::vector<size_t> ends;
    for (size_t i = 1; i <= v.size(); ++i)
        if (i == v.size() || v[i].first < v[i - 1].first) ends.push_back(i);
    if (ends.size() > v.size() / 16 + 8) {
        std::sort(v.begin(), v.end());
        return;
    }
    std::vector<Range> to(v.size());
    while (ends.size() > 1) {
        size_t from = 0, kept = 0;
        for (size_t k = 0; k < ends.size(); k += 2) {
            const size_t mid = ends[k], end = k + 1 < ends.size() ? ends[k + 1] : mid;
            std::merge(v.begin() + from, v.begin() + mid, v.begin() + mid, v.begin() + end, to.begin() + from);
            from = ends[kept++] = end;
        }
        ends.resize(kept);
        v.swap(to);
    }
}
// Two buffers on the same memory would be updated at once, in no order, and what is read there would change
// under the step.  Lists that were allocated one after the other, or tensor by tensor, ascend and need no sort,
// and gradients that lie apart from all of them no search (checks of 300 tensors with 8-bit states: 4 us of
// host time, 10 to 13 with gradients in between, 32 where params and gradients lie in no order).
r3_status check_adamw_distinct(const r3_adamw* c, const r3_adamw_tensor* ts, int32_t count,
                               const void* const* grads, const float* grad_scale, const float* scalars) {
    constexpr int KINDS = 6;
    uintptr_t low[KINDS], high[KINDS] = {}, past = 0, least = ~(uintptr_t)0, most = 0;
    bool ascending = true, lists = true;
    each_written(c, ts, count, [&](int k, uintptr_t begin, uintptr_t end) {
        ascending &= begin >= past;
        past = end;
        lists &= begin >= high[k];
        if (high[k] == 0 || begin < low[k]) low[k] = begin;
        if (end > high[k]) high[k] = end;
    });
    for (int k = 0; k < KINDS; ++k) {
        if (!high[k]) continue;
        least = std::min(least, low[k]);
        most = std::max(most, high[k]);
        for (int q = 0; q < k && lists; ++q)
            if (high[q] && low[k] < high[q] && low[q] < high[k]) lists = false;
    }
    auto meets = [&](int k, uintptr_t begin, uintptr_t end) { return high[k] && low[k] < end && begin < high[k]; };
    bool apart = true;
    each_read(c, ts, count, grads, grad_scale, scalars, [&](uintptr_t begin, uintptr_t end) {
        if (begin >= most || end <= least) return;
        for (int k = 0; k < KINDS; ++k) apart = apart && !meets(k, begin, end);
    });
    if ((ascending || lists) && apart) return R3_OK;
    try {
        // the written ranges in ascending order: tensor by tensor as they come, a few by insertion, or list
        // by list, whose runs are few and merged
        constexpr int FEW = 48;
        Range few[FEW];
        std::vector<Range> many;
        Range* all = few;
        size_t n = 0;
        if (count <= FEW / KINDS) {
            each_written(c, ts, count, [&](int, uintptr_t begin, uintptr_t end) {
                size_t i = n++;
                for (; i > 0 && begin < few[i - 1].first; --i) few[i] = few[i - 1];
                few[i] = {begin, end};
            });
        } else {
            many.reserve((size_t)count * KINDS);
            if (ascending) {
                each_written(c, ts, count,
                             [&](int, uintptr_t begin, uintptr_t end) { many.emplace_back(begin, end); });
            } else {
                std::vector<Range> list[KINDS];
                for (std::vector<Range>& v : list) v.reserve((size_t)count);
                each_written(c, ts, count,
                             [&](int k, uintptr_t begin, uintptr_t end) { list[k].emplace_back(begin, end); });
                for (const std::vector<Range>& v : list) many.insert(many.end(), v.begin(), v.end());
                sort_runs(many);
            }
            all = many.data();
            n = many.size();
        }
        for (size_t i = 1; i < n; ++i)
            if (all[i].first < all[i - 1].second) return R3_ERR_INVALID_ARG;
        // each read range has to lie between two neighbours; mostly a few places past the one before
        bool clear = true;
        size_t at = 0;                              // the first written range that ends behind `begin`
        each_read(c, ts, count, grads, grad_scale, scalars, [&](uintptr_t begin, uintptr_t end) {
            if (begin >= most || end <= least) return;
            for (int hop = 0; hop < 8 && at < n && all[at].second <= begin; ++hop) ++at;
            if ((at < n && all[at].second <= begin) || (at > 0 && all[at - 1].second > begin))
                at = std::upper_bound(all, all + n, begin, [](uintptr_t p, const Range& w) { return p < w.second; }) - all;
            clear = clear && (at == n || all[at].first >= end);
        });
        return clear ? R3_OK : R3_ERR_INVALID_ARG;
    } catch (...) {                                 // out of host memory
        return R3_ERR_INVALID_ARG;
    }
}

r3_status check_adamw_call(const r3_adamw* config, const r3_adamw_tensor* tensors, int32_t n_tensors,
                           const float* grad_scale, const float* scalars) {
    const r3_status st = check_adamw(config, tensors, n_tensors);
    if (st != R3_OK) return st;
    if (!aligned(grad_scale, 4) || !aligned(scalars, 4)) return R3_ERR_INVALID_ARG;
    return check_adamw_distinct(config, tensors, n_tensors, nullptr, grad_scale, scalars);
}

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
static r3_status launch_adamw(const AdamScalars& s, const r3_adamw_tensor* ts, int count, cudaStream_t cs) {
    AdamTable<CAP> a;
    a.s = s;
    for (int done = 0; done < count;) {
        // A CTA takes one chunk (CTAs that walk over chunks left SMs idle for 16% of the time, since not
        // all of them see the memory at the same speed).  Blocks per warp and chunk: as many as leave
        // the resident warps four chunks each, so that a short list still spreads over the GPU.
        long long blocks = 0;
        for (int i = done, k = 0; i < count && k < CAP; ++i) {
            blocks += (ts[i].n + kAdamBlock - 1) / kAdamBlock;
            k += ts[i].n > 0;
        }
        const long long share = blocks / (4LL * kAdamWarps * (BITS8 ? kAdamCtas8 : kAdamCtas) * sm_count());
        const long long most = BITS8 ? kAdamMaxPerWarp8 : kAdamMaxPerWarp;
        const int per_warp = (int)(share < 1 ? 1 : share > most ? most : share);
        const long long chunk = (long long)kAdamBlock * kAdamWarps * per_warp;
        long long chunks = 0;
        int k = 0;
        for (; done < count && k < CAP; ++done) {
            const r3_adamw_tensor& t = ts[done];
            if (t.n == 0) continue;
            const long long more = (t.n + chunk - 1) / chunk;
            if (chunks + more > 0x7fffffffLL) {
                if (k == 0) return R3_ERR_UNSUPPORTED;
                break;
            }
            a.t[k] = {t.param, t.master, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale,
                      t.exp_avg_sq_scale, t.n, t.weight_decay};
            a.first[k] = (unsigned)chunks;
            chunks += more;
            ++k;
        }
        if (k == 0) break;
        a.s.tensors = k;
        a.s.per_warp = per_warp;
        size_t smem = 0;
        if constexpr (BITS8) {
            smem = sizeof(typename AdamBlock<P, G, MASTER, BITS8>::Stage) * kAdamStages * kAdamWarps;
            static PerDevice ready;
            if (!ready.done()) {
                if (cudaFuncSetAttribute(adamw_kernel<P, G, MASTER, BITS8, CAP>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
                    return R3_ERR_CUDA;
                ready.mark();
            }
        }
        adamw_kernel<P, G, MASTER, BITS8, CAP>
            <<<(unsigned)chunks, kAdamThreads, smem, cs>>>(a);
        const r3_status st = launch_status();
        if (st != R3_OK) return st;
    }
    return R3_OK;
}
template <typename P, typename G, bool MASTER, bool BITS8>
static r3_status launch_adamw(const AdamScalars& s, const r3_adamw_tensor* ts, int count, cudaStream_t cs) {
    // the parameters of a launch are copied for it: a short list takes the short table
    return count <= kAdamSmall ? launch_adamw<P, G, MASTER, BITS8, kAdamSmall>(s, ts, count, cs)
                               : launch_adamw<P, G, MASTER, BITS8, kAdamLarge>(s, ts, count, cs);
}
template <typename P, typename G, bool MASTER>
static r3_status launch_adamw(const r3_adamw* c, const AdamScalars& s, const r3_adamw_tensor* ts,
                              int count, cudaStream_t cs) {
    return c->state_bits == 8 ? launch_adamw<P, G, MASTER, true>(s, ts, count, cs)
                              : launch_adamw<P, G, MASTER, false>(s, ts, count, cs);
}
template <typename G>
static r3_status launch_adamw(const r3_adamw* c, const AdamScalars& s, const r3_adamw_tensor* ts,
                              int count, cudaStream_t cs) {
    if (c->param_dtype == R3_F32) return launch_adamw<float, G, false>(c, s, ts, count, cs);
    return c->master ? launch_adamw<__nv_bfloat16, G, true>(c, s, ts, count, cs)
                     : launch_adamw<__nv_bfloat16, G, false>(c, s, ts, count, cs);
}

r3_status adamw_step(const r3_adamw* config, const r3_adamw_tensor* tensors, int32_t n_tensors,
                     const float* grad_scale, const float* scalars, const int32_t* dev_status,
                     cudaStream_t cs) {
    AdamScalars s = {};
    s.beta1 = (float)config->beta1;
    s.one_beta1 = (float)(1.0 - config->beta1);
    s.beta2 = (float)config->beta2;
    s.one_beta2 = (float)(1.0 - config->beta2);
    s.eps = (float)config->eps;
    s.lr = (float)config->lr;
    s.bias1 = (float)(1.0 / (1.0 - std::pow(config->beta1, (double)config->step)));
    s.bias2 = (float)(1.0 / std::sqrt(1.0 - std::pow(config->beta2, (double)config->step)));
    s.one = 1.f;
    s.grad_scale = grad_scale;
    s.dynamic = scalars;
    s.dev_status = dev_status;
    return config->grad_dtype == R3_F32 ? launch_adamw<float>(config, s, tensors, n_tensors, cs)
                                        : launch_adamw<__nv_bfloat16>(config, s, tensors, n_tensors, cs);
}

}  // namespace r3

extern "C" r3_status r3_adamw_step(const r3_adamw* config, const r3_adamw_tensor* tensors,
                                   int32_t n_tensors, const float* grad_scale, const float* scalars,
                                   void* stream) {
    const r3_status st = r3::check_adamw_call(config, tensors, n_tensors, grad_scale, scalars);
    if (st != R3_OK) return st;
    return r3::adamw_step(config, tensors, n_tensors, grad_scale, scalars, nullptr,
                          static_cast<cudaStream_t>(stream));
}
