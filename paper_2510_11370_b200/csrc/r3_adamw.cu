// One AdamW step over many tensors in one launch: what follows the weight gradients of the
// replayed layers.  Per element, with g the gradient times grad_scale:
//   m = beta1 m + (1 - beta1) g          v = beta2 v + (1 - beta2) g^2
//   w = w (1 - lr decay) - lr / (1 - beta1^t)  m / ( sqrt(v) / sqrt(1 - beta2^t) + eps )
//
// Bound by HBM (12.06 bytes an element for bf16 weights, float32 gradients and 8-bit states; 28 for
// float32 with 32-bit states).  States of 8 bits are kept in blocks of 256 elements with one scale:
// e4m3 codes times the smallest power of two (at least 2^-126) that brings the block's largest
// magnitude to 448 or less, so that scaling is exact both ways and the one rounding is the code's.
// The second moment is kept as its square root, which halves the range its codes have to span; a
// root above zero is never kept as zero, because the update divides by it (the smallest code is the
// safe side: a smaller step).  Every operation that leads to a stored state is rounded to float32
// by itself (no fused multiply-add), so the states are a function of the inputs alone and do not
// depend on how a compiler contracts the expressions.
//
// A warp takes a block: lane l holds elements 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3, so that
// every load and store of the warp covers consecutive bytes whatever the type's width, and one
// warp-wide maximum per state gives the scale.  The table of tensors travels in the kernel's
// parameters: no workspace, no copy, and a captured launch keeps its own.
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
constexpr int kAdamCtas = 4;                        // resident per SM at 64 registers a thread
constexpr int kAdamMaxPerWarp = 16;                 // blocks per warp and chunk
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
    unsigned first;                                 // first chunk of this tensor
};
struct AdamScalars {
    float beta1, one_beta1, beta2, one_beta2, eps, lr, bias1, bias2;
    const float* grad_scale;
    const float* dynamic;                           // {lr, bias1, bias2} on the device, or null
    unsigned chunks;
    int tensors, per_warp;
};
template <int CAP> struct AdamTable {
    AdamScalars s;
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
// A lane's eight elements of a block: 4 l .. and 128 + 4 l ..; `left` elements of the tensor follow
// from the block's first on (only looked at where FULL is false; what lies behind reads as 0 and is
// not written).
template <bool FULL, typename T>
__device__ __forceinline__ void take(const T* p, int lane, int left, Four<T> (&f)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = 128 * h + 4 * lane;
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
template <bool FULL, typename T>
__device__ __forceinline__ void put(T* p, int lane, int left, const Four<T> (&f)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = 128 * h + 4 * lane;
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
__device__ __forceinline__ float max_abs(float a, float b) {      // a NaN stays one
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
// Biased exponent of the block's scale from the bits of its largest magnitude f 2^e, f in [1, 2):
// 448 = 1.75 2^8, so e - 8, and one more where f > 1.75 (the addition carries then); at least 1.
__device__ __forceinline__ uint32_t scale_exponent(uint32_t bits) {
    const uint32_t e = (bits + 0x1fffffu) >> 23;
    return e > 9u ? e - 8u : 1u;
}
// The eight codes of a lane and the scale of its block.  ROOT: values are >= 0 and none above zero
// becomes code 0.
template <bool ROOT>
__device__ __forceinline__ float quantise(const float (&f)[8], Four<uint8_t> (&codes)[2]) {
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max_abs(big, f[i]);
    uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(big));
    const bool clean = top < 0x7f800000u;
    if (!clean) {                                   // the scale is that of the finite elements
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = __float_as_uint(f[i]) & 0x7fffffffu;
            if (b < 0x7f800000u) top = max(top, b);
        }
        top = __reduce_max_sync(0xffffffffu, top);
    }
    const uint32_t e = scale_exponent(top);
    const float inv = __uint_as_float((254u - e) << 23);
    float least = f[0];
    if (ROOT) {
#pragma unroll
        for (int i = 1; i < 8; ++i) least = fminf(least, f[i]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = f[4 * h + i] * inv;
        codes[h].pack(q);
        if (ROOT) {
            // 1 in every byte that is 0 (no code here has its top bit set, so nothing carries)
            const uint32_t zeros = (((codes[h].v + 0x7f7f7f7fu) & 0x80808080u) ^ 0x80808080u) >> 7;
            if (least > 0.f) {
                codes[h].v |= zeros;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (f[4 * h + i] > 0.f) codes[h].v |= zeros & (0xffu << (8 * i));
            }
        }
        if (!clean) {
#pragma unroll
            for (int i = 0; i < 4; ++i)             // 0x7f: NaN
                if ((__float_as_uint(f[4 * h + i]) & 0x7f800000u) == 0x7f800000u)
                    codes[h].v |= 0x7fu << (8 * i);
        }
    }
    return __uint_as_float(e << 23);
}

struct AdamRates {                                  // what the whole launch shares
    float beta1, one_beta1, beta2, one_beta2, eps, bias2, step, keep, gs;
};

// One block's values on their way: loaded a block ahead where the states are codes (the arithmetic
// around the codes is long enough to leave the memory idle otherwise; with 32-bit states the
// occupancy does as well, and the registers are better spent on it).
template <typename P, typename G, bool MASTER, bool BITS8> struct AdamBlock {
    typedef typename std::conditional<MASTER, float, P>::type Wt;
    typedef typename std::conditional<BITS8, uint8_t, float>::type St;
    Four<Wt> w[2];
    Four<G> g[2];
    Four<St> m[2], v[2];
    float ms, vs;

    template <bool FULL>
    __device__ __forceinline__ void load(const AdamTensor& t, long long block, int lane, int left) {
        const long long at = block * kAdamBlock;
        take<FULL>((MASTER ? reinterpret_cast<const Wt*>(t.master) : static_cast<const Wt*>(t.param)) + at,
                   lane, left, w);
        take<FULL>(static_cast<const G*>(t.grad) + at, lane, left, g);
        take<FULL>(static_cast<const St*>(t.m) + at, lane, left, m);
        take<FULL>(static_cast<const St*>(t.v) + at, lane, left, v);
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
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float gi = __fmul_rn(fg[i], a.gs);
            float m0 = fm[i], v0 = fv[i];
            if (BITS8) {
                m0 *= ms;                           // powers of two: exact
                v0 *= vs;
                v0 = __fmul_rn(v0, v0);
            }
            fm[i] = __fadd_rn(__fmul_rn(a.beta1, m0), __fmul_rn(a.one_beta1, gi));
            fv[i] = __fadd_rn(__fmul_rn(a.beta2, v0), __fmul_rn(a.one_beta2, __fmul_rn(gi, gi)));
            root[i] = __fsqrt_rn(fv[i]);
            // a quotient a few units of 2^-24 off moves the weight by far less than its rounding
            float inv;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(fmaf(root[i], a.bias2, a.eps)));
            fw[i] = fmaf(-a.step, fm[i] * inv, fw[i] * a.keep);
        }
        if constexpr (BITS8) {
            ms = quantise<false>(fm, m);
            vs = quantise<true>(root, v);
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
        put<FULL>(static_cast<St*>(t.m) + at, lane, left, m);
        put<FULL>(static_cast<St*>(t.v) + at, lane, left, v);
        Four<P> p[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) p[h].pack(fw + 4 * h);
        put<FULL>(static_cast<P*>(t.param) + at, lane, left, p);
        if constexpr (MASTER) {
#pragma unroll
            for (int h = 0; h < 2; ++h) w[h].pack(fw + 4 * h);
            put<FULL>(t.master + at, lane, left, w);
        }
    }
};

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamTable<CAP> a) {
    AdamRates r;
    r.gs = a.s.grad_scale ? *a.s.grad_scale : 1.f;
    if (!(fabsf(r.gs) <= 3.402823466e38f)) return;  // NaN or infinite: the step is skipped
    const float lr = a.s.dynamic ? a.s.dynamic[0] : a.s.lr;
    r.step = lr * (a.s.dynamic ? a.s.dynamic[1] : a.s.bias1);
    r.bias2 = a.s.dynamic ? a.s.dynamic[2] : a.s.bias2;
    r.beta1 = a.s.beta1;
    r.one_beta1 = a.s.one_beta1;
    r.beta2 = a.s.beta2;
    r.one_beta2 = a.s.one_beta2;
    r.eps = a.s.eps;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (unsigned chunk = blockIdx.x; chunk < a.s.chunks; chunk += gridDim.x) {
        int lo = 0, hi = a.s.tensors - 1;           // the last tensor that starts at or before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.t[mid].first <= chunk) lo = mid;
            else hi = mid - 1;
        }
        const AdamTensor t = a.t[lo];
        r.keep = 1.f - lr * t.decay;
        // the warps of a CTA take the chunk's blocks in turn
        long long block = (long long)(chunk - t.first) * (kAdamWarps * a.s.per_warp) + warp;
        const long long whole = t.n / kAdamBlock;   // blocks without a ragged end
        const long long end = min(whole, block + (long long)kAdamWarps * a.s.per_warp);
        AdamBlock<P, G, MASTER, BITS8> b;
        if (BITS8) {
            if (block < end) b.template load<true>(t, block, lane, kAdamBlock);
            while (block < end) {
                AdamBlock<P, G, MASTER, BITS8> now = b;
                const long long next = block + kAdamWarps;
                if (next < end) b.template load<true>(t, next, lane, kAdamBlock);
                now.template update<true>(t, block, lane, kAdamBlock, r);
                block = next;
            }
        } else {
            for (; block < end; block += kAdamWarps) {
                b.template load<true>(t, block, lane, kAdamBlock);
                b.template update<true>(t, block, lane, kAdamBlock, r);
            }
        }
        // the warp whose turn it is takes the ragged end
        const long long past = (long long)(chunk - t.first + 1) * (kAdamWarps * a.s.per_warp);
        if (block == whole && block < past && t.n > whole * kAdamBlock) {
            const int left = (int)(t.n - whole * kAdamBlock);
            b.template load<false>(t, block, lane, left);
            b.template update<false>(t, block, lane, left, r);
        }
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
// Two entries on the same memory would be updated at once, in no order.
static r3_status check_distinct(const r3_adamw* c, const r3_adamw_tensor* ts, int32_t count) {
    try {
        std::vector<std::pair<uintptr_t, uintptr_t>> r;
        r.reserve(count);
        const uintptr_t size = c->param_dtype == R3_BF16 ? 2 : 4;
        for (int32_t i = 0; i < count; ++i)
            if (ts[i].n > 0) {
                const uintptr_t p = reinterpret_cast<uintptr_t>(ts[i].param);
                r.emplace_back(p, p + (uintptr_t)ts[i].n * size);
            }
        std::sort(r.begin(), r.end());
        for (size_t i = 1; i < r.size(); ++i)
            if (r[i].first < r[i - 1].second) return R3_ERR_INVALID_ARG;
        return R3_OK;
    } catch (...) {                                 // out of host memory
        return R3_ERR_INVALID_ARG;
    }
}

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
static r3_status launch_adamw(const AdamScalars& s, const r3_adamw_tensor* ts, int count, cudaStream_t cs) {
    AdamTable<CAP> a;
    a.s = s;
    for (int done = 0; done < count;) {
        // Blocks per warp and chunk: as many as leave the resident warps four chunks each, so that a
        // long run of blocks hides its loads and a short list still spreads over the GPU.
        long long blocks = 0;
        for (int i = done, k = 0; i < count && k < CAP; ++i) {
            blocks += (ts[i].n + kAdamBlock - 1) / kAdamBlock;
            k += ts[i].n > 0;
        }
        const long long share = blocks / (4LL * kAdamWarps * kAdamCtas * sm_count());
        const int per_warp = share < 1 ? 1 : share > kAdamMaxPerWarp ? kAdamMaxPerWarp : (int)share;
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
                      t.exp_avg_sq_scale, t.n, t.weight_decay, (unsigned)chunks};
            chunks += more;
            ++k;
        }
        if (k == 0) break;
        a.s.tensors = k;
        a.s.per_warp = per_warp;
        a.s.chunks = (unsigned)chunks;
        const long long most = (long long)kAdamCtas * sm_count();
        adamw_kernel<P, G, MASTER, BITS8, CAP>
            <<<(unsigned)(chunks < most ? chunks : most), kAdamThreads, 0, cs>>>(a);
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

}  // namespace r3

extern "C" r3_status r3_adamw_step(const r3_adamw* config, const r3_adamw_tensor* tensors,
                                   int32_t n_tensors, const float* grad_scale, const float* scalars,
                                   void* stream) {
    r3_status st = r3::check_adamw(config, tensors, n_tensors);
    if (st != R3_OK) return st;
    if (!r3::aligned(grad_scale, 4) || !r3::aligned(scalars, 4)) return R3_ERR_INVALID_ARG;
    if ((st = r3::check_distinct(config, tensors, n_tensors)) != R3_OK) return st;
    r3::AdamScalars s = {};
    s.beta1 = (float)config->beta1;
    s.one_beta1 = (float)(1.0 - config->beta1);
    s.beta2 = (float)config->beta2;
    s.one_beta2 = (float)(1.0 - config->beta2);
    s.eps = (float)config->eps;
    s.lr = (float)config->lr;
    s.bias1 = (float)(1.0 / (1.0 - std::pow(config->beta1, (double)config->step)));
    s.bias2 = (float)(1.0 / std::sqrt(1.0 - std::pow(config->beta2, (double)config->step)));
    s.grad_scale = grad_scale;
    s.dynamic = scalars;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    return config->grad_dtype == R3_F32
               ? r3::launch_adamw<float>(config, s, tensors, n_tensors, cs)
               : r3::launch_adamw<__nv_bfloat16>(config, s, tensors, n_tensors, cs);
}
