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
#include <new>
#include <utility>
#include <vector>

#include "r3_common.cuh"
#include "r3_internal.h"

namespace r3 {

constexpr int kAdamBlock = 256;                     // elements per scale
constexpr int kAdamThreads = 256;
constexpr int kAdamWarps = kAdamThreads / 32;
constexpr int kAdamPerWarp = 4;                     // blocks per warp and chunk
constexpr int kAdamChunk = kAdamBlock * kAdamWarps * kAdamPerWarp;
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
    int tensors;
};
template <int CAP> struct AdamTable {
    AdamScalars s;
    AdamTensor t[CAP];
};

// Four consecutive elements as float32.
template <typename T> __device__ __forceinline__ float4 load4(const T* p);
template <> __device__ __forceinline__ float4 load4<float>(const float* p) {
    return *reinterpret_cast<const float4*>(p);
}
template <> __device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16* p) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
    const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void store4(float* p, const float* f) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* f) {
    __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
    uint2 u;
    u.x = *reinterpret_cast<uint32_t*>(&a);
    u.y = *reinterpret_cast<uint32_t*>(&b);
    *reinterpret_cast<uint2*>(p) = u;
}
// Elements at, .. at + 3 of an array of n; 0 behind its end.
template <typename T>
__device__ __forceinline__ void take4(const T* p, long long at, long long n, bool full, float* f) {
    if (full) {
        const float4 v = load4<T>(p + at);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = at + i < n ? to_f32(p[at + i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void put4(T* p, long long at, long long n, bool full, const float* f) {
    if (full) {
        store4(p + at, f);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at + i < n) p[at + i] = from_f32<T>(f[i]);
    }
}
__device__ __forceinline__ void unpack_codes(uint32_t c, float scale, float* f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c >> (16 * i)), __NV_E4M3);
        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&h));
        f[2 * i] = t.x * scale;                     // a power of two: exact
        f[2 * i + 1] = t.y * scale;
    }
}
__device__ __forceinline__ uint32_t pack_codes(const float* f, float inv) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[0] * inv, f[1] * inv), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[2] * inv, f[3] * inv), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ uint32_t take_codes(const uint8_t* p, long long at, long long n, bool full) {
    if (full) return *reinterpret_cast<const uint32_t*>(p + at);
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) c |= (uint32_t)p[at + i] << (8 * i);
    return c;
}
__device__ __forceinline__ void put_codes(uint8_t* p, long long at, long long n, bool full, uint32_t c) {
    if (full) {
        *reinterpret_cast<uint32_t*>(p + at) = c;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at + i < n) p[at + i] = (uint8_t)(c >> (8 * i));
    }
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
__device__ __forceinline__ float quantise(const float (&f)[8], uint32_t (&codes)[2]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
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
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        codes[h] = pack_codes(f + 4 * h, inv);
        if (ROOT) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (f[4 * h + i] > 0.f && (codes[h] >> (8 * i) & 0xffu) == 0u) codes[h] |= 1u << (8 * i);
        }
        if (!clean) {
#pragma unroll
            for (int i = 0; i < 4; ++i)             // 0x7f: NaN
                if ((__float_as_uint(f[4 * h + i]) & 0x7f800000u) == 0x7f800000u)
                    codes[h] |= 0x7fu << (8 * i);
        }
    }
    return __uint_as_float(e << 23);
}

template <typename P, typename G, bool MASTER, bool BITS8, int CAP>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamTable<CAP> a) {
    const float gs = a.s.grad_scale ? *a.s.grad_scale : 1.f;
    if (!(fabsf(gs) <= 3.402823466e38f)) return;    // NaN or infinite: the step is skipped
    const float lr = a.s.dynamic ? a.s.dynamic[0] : a.s.lr;
    const float bias1 = a.s.dynamic ? a.s.dynamic[1] : a.s.bias1;
    const float bias2 = a.s.dynamic ? a.s.dynamic[2] : a.s.bias2;
    const float step = lr * bias1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (unsigned chunk = blockIdx.x; chunk < a.s.chunks; chunk += gridDim.x) {
        int lo = 0, hi = a.s.tensors - 1;           // the last tensor that starts at or before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.t[mid].first <= chunk) lo = mid;
            else hi = mid - 1;
        }
        const AdamTensor& t = a.t[lo];
        const long long n = t.n;
        const float keep = 1.f - lr * t.decay;
        P* param = static_cast<P*>(t.param);
        const G* grad = static_cast<const G*>(t.grad);
        const long long block0 = (long long)(chunk - t.first) * (kAdamWarps * kAdamPerWarp) + warp;
#pragma unroll 1
        for (int k = 0; k < kAdamPerWarp; ++k) {
            const long long block = block0 + k * kAdamWarps, at = block * kAdamBlock + 4 * lane;
            if (block * kAdamBlock >= n) break;
            const bool full = (block + 1) * kAdamBlock <= n;
            float w[8], g[8], m[8], v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const long long i = at + 128 * h;
                if (MASTER) take4<float>(t.master, i, n, full, w + 4 * h);
                else take4<P>(param, i, n, full, w + 4 * h);
                take4<G>(grad, i, n, full, g + 4 * h);
                if (BITS8) {
                    unpack_codes(take_codes(static_cast<const uint8_t*>(t.m), i, n, full),
                                 t.m_scale[block], m + 4 * h);
                    unpack_codes(take_codes(static_cast<const uint8_t*>(t.v), i, n, full),
                                 t.v_scale[block], v + 4 * h);
                } else {
                    take4<float>(static_cast<const float*>(t.m), i, n, full, m + 4 * h);
                    take4<float>(static_cast<const float*>(t.v), i, n, full, v + 4 * h);
                }
            }
            float root[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gi = __fmul_rn(g[i], gs);
                const float v0 = BITS8 ? __fmul_rn(v[i], v[i]) : v[i];
                m[i] = __fadd_rn(__fmul_rn(a.s.beta1, m[i]), __fmul_rn(a.s.one_beta1, gi));
                v[i] = __fadd_rn(__fmul_rn(a.s.beta2, v0), __fmul_rn(a.s.one_beta2, __fmul_rn(gi, gi)));
                root[i] = __fsqrt_rn(v[i]);
                // a quotient a few units of 2^-24 off moves the weight by far less than its rounding
                w[i] = fmaf(-step, __fdividef(m[i], fmaf(root[i], bias2, a.s.eps)), w[i] * keep);
            }
            uint32_t mc[2], vc[2];
            if (BITS8) {
                const float ms = quantise<false>(m, mc), vs = quantise<true>(root, vc);
                if (lane == 0) {
                    t.m_scale[block] = ms;
                    t.v_scale[block] = vs;
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const long long i = at + 128 * h;
                if (MASTER) put4(t.master, i, n, full, w + 4 * h);
                put4(param, i, n, full, w + 4 * h);
                if (BITS8) {
                    put_codes(static_cast<uint8_t*>(t.m), i, n, full, mc[h]);
                    put_codes(static_cast<uint8_t*>(t.v), i, n, full, vc[h]);
                } else {
                    put4(static_cast<float*>(t.m), i, n, full, m + 4 * h);
                    put4(static_cast<float*>(t.v), i, n, full, v + 4 * h);
                }
            }
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
        long long chunks = 0;
        int k = 0;
        for (; done < count && k < CAP; ++done) {
            const r3_adamw_tensor& t = ts[done];
            if (t.n == 0) continue;
            const long long more = (t.n + kAdamChunk - 1) / kAdamChunk;
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
        a.s.chunks = (unsigned)chunks;
        const long long most = 8LL * sm_count();
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
