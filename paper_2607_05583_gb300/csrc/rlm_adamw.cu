// rlm_adamw.cu -- one AdamW step over many tensors in one launch.
//
//   g' = s g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
//   p = p (1 - lr wd) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Bound by memory: 28 bytes a value with fp32 weights, gradients and moments, 10 with bf16
// weights and gradients and 8-bit moments.  Every tensor is cut into chunks of kChunk
// values; a block takes one chunk, found by bisection in the tensors' running chunk counts.
// The tensors' pointers travel in the kernel's parameters (up to kMaxTensors a launch), so
// a step copies nothing to the device first.  A thread holds 8 values in registers, moved
// by 16-byte accesses; tensors whose pointers or ends do not allow that go value by value.
//
// 8-bit moments.  Blocks of 256 values share a power-of-two scale 2^(e - 8), 2^e the first
// power of two above the block's largest magnitude, so scaling is exact; the values are
// kept as 8-bit floats with 3 mantissa bits (relative step 2^-3 over 17 binades), m signed
// and sqrt(v) in place of v, which halves the binades v needs.  A sqrt(v) that would round
// to zero is kept at the smallest code: a zero under a nonzero m would let the step grow
// to m / eps.  The step itself uses the moments before they are rounded.  A warp's 32 x 8
// values are one block.
//
// The products and sums of m and v are rounded one by one (no contraction), so scales do
// not depend on how a compiler fuses them.  sqrt and the quotient of the step are the
// approximate instructions (2^-22): with the exact sequences the 8-bit step was bound by
// its instructions (379 us at 120 M values, against 178 us for its bytes).
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>

#include "rlm_device.cuh"
#include "rlm_internal.h"

namespace rlm {

namespace {

constexpr int kBlock = RLM_ADAMW_BLOCK;         // values that share a scale
constexpr int kThreads = 256;
constexpr int kChunk = 2048;                    // values of a block: 8 a thread
constexpr int kMaxTensors = 400;

struct Entry {
    void *p, *g, *m, *v;
    float *master;          // nullable
    float *m_scale, *v_scale;
    int64_t n;
};
struct StepArgs {
    const float *grad_scale;        // nullable
    float beta1, one_minus_beta1, beta2, one_minus_beta2, inv_sqrt_bc2, eps, decay, step_size;
    int count;
    unsigned first[kMaxTensors + 1];        // chunks before each tensor
    Entry t[kMaxTensors];
};
static_assert(sizeof(StepArgs) <= 32764, "kernel parameter space");

template <typename T>
struct Eight;
template <>
struct Eight<float> {
    static __device__ __forceinline__ void load(const float *p, float (&v)[8]) {
        const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
    static __device__ __forceinline__ void store(float *p, const float (&v)[8]) {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    }
};
template <>
struct Eight<__nv_bfloat16> {
    static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&v)[8]) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(w[0], w[1], w[2], w[3]));
    }
};

// The first `n` (at most 8) values at p; vec: 8 values by 16-byte accesses.
template <typename T>
__device__ __forceinline__ void load8(const T *p, int n, bool vec, float (&v)[8]) {
    if (vec) {
        Eight<T>::load(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? ld_elem(p + i) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store8(T *p, int n, bool vec, const float (&v)[8]) {
    if (vec) {
        Eight<T>::store(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) st_elem(p + i, v[i]);
}

// 8 codes, as values of their block's scale.
__device__ __forceinline__ void load_codes(const uint8_t *p, int n, bool vec, float (&v)[8]) {
    uint32_t w[2] = {0u, 0u};
    if (vec) {
        const uint2 a = __ldcs(reinterpret_cast<const uint2 *>(p));
        w[0] = a.x, w[1] = a.y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) w[i >> 2] |= (uint32_t)p[i] << 8 * (i & 3);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> 16 * (i & 1)), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void store_codes(uint8_t *p, int n, bool vec, const float (&v)[8]) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[2 * i], v[2 * i + 1]), __NV_SATFINITE, __NV_E4M3)
                     << 16 * (i & 1);
    if (vec) {
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(w[0], w[1]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = (uint8_t)(w[i >> 2] >> 8 * (i & 3));
}

// The bits of the largest magnitude among the warp's values.
__device__ __forceinline__ unsigned block_top(const float (&v)[8]) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    return __reduce_max_sync(~0u, top);
}
// e of the block scale 2^(e - 8): the least e with top < 2^e, at least -100 (so both
// 2^(e - 8) and its inverse are normal).
__device__ __forceinline__ int exponent(unsigned top) { return max((int)(top >> 23) - 126, -100); }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

__device__ __forceinline__ f32x2 pair(const float *v) { return pack(make_float2(v[0], v[1])); }
__device__ __forceinline__ f32x2 twice(float v) { return pack(make_float2(v, v)); }
__device__ __forceinline__ void unpair(f32x2 p, float *v) {
    const float2 f = unpack(p);
    v[0] = f.x;
    v[1] = f.y;
}

template <typename P, typename G, bool kMaster, bool k8Bit>
__global__ void __launch_bounds__(kThreads) k_adamw(const __grid_constant__ StepArgs a) {
    // The tensor whose chunks this block's index falls into.
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.first[mid] <= blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const Entry &e = a.t[lo];
    const int64_t at = (int64_t)(blockIdx.x - a.first[lo]) * kChunk + threadIdx.x * 8;
    const int n = (int)min((int64_t)8, max((int64_t)0, e.n - at));
    float scale = 1.f;
    if (a.grad_scale) {
        scale = __ldg(a.grad_scale);
        if (!isfinite(scale)) return;           // an overflowed step: nothing changes
    }
    P *p = static_cast<P *>(e.p) + at;
    const G *g = static_cast<const G *>(e.g) + at;
    const bool whole = n == 8;
    auto wide = [&](const void *q, unsigned to) { return whole && (reinterpret_cast<uintptr_t>(q) & (to - 1)) == 0; };
    float gv[8], m[8], v[8], w[8];
    load8(g, n, wide(g, 16), gv);
    float *master = kMaster ? e.master + at : nullptr;
    if constexpr (kMaster) load8(master, n, wide(master, 16), w); else load8(p, n, wide(p, 16), w);
    uint8_t *m8 = static_cast<uint8_t *>(e.m) + at, *v8 = static_cast<uint8_t *>(e.v) + at;
    float *mf = static_cast<float *>(e.m) + at, *vf = static_cast<float *>(e.v) + at;
    if constexpr (k8Bit) {
        const int64_t blk = at / kBlock;
        const float ms = n > 0 ? e.m_scale[blk] : 0.f, vs = n > 0 ? e.v_scale[blk] : 0.f;
        load_codes(m8, n, wide(m8, 8), m);
        load_codes(v8, n, wide(v8, 8), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] *= ms;
            const float r = v[i] * vs;
            v[i] = __fmul_rn(r, r);
        }
    } else {
        load8(mf, n, wide(mf, 16), m);
        load8(vf, n, wide(vf, 16), v);
    }
    float root[8];
    const f32x2 b1 = twice(a.beta1), c1 = twice(a.one_minus_beta1), b2 = twice(a.beta2), c2 = twice(a.one_minus_beta2);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        f32x2 gs = pair(gv + i);
        if (a.grad_scale) gs = mul2(gs, twice(scale));
        const f32x2 m2 = add2(mul2(b1, pair(m + i)), mul2(c1, gs));
        const f32x2 v2 = add2(mul2(b2, pair(v + i)), mul2(c2, mul2(gs, gs)));
        unpair(m2, m + i);
        unpair(v2, v + i);
        float r[2];
        asm("sqrt.approx.f32 %0, %1;" : "=f"(root[i]) : "f"(v[i]));
        asm("sqrt.approx.f32 %0, %1;" : "=f"(root[i + 1]) : "f"(v[i + 1]));
        unpair(fma2(pair(root + i), twice(a.inv_sqrt_bc2), twice(a.eps)), r);
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r[0]));
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r[1]));
        unpair(fma2(twice(-a.step_size), mul2(m2, pair(r)), mul2(pair(w + i), twice(a.decay))), w + i);
    }
    store8(p, n, wide(p, 16), w);
    if constexpr (kMaster) store8(master, n, wide(master, 16), w);
    if constexpr (k8Bit) {
        const int em = exponent(block_top(m)), ev = exponent(__float_as_uint(__fsqrt_rn(__uint_as_float(block_top(v)))));
        const float im = power_of_two(8 - em), iv = power_of_two(8 - ev);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] *= im;
            root[i] = root[i] > 0.f ? fmaxf(root[i] * iv, 0x1p-9f) : root[i] * iv;
        }
        store_codes(m8, n, wide(m8, 8), m);
        store_codes(v8, n, wide(v8, 8), root);
        if ((threadIdx.x & 31) == 0 && n > 0) {
            e.m_scale[at / kBlock] = power_of_two(em - 8);
            e.v_scale[at / kBlock] = power_of_two(ev - 8);
        }
    } else {
        store8(mf, n, wide(mf, 16), m);
        store8(vf, n, wide(vf, 16), v);
    }
}

using StepKernel = void (*)(const StepArgs);
template <typename P, typename G>
StepKernel step_kernel(bool master, bool bits8) {
    if constexpr (sizeof(P) == 2) {
        if (master) return bits8 ? k_adamw<P, G, true, true> : k_adamw<P, G, true, false>;
    }
    return bits8 ? k_adamw<P, G, false, true> : k_adamw<P, G, false, false>;
}

}  // namespace

cudaError_t adamw_step(const rlm_adamw_tensor *tensors, int count, rlm_dtype param, rlm_dtype grad, bool master, int bits,
                       const rlm_adamw_hyper &h, const float *grad_scale, cudaStream_t st) {
    const StepKernel fn = param == RLM_BF16
                              ? (grad == RLM_BF16 ? step_kernel<__nv_bfloat16, __nv_bfloat16>(master, bits == 8)
                                                  : step_kernel<__nv_bfloat16, float>(master, bits == 8))
                              : (grad == RLM_BF16 ? step_kernel<float, __nv_bfloat16>(master, bits == 8)
                                                  : step_kernel<float, float>(master, bits == 8));
    StepArgs a;
    const double bc1 = 1.0 - std::pow(h.beta1, (double)h.step), bc2 = 1.0 - std::pow(h.beta2, (double)h.step);
    a.grad_scale = grad_scale;
    a.beta1 = (float)h.beta1;
    a.one_minus_beta1 = (float)(1.0 - h.beta1);
    a.beta2 = (float)h.beta2;
    a.one_minus_beta2 = (float)(1.0 - h.beta2);
    a.inv_sqrt_bc2 = (float)(1.0 / std::sqrt(bc2));
    a.eps = (float)h.eps;
    a.decay = (float)(1.0 - h.lr * h.weight_decay);
    a.step_size = (float)(h.lr / bc1);
    for (int i = 0; i < count;) {
        a.count = 0;
        unsigned chunks = 0;
        for (; i < count && a.count < kMaxTensors; ++i) {
            const rlm_adamw_tensor &t = tensors[i];
            const int64_t c = (t.n + kChunk - 1) / kChunk;
            if (a.count > 0 && c > (int64_t)0x7fffffff - chunks) break;     // the grid's limit
            a.first[a.count] = chunks;
            a.t[a.count] = {t.param, const_cast<void *>(t.grad), t.exp_avg, t.exp_avg_sq, t.master, t.exp_avg_scale,
                            t.exp_avg_sq_scale, t.n};
            ++a.count;
            chunks += (unsigned)c;
        }
        a.first[a.count] = chunks;
        fn<<<chunks, kThreads, 0, st>>>(a);
        count_launches(1);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace rlm
