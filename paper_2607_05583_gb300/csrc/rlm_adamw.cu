// rlm_adamw.cu -- one AdamW step over many tensors in one launch.
//
//   g' = s g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
//   p = p (1 - lr wd) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Bound by memory: 28 bytes a value with fp32 weights, gradients and moments, 10 with bf16
// weights and gradients and 8-bit moments.  Every tensor is cut into chunks of kChunk
// values; a block takes one chunk, found by one warp's bisection in the tensors' running
// chunk counts.
// The tensors' pointers travel in the kernel's parameters (up to kMaxTensors a launch), so
// a step copies nothing to the device first.  A thread holds 8 values in registers, moved
// by 16-byte accesses; tensors whose pointers do not allow that, and ends, go value by value.
//
// 8-bit moments.  Blocks of 256 values share a power-of-two scale 2^(e - 8), 2^e the first
// power of two above the block's largest magnitude, so scaling is exact; the values are
// kept as 8-bit floats with 3 mantissa bits (relative step 2^-3 over 14 binades, and three more
// at the fixed step 2^-9 of the scale), m signed
// and sqrt(v) in place of v, which halves the binades v needs.  A sqrt(v) that would round
// to zero is kept at the smallest code: a zero under a nonzero m would let the step grow
// to m / eps.  The step itself uses the moments before they are rounded.  A warp's 32 x 8
// values are one block.
//
// Rounding the codes.  A step moves sqrt(v) by at most 1 - sqrt(beta2) of itself, 2.5 % at 0.95
// and 0.05 % at 0.999, and codes lie 6 to 12 % apart: rounded to nearest it goes back to the code
// that it came from, and never decays.  By draw (kDraw), a value less than 3/4 of a code from the
// one it came from goes up or down by chance, with the mean that it has; over many steps the
// moments then follow the 32-bit ones (N(0, 1) gradients, 1000 steps: mean sqrt(v) within 1.5 %;
// with nearest codes 2.0 times too large at beta2 = 0.95 and 0.4 at 0.999).  The draw is a hash of
// the step, the tensor's place and the value's index: the same call gives the same codes.  Larger
// changes go to the nearest code, whose error is half of the draw's.  A zero m is left by chance
// where the gradient is one that m could hold to all its bits (2^-14 of the block's largest m),
// below that only by a change that is nearer to the smallest code.
//
// The products and sums of m and v are rounded one by one: an 8-bit m and a bf16 gradient have
// few bits, so 0.9 m + 0.1 g meets the ties of the 4-bit codes about once in 500 values, and a
// fused product would decide them (and with them whole steps) otherwise than its definition.
// Scalar instructions, because mul and add on packed pairs were fused.  sqrt and the
// quotient of the step are the approximate instructions (2^-22): with the exact sequences
// the 8-bit step, which its instructions bound (82 % of issue slots), took 379 us at 120 M
// values against 211 us now (bf16 weights, codes to nearest) and 178 us for its bytes.  By draw it
// takes 337 us (370 with fp32 weights, 376 with masters): some 30 instructions a value more.  The
// 32-bit steps run at the copy rate: 478 us for 3.36 GB (fp32, and bf16 with masters), 7.0 TB/s.
#include <cuda_fp8.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "rlm_device.cuh"
#include "rlm_internal.h"

namespace rlm {

namespace {

constexpr int kBlock = RLM_ADAMW_BLOCK;         // values that share a scale
constexpr int kThreads = 256;
// Values of a thread block: 8 a thread.  Several rounds a thread, the next round's loads issued
// before this one's arithmetic or not, measured slower (the blocks at work then spread over more
// of each buffer): 276 against 227 us for the 8-bit step (as it was then) at 120 M values with
// two rounds, 491 against 478 us for the fp32 one with four.
constexpr int kChunk = 8 * kThreads;
constexpr int kMaxTensors = 400;

struct Entry {
    void *p, *g, *m, *v;
    float *master;          // nullable
    float *m_scale, *v_scale;
    int64_t n;
    int wide;               // every buffer allows 16-byte (codes: 8-byte) accesses
};
struct StepArgs {
    const float *grad_scale;        // nullable
    float beta1, one_minus_beta1, beta2, one_minus_beta2, inv_sqrt_bc2, eps, decay, step_size;
    int count;
    uint32_t draw, before;                  // 8-bit moments: hash of the step; the call's tensors in earlier launches
    float leave_zero;                       // (1 - beta1) of the smallest normal code
    unsigned first[kMaxTensors + 1];        // chunks before each tensor
    Entry t[kMaxTensors];
};
static_assert(sizeof(StepArgs) <= 32764, "kernel parameter space");

// Eight values as they lie in memory, so that a load can be issued long before its use.
template <typename T>
struct Eight {
    static constexpr int kWords = 2 * (int)sizeof(T);
    uint32_t w[kWords];
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = __float_as_uint(v[i]);
            } else {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&b);
            }
        }
    }
};
// Eight codes, as values of their block's scale.
struct Codes {
    static constexpr int kWords = 2;
    uint32_t w[2];
    // Values i and i + 1.
    __device__ __forceinline__ f32x2 two(int i) const {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 2] >> 8 * (i & 3)), __NV_E4M3);
        return pack(__half22float2(*reinterpret_cast<const __half2 *>(&h)));
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        w[0] = w[1] = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[2 * i], v[2 * i + 1]), __NV_SATFINITE, __NV_E4M3)
                         << 16 * (i & 1);
    }
};
// The first n (at most 8) values at p, the others zero: 16-byte (codes: 8-byte) accesses where
// `wide`, else value by value.  E: bytes of a value.
template <typename V, int E>
__device__ __forceinline__ V load8(const void *p, int n, bool wide) {
    V v;
    constexpr int kBytes = 4 * V::kWords, kWide = kBytes < 16 ? kBytes : 16;
    if (wide) {
#pragma unroll
        for (int i = 0; i < kBytes / kWide; ++i) {
            if constexpr (kWide == 16) {
                const uint4 q = load_once(static_cast<const uint4 *>(p) + i);
                v.w[4 * i] = q.x, v.w[4 * i + 1] = q.y, v.w[4 * i + 2] = q.z, v.w[4 * i + 3] = q.w;
            } else {
                const uint2 q = load_once8(p);
                v.w[0] = q.x, v.w[1] = q.y;
            }
        }
        return v;
    }
#pragma unroll
    for (int i = 0; i < V::kWords; ++i) v.w[i] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= n) break;
        if constexpr (E == 4) v.w[i] = static_cast<const uint32_t *>(p)[i];
        if constexpr (E == 2) v.w[i >> 1] |= (uint32_t) static_cast<const uint16_t *>(p)[i] << 16 * (i & 1);
        if constexpr (E == 1) v.w[i >> 2] |= (uint32_t) static_cast<const uint8_t *>(p)[i] << 8 * (i & 3);
    }
    return v;
}
template <typename V, int E>
__device__ __forceinline__ void store8(void *p, int n, bool wide, const V &v) {
    constexpr int kBytes = 4 * V::kWords, kWide = kBytes < 16 ? kBytes : 16;
    if (wide) {
#pragma unroll
        for (int i = 0; i < kBytes / kWide; ++i) {
            if constexpr (kWide == 16)
                __stcs(static_cast<uint4 *>(p) + i, make_uint4(v.w[4 * i], v.w[4 * i + 1], v.w[4 * i + 2], v.w[4 * i + 3]));
            else
                __stcs(static_cast<uint2 *>(p), make_uint2(v.w[0], v.w[1]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= n) break;
        if constexpr (E == 4) static_cast<uint32_t *>(p)[i] = v.w[i];
        if constexpr (E == 2) static_cast<uint16_t *>(p)[i] = (uint16_t)(v.w[i >> 1] >> 16 * (i & 1));
        if constexpr (E == 1) static_cast<uint8_t *>(p)[i] = (uint8_t)(v.w[i >> 2] >> 8 * (i & 3));
    }
}

// The bits of the largest magnitude among the warp's values.
__device__ __forceinline__ unsigned block_top(const float (&v)[8]) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]));
    return __reduce_max_sync(~0u, __float_as_uint(top));
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

// 32 bits that look random, of 32 (multipliers: fractional digits of the roots of 2 and 3).
__host__ __device__ __forceinline__ uint32_t scramble(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}
// Rounding to codes is done on fp32 numbers 2^-120 times those that the codes stand for: the bits
// from 20 on are then the code, below its normal range too, and neighbours are 2^20 apart.
constexpr float kDown = 0x1p-120f, kUp = 0x1p120f;
constexpr int kCode = 1 << 20, kNear = 3 * kCode / 4;
// Bits of the code that x goes to: by the draw (0 .. 2^20 - 1), or the nearest.  (NaN stays NaN.)
__device__ __forceinline__ int to_code(int x, bool by_draw, uint32_t draw) {
    return (min(x, 0x7ff00000) + (by_draw ? (int)draw : kCode / 2)) & -kCode;
}
// Whether two numbers of one sign are less than 3/4 of a code apart.
__device__ __forceinline__ bool near_code(int a, int b) { return (unsigned)(a - b + kNear) < 2u * kNear; }

// What a thread reads of 8 values.
template <typename P, typename G, bool kMaster, bool k8Bit>
struct Reads {
    using W = typename std::conditional<kMaster, Eight<float>, Eight<P>>::type;
    using M = typename std::conditional<k8Bit, Codes, Eight<float>>::type;
    Eight<G> g;
    W w;
    M m, v;
    float ms, vs;
};

// The 8-bit step has more arithmetic to hide its loads behind, so its registers are held down
// for more warps.  To nearest: 246 -> 211 us (bf16 weights), 291 -> 276 us (fp32) and 297 -> 281 us
// (masters) at 120 M values.  By draw: 420 us with three blocks per SM, 369 with four, 336 with five,
// 342 with six (bf16 weights; fp32 361 with five, 401 with six; masters 373 with four, 375 with
// five).  The 32-bit step loses by it.
enum : int { k32Bit = 0, kNearest = 1, kDrawn = 2 };        // moments, and how 8-bit codes are rounded
constexpr int blocks_per_sm(int moments, bool master) {
    return moments == k32Bit ? 1 : moments == kNearest ? (master ? 5 : 6) : (master ? 4 : 5);
}
template <typename P, typename G, bool kMaster, int kMoments>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(kMoments, kMaster)) k_adamw(const __grid_constant__ StepArgs a) {
    constexpr bool k8Bit = kMoments != k32Bit;
    wait_for_previous();
    // The tensor whose chunks this block's index falls into: found by one warp for all.
    __shared__ int tensor;
    if (threadIdx.x < 32) {
        int lo = 0, hi = a.count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.first[mid] <= blockIdx.x) lo = mid; else hi = mid - 1;
        }
        if (threadIdx.x == 0) tensor = lo;
    }
    __syncthreads();
    const int lo = __shfl_sync(~0u, tensor, 0);
    const Entry &e = a.t[lo];
    const int64_t at = (int64_t)(blockIdx.x - a.first[lo]) * kChunk + threadIdx.x * 8;
    float scale = 1.f;
    if (a.grad_scale) {
        scale = *a.grad_scale;
        if (!isfinite(scale)) return;           // an overflowed step: nothing changes
    }
    constexpr int kMoment = k8Bit ? 1 : 4;
    using R = Reads<P, G, kMaster, k8Bit>;
    auto bytes = [](void *p, int64_t at, int size) { return static_cast<char *>(p) + at * size; };
    const int n = (int)min((int64_t)8, max((int64_t)0, e.n - at));
    const bool wide = e.wide && n == 8;
    R cur;
    cur.g = load8<Eight<G>, sizeof(G)>(bytes(e.g, at, sizeof(G)), n, wide);
    if constexpr (kMaster) cur.w = load8<typename R::W, 4>(e.master + at, n, wide);
    else cur.w = load8<typename R::W, sizeof(P)>(bytes(e.p, at, sizeof(P)), n, wide);
    cur.m = load8<typename R::M, kMoment>(bytes(e.m, at, kMoment), n, wide);
    cur.v = load8<typename R::M, kMoment>(bytes(e.v, at, kMoment), n, wide);
    if constexpr (k8Bit) {
        cur.ms = n > 0 ? e.m_scale[at / kBlock] : 0.f;
        cur.vs = n > 0 ? e.v_scale[at / kBlock] : 0.f;
    }
    float m[8], v[8], w[8], root[8];
    if constexpr (k8Bit) {
        const f32x2 ms = twice(cur.ms), vs = twice(cur.vs);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const f32x2 r = mul2(cur.v.two(i), vs);
            unpair(mul2(cur.m.two(i), ms), m + i);
            unpair(mul2(r, r), v + i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = cur.m[i], v[i] = cur.v[i];
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
#pragma unroll
        for (int j = i; j < i + 2; ++j) {
            const float gs = a.grad_scale ? cur.g[j] * scale : cur.g[j];
            m[j] = __fadd_rn(__fmul_rn(a.beta1, m[j]), __fmul_rn(a.one_minus_beta1, gs));
            v[j] = __fadd_rn(__fmul_rn(a.beta2, v[j]), __fmul_rn(a.one_minus_beta2, __fmul_rn(gs, gs)));
        }
        float r[2];
        asm("sqrt.approx.f32 %0, %1;" : "=f"(root[i]) : "f"(v[i]));
        asm("sqrt.approx.f32 %0, %1;" : "=f"(root[i + 1]) : "f"(v[i + 1]));
        unpair(fma2(pair(root + i), twice(a.inv_sqrt_bc2), twice(a.eps)), r);
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r[0]));
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r[1]));
        const f32x2 old = pack(make_float2(cur.w[i], cur.w[i + 1]));
        unpair(fma2(twice(-a.step_size), mul2(pair(m + i), pair(r)), mul2(old, twice(a.decay))), w + i);
    }
    Eight<P> p;
    p.set(w);
    store8<Eight<P>, sizeof(P)>(bytes(e.p, at, sizeof(P)), n, wide, p);
    if constexpr (kMaster) {
        Eight<float> q;
        q.set(w);
        store8<Eight<float>, 4>(e.master + at, n, wide, q);
    }
    typename R::M mo, vo;
    if constexpr (k8Bit) {
        const int em = exponent(block_top(m)), ev = exponent(__float_as_uint(__fsqrt_rn(__uint_as_float(block_top(v)))));
        const float im = power_of_two(8 - em), iv = power_of_two(8 - ev);
        if constexpr (kMoments == kDrawn) {
            const f32x2 old_m = twice(cur.ms * im * kDown), old_v = twice(cur.vs * iv * kDown);
            const int64_t eighth = at >> 3;
            const uint32_t seed = scramble((uint32_t)eighth * 0x9E3779B9u + (uint32_t)(eighth >> 32) * 0x6A09E667u + (a.before + lo) * 0xBB67AE85u + a.draw);
            // Odd multipliers (fractional digits of square roots): each turns the uniform seed into another.
            constexpr uint32_t kDraws[8] = {0x9E3779B9u, 0x3C6EF373u, 0xA54FF53Bu, 0x510E527Fu, 0x9B05688Du, 0x1F83D9ABu, 0x5BE0CD19u, 0xCBBB9D5Du};
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                float x[2], o[2], y[2], p[2];
                unpair(mul2(mul2(pair(m + i), twice(im)), twice(kDown)), x);
                unpair(mul2(cur.m.two(i), old_m), o);
                unpair(mul2(mul2(pair(root + i), twice(iv)), twice(kDown)), y);
                unpair(mul2(cur.v.two(i), old_v), p);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t z = seed * kDraws[i + j];
                    const int xi = __float_as_int(x[j]), yi = __float_as_int(y[j]);
                    const bool from_zero = fabsf(o[j]) < __int_as_float(kCode);
                    const bool draw_m = near_code(xi, from_zero ? xi & 0x80000000 : __float_as_int(o[j])) && (!from_zero || fabsf(x[j]) >= a.leave_zero);
                    m[i + j] = __int_as_float(to_code(xi, draw_m, z >> 12));
                    int c = to_code(yi, near_code(yi, __float_as_int(p[j])), z & (kCode - 1));
                    if (root[i + j] > 0.f) c = max(c, kCode);
                    root[i + j] = __int_as_float(c);
                }
                unpair(mul2(pair(m + i), twice(kUp)), m + i);
                unpair(mul2(pair(root + i), twice(kUp)), root + i);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                float c[2];
                unpair(mul2(pair(m + i), twice(im)), m + i);
                unpair(mul2(pair(root + i), twice(iv)), c);
                root[i] = root[i] > 0.f ? fmaxf(c[0], 0x1p-9f) : c[0];
                root[i + 1] = root[i + 1] > 0.f ? fmaxf(c[1], 0x1p-9f) : c[1];
            }
        }
        mo.set(m);
        vo.set(root);
        if ((threadIdx.x & 31) == 0 && n > 0) {
            e.m_scale[at / kBlock] = power_of_two(em - 8);
            e.v_scale[at / kBlock] = power_of_two(ev - 8);
        }
    } else {
        mo.set(m);
        vo.set(v);
    }
    store8<typename R::M, kMoment>(bytes(e.m, at, kMoment), n, wide, mo);
    store8<typename R::M, kMoment>(bytes(e.v, at, kMoment), n, wide, vo);
}

using StepKernel = void (*)(const StepArgs);
template <typename P, typename G, bool kMaster>
StepKernel step_kernel(int moments) {
    return moments == kDrawn     ? k_adamw<P, G, kMaster, kDrawn>
           : moments == kNearest ? k_adamw<P, G, kMaster, kNearest>
                                 : k_adamw<P, G, kMaster, k32Bit>;
}
template <typename P, typename G>
StepKernel step_kernel(bool master, int moments) {
    if constexpr (sizeof(P) == 2) {
        if (master) return step_kernel<P, G, true>(moments);
    }
    return step_kernel<P, G, false>(moments);
}

}  // namespace

cudaError_t adamw_step(const rlm_adamw_tensor *tensors, int count, rlm_dtype param, rlm_dtype grad, bool master, int bits,
                       bool draw, const rlm_adamw_hyper &h, const float *grad_scale, cudaStream_t st) {
    const int moments = bits == 32 ? k32Bit : draw ? kDrawn : kNearest;
    const StepKernel fn = param == RLM_BF16
                              ? (grad == RLM_BF16 ? step_kernel<__nv_bfloat16, __nv_bfloat16>(master, moments)
                                                  : step_kernel<__nv_bfloat16, float>(master, moments))
                              : (grad == RLM_BF16 ? step_kernel<float, __nv_bfloat16>(master, moments)
                                                  : step_kernel<float, float>(master, moments));
    StepArgs a;
    const double bc1 = 1.0 - std::pow(h.beta1, (double)h.step), bc2 = 1.0 - std::pow(h.beta2, (double)h.step);
    a.grad_scale = grad_scale;
    a.beta1 = (float)h.beta1;
    a.one_minus_beta1 = (float)(1.0 - h.beta1);
    a.beta2 = (float)h.beta2;
    a.one_minus_beta2 = (float)(1.0 - h.beta2);
    a.inv_sqrt_bc2 = (float)(1.0 / std::sqrt(bc2));
    // The step's reciprocal takes denormal numbers for zero; beside a root, which is 0 or above 2^-75,
    // so small an eps is nothing anyway.
    a.eps = h.eps > 0 ? std::max((float)h.eps, FLT_MIN) : 0.f;
    a.decay = (float)(1.0 - h.lr * h.weight_decay);
    a.step_size = (float)(h.lr / bc1);
    a.draw = scramble((uint32_t)h.step + scramble((uint32_t)((uint64_t)h.step >> 32)));
    a.leave_zero = a.one_minus_beta1 * 0x1p-6f * kDown;
    for (int i = 0; i < count;) {
        a.count = 0;
        a.before = (uint32_t)i;
        unsigned chunks = 0;
        for (; i < count && a.count < kMaxTensors; ++i) {
            const rlm_adamw_tensor &t = tensors[i];
            const int64_t c = (t.n + kChunk - 1) / kChunk;
            if (a.count > 0 && c > (int64_t)0x7fffffff - chunks) break;     // the grid's limit
            a.first[a.count] = chunks;
            const uintptr_t all = reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.grad) |
                                  reinterpret_cast<uintptr_t>(t.master);
            const uintptr_t moments = reinterpret_cast<uintptr_t>(t.exp_avg) | reinterpret_cast<uintptr_t>(t.exp_avg_sq);
            const bool wide = (all & 15) == 0 && (moments & (bits == 8 ? 7 : 15)) == 0;
            a.t[a.count] = {t.param, const_cast<void *>(t.grad), t.exp_avg, t.exp_avg_sq, t.master, t.exp_avg_scale,
                            t.exp_avg_sq_scale, t.n, wide};
            ++a.count;
            chunks += (unsigned)c;
        }
        a.first[a.count] = chunks;
        const cudaError_t e = launch_dependent(fn, dim3(chunks), kThreads, 0, st, 1, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace rlm
