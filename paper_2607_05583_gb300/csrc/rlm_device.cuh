// rlm_device.cuh -- small device helpers shared by the CUDA translation units.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace rlm {

template <typename T>
__device__ __forceinline__ float ld_elem(const T *p);
template <>
__device__ __forceinline__ float ld_elem<float>(const float *p) { return __ldg(p); }
template <>
__device__ __forceinline__ float ld_elem<__nv_bfloat16>(const __nv_bfloat16 *p) {
    return __bfloat162float(__ldg(p));
}

template <typename T>
__device__ __forceinline__ void st_elem(T *p, float v);
template <>
__device__ __forceinline__ void st_elem<float>(float *p, float v) { *p = v; }
template <>
__device__ __forceinline__ void st_elem<__nv_bfloat16>(__nv_bfloat16 *p, float v) {
    *p = __float2bfloat16_rn(v);
}

// Complex helpers on float2 (x = Re, y = Im).
__device__ __forceinline__ float2 cmul(float2 a, float2 b) {
    return make_float2(fmaf(a.x, b.x, -a.y * b.y), fmaf(a.x, b.y, a.y * b.x));
}
__device__ __forceinline__ float2 conj2(float2 a) { return make_float2(a.x, -a.y); }
// a*b + c
__device__ __forceinline__ float2 cfma(float2 a, float2 b, float2 c) {
    return make_float2(fmaf(a.x, b.x, fmaf(-a.y, b.y, c.x)), fmaf(a.x, b.y, fmaf(a.y, b.x, c.y)));
}

// lambda^n = exp(-gamma n) (cos(omega n) + i sin(omega n)) in fp32.  The
// products gamma*n and omega*n are formed with their exact FMA residuals, so
// the phase keeps full accuracy for large n (a plain fp32 omega*n is off by up
// to |omega n| * 2^-24 rad).  n must be an integer below 2^24.
__device__ __forceinline__ float2 lambda_pow(float gamma, float omega, float n) {
    float p = omega * n;
    float pe = fmaf(omega, n, -p);
    float sp, cp;
    sincosf(p, &sp, &cp);
    float q = gamma * n;
    float qe = fmaf(gamma, n, -q);
    float r = expf(-q) * (1.0f - qe);
    return make_float2(r * fmaf(-pe, sp, cp), r * fmaf(pe, cp, sp));
}

// Programmatic dependent launch: returns once the kernels before this one in the stream have
// finished, and lets the next one start its own set-up (it waits here in turn).  For kernels
// launched with launch_dependent().
// What that kernel may have written is read by coherent loads that stay behind the wait: plain
// ones or the volatile one below.  The read-only path (ld.global.nc, __ldg) may be used for
// nothing that changes while a kernel is resident, and a dependent kernel is resident early;
// neither __ldg nor __ldcs is bound to stay behind the wait.
__device__ __forceinline__ void wait_for_previous() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// 16 bytes that are read once, and 8.
__device__ __forceinline__ uint4 load_once(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

__device__ __forceinline__ uint2 load_once8(const void *p) {
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}

// Two fp32 values in one 64-bit register, and the packed arithmetic on them (each half
// rounded as the scalar operation rounds it).
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pack(float2 v) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 unpack(f32x2 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// c = A exp(i phi).
__device__ __forceinline__ float2 mode_coef(float amp, float phase) {
    float s, c;
    sincosf(phase, &s, &c);
    return make_float2(amp * c, amp * s);
}

}  // namespace rlm
