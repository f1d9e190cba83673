// rlm_ssm.cuh -- what the kernels of the selective state space scan share (rlm_ssm.cu, rlm_ssm_backward.cu).
//
//   D_t = softplus(dt_t + bias) (or without softplus),  a_tn = e^(D_t A_n),  h_tn = a_tn h_{t-1,n} + D_t x_t B_tn
//   o_t = sum_n C_tn h_tn + skip x_t,  y_t = o_t silu(z_t) (or o_t)
//
// per channel, with N states a channel and B, C shared by the channels.
//
// Layout of the forward kernels and of both kernels that form segments' ends.  A thread owns 4
// neighbouring channels and 4 of their states, P = N / 4 neighbouring lanes share the channels: a token's D
// and D x of 4 channels and B and C of 4 states, 64 bytes out of shared memory, serve 16 states.  (Shared
// memory gives a warp 128 bytes a clock: with one channel a thread, 48 bytes for 4 states, it bounded the
// kernel, 138 us against 36 of arithmetic at B = 4, L = 4096, D = 1024, N = 16.)  A block is 64 threads, 64 / P
// groups of channels, and walks tiles of 4 P tokens, 16 at most: 4 groups of 4 channels a thread and field, 2 at N = 32.  They
// are loaded one tile ahead, D and D x formed in fp32 and left in shared memory.
#pragma once

#include "rlm_device.cuh"
#include "rlm_internal.h"

namespace rlm {
namespace ssm {

constexpr int kTile = RLM_SSM_CHUNK;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// ex2.approx is off by 3e-8 of itself (rms) and on the average too small: by 5.5e-9 of itself (within 1.5e-9) at exponents x
// above -2^-8.5, by 1e-8 at -2^-8.2, 2.2e-8 (0.8 to 3e-8) from -2^-7.5 on (means over factors of 1.4).  A state that
// remembers n steps would collect n times the mean.  The middle of it is added to the exponents (kShift; at an exponent of 0
// a is 1 all the same).  What is left is taken off by what the tokens did: the product P of the decays that a state went
// through is kept beside it, and after kPeriod tokens it is multiplied by e^(A sum of D) / P (put_right).  So is the
// gradient G.  (dA at B = 4, L = 4096, steps of 0.001 to 0.1, A = -1 .. -16, is off by 6.0e-7 in norm; by 3.9e-6 with
// the exponentials as they are, 6.8e-7 with each decay rounded correctly.  With one token's step taken for kPeriod of them it
// was 8.5e-7, and 5e-5 in a state that only that token moves.)
constexpr float kShift = 2e-8f;
constexpr int kPeriod = 32;             // (of the gradients' main kernel: kTile)

__device__ __forceinline__ float ex2(float v) {
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
    return e;
}
__device__ __forceinline__ float sigma(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2(-kLog2e * v)));
    return r;
}
// Four neighbouring values as loaded and as stored.
template <typename T>
struct Four;
template <>
struct Four<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint2 *>(p); }
    __device__ __forceinline__ void clear() { v = make_uint2(0, 0); }
    __device__ __forceinline__ float4 values() const {
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                           __uint_as_float(v.y & 0xffff0000u));
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, float4 f) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(f.x, f.y), b = __floats2bfloat162_rn(f.z, f.w);
        *reinterpret_cast<uint2 *>(p) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
};
template <>
struct Four<float> {
    float4 v;
    __device__ __forceinline__ void load(const float *p) { v = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void clear() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ float4 values() const { return v; }
    static __device__ __forceinline__ void store(float *p, float4 f) { *reinterpret_cast<float4 *>(p) = f; }
};

// Four states (or what belongs to them) as two packed pairs.
struct alignas(16) Quad {
    f32x2 lo, hi;
};
__device__ __forceinline__ f32x2 both(float v) { return pack(make_float2(v, v)); }
__device__ __forceinline__ Quad quad(float4 v) { return {pack(make_float2(v.x, v.y)), pack(make_float2(v.z, v.w))}; }
__device__ __forceinline__ float4 unquad(Quad q) {
    const float2 a = unpack(q.lo), b = unpack(q.hi);
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ Quad mul4(f32x2 a, Quad b) { return {mul2(a, b.lo), mul2(a, b.hi)}; }
__device__ __forceinline__ Quad mul4(Quad a, Quad b) { return {mul2(a.lo, b.lo), mul2(a.hi, b.hi)}; }
__device__ __forceinline__ Quad fma4(f32x2 a, Quad b, Quad c) { return {fma2(a, b.lo, c.lo), fma2(a, b.hi, c.hi)}; }
__device__ __forceinline__ Quad fma4(Quad a, Quad b, Quad c) { return {fma2(a.lo, b.lo, c.lo), fma2(a.hi, b.hi, c.hi)}; }
__device__ __forceinline__ float dot4(Quad a, Quad b) {
    const float2 s = unpack(fma2(a.hi, b.hi, mul2(a.lo, b.lo)));
    return s.x + s.y;
}
// e^(D A) from D and A log2 e.
__device__ __forceinline__ f32x2 decay(f32x2 delta, f32x2 a2) {
    const float2 v = unpack(fma2(delta, a2, both(kShift)));
    return pack(make_float2(ex2(v.x), ex2(v.y)));
}
// 2^x for |x| <= 1, by its Taylor series up to the 9th power (the 10th is below 7.1e-9): its rounding has no mean.
__device__ __forceinline__ f32x2 exp2_series(f32x2 x) {
    f32x2 f = fma2(x, both(1.0178086e-7f), both(1.3215487e-6f));        // (ln 2)^k / k!, k = 9, 8 ..
    f = fma2(x, f, both(1.5252734e-5f));
    f = fma2(x, f, both(1.5403530e-4f));
    f = fma2(x, f, both(1.3333558e-3f));
    f = fma2(x, f, both(9.6181291e-3f));
    f = fma2(x, f, both(5.5504109e-2f));
    f = fma2(x, f, both(0.24022651f));
    f = fma2(x, f, both(kLn2));
    return fma2(x, f, both(1.f));
}
// decay() for a token by itself: by the series where the state will remember it.
__device__ __forceinline__ f32x2 decay_alone(f32x2 delta, f32x2 a2) {
    const f32x2 x = mul2(delta, a2);
    const float2 v = unpack(x), near = unpack(exp2_series(x)), far = unpack(decay(delta, a2));
    return pack(make_float2(fabsf(v.x) <= 1.f ? near.x : far.x, fabsf(v.y) <= 1.f ? near.y : far.y));
}
// max(v, 0) + log(1 + e), e = e^-|v|, the logarithm as 2 artanh(e / (2 + e)) by its series up to the 13th power
// (1 / 3 to the 14th over 15 is 1.4e-8): to about (|v| + 9) 2^-24 of itself at every v, where log1pf takes four
// times the instructions, a third of the forward kernel's.
__device__ __forceinline__ f32x2 softplus(f32x2 v) {
    const float2 x = unpack(v);
    const f32x2 e = pack(make_float2(ex2(-kLog2e * fabsf(x.x)), ex2(-kLog2e * fabsf(x.y))));
    float2 r = unpack(add2(e, both(2.f)));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r.x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r.y));
    const f32x2 s = mul2(e, pack(r)), q = mul2(s, s);
    f32x2 f = fma2(q, both(1.f / 13), both(1.f / 11));
    f = fma2(q, f, both(1.f / 9));
    f = fma2(q, f, both(1.f / 7));
    f = fma2(q, f, both(1.f / 5));
    f = fma2(q, f, both(1.f / 3));
    f = fma2(q, f, both(1.f));
    return fma2(add2(s, s), f, pack(make_float2(fmaxf(x.x, 0.f), fmaxf(x.y, 0.f))));
}
// D of 4 channels, 0 where there is no token.
__device__ __forceinline__ Quad step_of(float4 dt, Quad bias, int softplus_, bool live) {
    const Quad v = quad(dt);
    Quad d = {add2(v.lo, bias.lo), add2(v.hi, bias.hi)};
    if (softplus_) d = {softplus(d.lo), softplus(d.hi)};
    return live ? d : Quad{0, 0};
}

template <typename T>
struct Args {
    const T *x, *dt, *b, *c, *z;        // z nullable
    T *y;
    int64_t x_b, x_l, dt_b, dt_l, b_b, b_l, c_b, c_l, z_b, z_l, y_b, y_l;       // strides in elements
    const float *A, *skip, *bias;       // [D][N], nullable [D], nullable [D]
    const float *state_in;              // nullable, [B][D][N]
    float *state_out, *saved;           // nullable; saved [B][ntiles][D][N]
    const int *lengths;                 // nullable
    float *end_state, *end_delta;       // of the segments but the last, from a zero state: [B][nseg][D][N], [B][nseg][D]
    int L, D, ntiles, nseg, per, softplus;      // per: tiles of a segment
    // backward
    const T *dy;
    T *dx, *ddt, *db, *dc, *dz;         // dz nullable
    int64_t dy_b, dy_l, dx_b, dx_l, ddt_b, ddt_l, db_b, db_l, dc_b, dc_l, dz_b, dz_l;
    const float *d_state_out;           // nullable
    float *d_state_in;                  // nullable
    float *part_bc;                     // [B][L][groups][2 N]: dB and dC of a block's channels
    float *part_A, *part_d;             // [B * nseg][D][N], [B * nseg][2][D]: dA; dskip and dbias
};

template <typename T>
__device__ __forceinline__ int length_of(const Args<T> &a, int b) {
    return a.lengths ? max(0, min(a.lengths[b], a.L)) : a.L;
}

constexpr int kThreads = 64;
template <int N>
struct Block {
    static constexpr int P = N / 4, kGroups = kThreads / P, kWidth = 4 * kGroups, kTok = 4 * P < kTile ? 4 * P : kTile;
    static constexpr int kUnits = kTok * kGroups / kThreads;                    // groups of 4 channels a thread and field
    static constexpr int kRows = (kTok * P + kThreads - 1) / kThreads;          // groups of 4 of B's values a thread
    static constexpr int64_t blocks_of(int64_t B, int D, int nseg) { return B * ((D + kWidth - 1) / kWidth) * nseg; }
};

// A thread's place: batch row, segment and its tiles; the channels that it scans (c, states 4 p on) and those that
// it loads (cu, the same for all its units; tokens token(k) of a tile).
template <typename T, int N>
struct Place {
    using S = Block<N>;
    int b, seg, first, last, c, p, cu, len;
    bool on, on_u;
    __device__ __forceinline__ explicit Place(const Args<T> &a) {
        const int groups = (a.D + S::kWidth - 1) / S::kWidth, r = blockIdx.x / a.nseg;
        seg = blockIdx.x - r * a.nseg;
        b = r / groups;
        const int c0 = (r - b * groups) * S::kWidth;
        first = min(seg * a.per, a.ntiles) * (kTile / S::kTok);
        last = min((seg + 1) * a.per, a.ntiles) * (kTile / S::kTok);
        p = threadIdx.x % S::P;
        c = c0 + threadIdx.x / S::P * 4;
        cu = c0 + threadIdx.x % S::kGroups * 4;
        on = c < a.D;
        on_u = cu < a.D;
        len = length_of(a, b);
    }
    static __device__ __forceinline__ int token(int k) { return (threadIdx.x + k * kThreads) / S::kGroups; }
    static __device__ __forceinline__ int unit(int k) { return threadIdx.x + k * kThreads; }        // token, group
    // Tokens from len on and channels from D on are 0.
    __device__ __forceinline__ void load(Four<T> (&r)[S::kUnits], const T *q, int64_t stride, int t0) const {
#pragma unroll
        for (int k = 0; k < S::kUnits; ++k) {
            const int at = t0 + token(k);
            if (on_u && at < len) {
                r[k].load(q + (int64_t)at * stride + cu);
            } else {
                r[k].clear();
            }
        }
    }
    __device__ __forceinline__ void load_row(Four<T> (&r)[S::kRows], const T *q, int64_t stride, int t0) const {
#pragma unroll
        for (int k = 0; k < S::kRows; ++k) {
            const int i = threadIdx.x + k * kThreads, at = t0 + i / S::P;
            if (at < len && i < S::kTok * S::P) {
                r[k].load(q + (int64_t)at * stride + i % S::P * 4);
            } else {
                r[k].clear();
            }
        }
    }
    static __device__ __forceinline__ void store_row(float4 *to, const Four<T> (&r)[S::kRows]) {
#pragma unroll
        for (int k = 0; k < S::kRows; ++k)
            if (const int i = threadIdx.x + k * kThreads; i < S::kTok * S::P) to[i] = r[k].values();
    }
    // The thread's states of [..][D][N]: row `row`'s.
    __device__ __forceinline__ int64_t state(const Args<T> &a, int64_t row) const { return (row * a.D + c) * N + 4 * p; }
    __device__ __forceinline__ void load_states(Quad (&h)[4], const float *q) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = on && q ? quad(*reinterpret_cast<const float4 *>(q + i * N)) : Quad{0, 0};
    }
    __device__ __forceinline__ void store_states(const Quad (&h)[4], float *q) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (on) *reinterpret_cast<float4 *>(q + i * N) = unquad(h[i]);
    }
    __device__ __forceinline__ void load_decays(Quad (&a2)[4], const Args<T> &a) const {
        load_states(a2, a.A + (int64_t)c * N + 4 * p);
#pragma unroll
        for (int i = 0; i < 4; ++i) a2[i] = mul4(both(kLog2e), a2[i]);
    }
};
// h <- e^(D A) h + v, D of 4 channels.
__device__ __forceinline__ void advance(Quad (&h)[4], const Quad (&a2)[4], float4 delta, const Quad (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 d = both(i == 0 ? delta.x : i == 1 ? delta.y : i == 2 ? delta.z : delta.w);
        h[i] = {fma2(decay(d, a2[i].lo), h[i].lo, v[i].lo), fma2(decay(d, a2[i].hi), h[i].hi, v[i].hi)};
    }
}

// The states before a segment from those before the first one, which start(h) gives: step after step h <- e^(A S) h + v over
// the segments before it, S a segment's sum of D and v what it leaves of a zero state; load(s, delta, v) gives the s-th's.
// Where decays grow past fp32's range a factor is infinite, and what it makes is infinite or NaN whatever the later steps do.
// Then the steps are taken again with the factor in three: what is 0 stays 0, and what the whole factor would bring back
// into range does so.
__device__ __forceinline__ f32x2 grown(f32x2 delta, f32x2 a2, f32x2 h, f32x2 v) {
    const float2 x = unpack(mul2(fma2(delta, a2, both(kShift)), both(1 / 3.f)));
    const f32x2 third = pack(make_float2(ex2(fminf(x.x, 126.f)), ex2(fminf(x.y, 126.f))));
    return fma2(third, mul2(third, mul2(third, h)), v);
}
template <typename Start, typename Load>
__device__ __forceinline__ void through_segments(Quad (&h)[4], const Quad (&a2)[4], int count, Start start, Load load) {
    start(h);
    float4 delta;
    Quad v[4];
#pragma unroll 2
    for (int s = 0; s < count; ++s) {
        load(s, delta, v);
        advance(h, a2, delta, v);
    }
    bool fine = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 f = unquad(h[i]);
        fine &= fabsf(f.x) < __builtin_huge_valf() && fabsf(f.y) < __builtin_huge_valf() && fabsf(f.z) < __builtin_huge_valf() &&
                fabsf(f.w) < __builtin_huge_valf();
    }
    if (fine) return;
    start(h);
#pragma unroll 1
    for (int s = 0; s < count; ++s) {
        load(s, delta, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 d = both(i == 0 ? delta.x : i == 1 ? delta.y : i == 2 ? delta.z : delta.w);
            h[i] = {grown(d, a2[i].lo, h[i].lo, v[i].lo), grown(d, a2[i].hi, h[i].hi, v[i].hi)};
        }
    }
}

// The product P of the decays that 4 channels' states went through, and the sum of -D.
struct Passed {
    Quad product[4], minus;
    __device__ __forceinline__ void clear() {
        minus = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) product[i] = {both(1.f), both(1.f)};
    }
    __device__ __forceinline__ void add(Quad delta) { minus = {fma2(delta.lo, both(-1.f), minus.lo), fma2(delta.hi, both(-1.f), minus.hi)}; }
};
__device__ __forceinline__ void advance(Quad (&h)[4], const Quad (&a2)[4], float4 delta, const Quad (&v)[4], Passed &passed) {
    passed.add(quad(delta));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 d = both(i == 0 ? delta.x : i == 1 ? delta.y : i == 2 ? delta.z : delta.w);
        const Quad a = {decay(d, a2[i].lo), decay(d, a2[i].hi)};
        h[i] = fma4(a, h[i], v[i]);
        passed.product[i] = mul4(a, passed.product[i]);
    }
}

// h 2^-x / P as h + h (1 - P 2^x), x the sum of -D A log2 e and |x| <= 1: what forgets faster (within 46 tokens) collects too
// little to matter, and there what h has gained since would lose more by x's rounding.  (The factor itself has too few
// bits.)  An infinite h stays: its second term is infinite or NaN.
__device__ __forceinline__ f32x2 put_right(f32x2 h, f32x2 product, f32x2 x) {
    const f32x2 over = fma2(product, exp2_series(x), both(-1.f));
    const float2 t = unpack(mul2(over, h)), e = unpack(x), v = unpack(h);
    constexpr float kInf = __builtin_huge_valf();
    return pack(make_float2(v.x - (fabsf(e.x) <= 1.f && fabsf(t.x) < kInf ? t.x : 0.f), v.y - (fabsf(e.y) <= 1.f && fabsf(t.y) < kInf ? t.y : 0.f)));
}
__device__ __forceinline__ void put_right(Quad (&h)[4], const Quad (&a2)[4], const Passed &passed) {
    const float4 d = unquad(passed.minus);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Quad x = mul4(both(i == 0 ? d.x : i == 1 ? d.y : i == 2 ? d.z : d.w), a2[i]);
        h[i] = {put_right(h[i].lo, passed.product[i].lo, x.lo), put_right(h[i].hi, passed.product[i].hi, x.hi)};
    }
}

__device__ __forceinline__ float4 four_of(const float *p, int c, bool on) {
    return p && on ? *reinterpret_cast<const float4 *>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
}
__device__ __forceinline__ float at(const float4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Segments for a kernel of `blocks` blocks without them, `resident` of which an SM holds: the count with the least of
// rounds of blocks times the tiles of a segment (and about one more for its set-up), and, where there are several,
// times what the kernel that forms their ends adds.
int segments(int64_t blocks, int ntiles, int resident, double ends);

}  // namespace ssm
}  // namespace rlm
