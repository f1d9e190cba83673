// rlm_scan.cu -- the gated linear recurrence: sequence form, gradients, one step.
//
//   a_t = sigma(g_t),  h_t = a_t h_{t-1} + i_t,  i_t = (1 - a_t) x_t (leak) or x_t
//
// per channel, with b_t = 1 - a_t = 1 / (1 + e^{g_t}) formed directly: gates sit near
// a = 1 and 1 - a would lose b's leading bits.  The kernels keep b and use
//   leak  h += b (x - h)          unit  h = (h + x) - b h
//
// A run of tokens maps the state by h -> A h + H (A the product of its a, H its end
// state from zero), and runs compose: (A2, H2) o (A1, H1) = (A2 A1, A2 H1 + H2).
// The gradient is the same scan with time reversed: with C_t the gradient that
// reaches h_{t-1}, G_t = dy_t + C_{t+1} and C_t = a_t G_t; then
//   leak  dx = b G, dg = a b G (h_{t-1} - x)      unit  dx = G, dg = a b G h_{t-1}.
//
// Bound by memory: 3 fields move in the forward pass and 5 in the backward pass,
// about 20 instructions an element beside.  So each field is read once: a thread
// holds kS tokens of two channels in registers, the runs of a tile's threads compose
// through shuffles and shared memory, and the tiles' runs through a workspace.
//
// Tiles.  A CTA of 256 threads covers P channel pairs (P = 4, 8, 16 or 32, the least
// that holds D / 2) by 256 / P runs of kS tokens: 128-byte row slices at D >= 64, a
// whole row below.  It walks its channels' tiles in time order with the carry in
// registers, loading the next tile's fields while it works on this one.
//
// Segments.  Few channels (B ceil(D / 64) CTAs below the resident number) would
// leave SMs idle, so nseg CTAs share a chain of tiles: in wave w CTA s takes tile
// w nseg + s, publishes the tile's (A, H), reads those of the whole wave and composes
// the ones before its own on top of the carry (and all of them for the next wave's
// carry).  Nobody waits for a neighbour's output, so a wave costs one exchange
// through L2, whatever nseg is, and no field is read twice.  The launch is
// cooperative (all CTAs resident) and every wait is bounded.  The order of all
// products and sums is fixed by the shape: results repeat bit for bit.
#include <algorithm>
#include <mutex>
#include <vector>

#include "rlm_device.cuh"
#include "rlm_internal.h"

namespace rlm {

__device__ int g_scan_status = 0;

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = RLM_SCAN_CHUNK;              // tokens between saved states
constexpr long long kWaitLimit = 4000000000ll;      // SM cycles: about 2 s

// Two neighbouring channels of a field, as loaded and as values.
template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
    using Raw = uint32_t;
    static __device__ __forceinline__ Raw load(const __nv_bfloat16 *p) {
        Raw r;
        asm("ld.global.nc.L1::no_allocate.b32 %0, [%1];" : "=r"(r) : "l"(p));
        return r;
    }
    static __device__ __forceinline__ Raw zero() { return 0u; }
    static __device__ __forceinline__ float2 value(Raw r) {
        return make_float2(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u));
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, float2 v) {
        __nv_bfloat162 o = __floats2bfloat162_rn(v.x, v.y);
        __stcs(reinterpret_cast<unsigned *>(p), *reinterpret_cast<unsigned *>(&o));
    }
};
template <>
struct Pair<float> {
    using Raw = float2;
    static __device__ __forceinline__ Raw load(const float *p) {
        Raw r;
        asm("ld.global.nc.L1::no_allocate.v2.f32 {%0, %1}, [%2];" : "=f"(r.x), "=f"(r.y) : "l"(p));
        return r;
    }
    static __device__ __forceinline__ Raw zero() { return make_float2(0.f, 0.f); }
    static __device__ __forceinline__ float2 value(Raw r) { return r; }
    static __device__ __forceinline__ void store(float *p, float2 v) { __stcs(reinterpret_cast<float2 *>(p), v); }
};

// Tokens of one thread's run.  The forward pass holds b (8 bytes), x and the next
// tile's x and g for each token and channel pair, the backward pass also dy and
// h_{t-1}: the largest powers of two that stay under 128 registers.
template <typename T>
constexpr int kFwdRun = sizeof(T) == 2 ? 16 : 8;
constexpr int kBwdRun = 8;

// 1 - sigma(g); g = +inf gives 0, -inf gives 1.
__device__ __forceinline__ float rest(float g) { return __fdividef(1.0f, 1.0f + expf(g)); }

template <typename T>
struct ScanArgs {
    const T *x, *g, *dy;
    T *y, *dx, *dg;
    int64_t x_b, x_l, g_b, g_l, dy_b, dy_l, y_b, y_l, dx_b, dx_l, dg_b, dg_l;   // strides in elements
    const float *state_in;      // forward: h_{-1}; backward: dl/dh_{L-1}; nullable (zero)
    float *state_out;           // forward: h_{L-1}; backward: dl/dh_{-1}; nullable
    float *saved;               // [B][ceil(L / kChunk)][D]: h before each chunk (forward: nullable output)
    const int *lengths;         // nullable, [B]
    int L, D, groups, log2p, nseg, ntiles, nchunks;
    float4 *agg;                // [chain][2][nseg][32]: (A, A', H, H') of a tile, by wave parity
    unsigned *flag;             // [chain][nseg]: waves published
};

// (A, H) of two channels as (A.x, A.y, H.x, H.y); `later` o `earlier`.
__device__ __forceinline__ float4 compose(float4 earlier, float4 later) {
    return make_float4(later.x * earlier.x, later.y * earlier.y, fmaf(later.x, earlier.z, later.z),
                       fmaf(later.y, earlier.w, later.w));
}
__device__ __forceinline__ float4 shfl4(float4 v, int src) {
    return make_float4(__shfl_sync(~0u, v.x, src), __shfl_sync(~0u, v.y, src), __shfl_sync(~0u, v.z, src),
                       __shfl_sync(~0u, v.w, src));
}
__device__ __forceinline__ float4 identity4() { return make_float4(1.f, 1.f, 0.f, 0.f); }
__device__ __forceinline__ float2 apply(float4 f, float2 h) {
    return make_float2(fmaf(f.x, h.x, f.z), fmaf(f.y, h.y, f.w));
}

// Inclusive scan over the lanes of one channel pair (P apart); kRev: over those after.
template <bool kRev>
__device__ __forceinline__ float4 lane_scan(float4 v, int P, int lane) {
    for (int d = P; d < 32; d <<= 1) {
        const int src = kRev ? lane + d : lane - d;
        const float4 o = shfl4(v, src & 31);
        if (kRev ? src < 32 : src >= 0) v = compose(o, v);
    }
    return v;
}
// The same, without this lane's own run.
template <bool kRev>
__device__ __forceinline__ float4 lane_exclusive(float4 incl, int P, int lane) {
    const int src = kRev ? lane + P : lane - P;
    const float4 o = shfl4(incl, src & 31);
    return (kRev ? src < 32 : src >= 0) ? o : identity4();
}

// Waits until segment `flag` has published `want` waves; bounded.  The acquire
// orders this thread's later loads of the published values.
__device__ __forceinline__ void wait_published(const unsigned *flag, unsigned want, volatile int *abort_flag) {
    long long t0 = 0;
    for (uint32_t it = 1;; ++it) {
        unsigned v;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(flag) : "memory");
        if (v >= want) return;
        if ((it & 255u) == 0) {
            if (*abort_flag) return;
            const long long now = clock64();
            if (t0 == 0) {
                t0 = now;
            } else if (now - t0 > kWaitLimit) {
                *abort_flag = 1;
                atomicExch(&g_scan_status, (int)RLM_ERR_TIMEOUT);
                return;
            }
        }
    }
}

struct ScanShared {
    float4 run[2][kWarps][32];          // a warp's composed run, by tile parity
    float4 pre[2][kWarps][32];          // folds of a wave's tiles: those before this CTA's own,
    float4 all[2][kWarps][32];          //   and all of them
    int abort_flag;
};

// One wave's exchange: publishes this tile's run `mine` and returns the composition of
// the tiles before it (*pre) and of the `live` tiles of the wave (*all).
__device__ __forceinline__ void exchange(float4 mine, float4 *agg, unsigned *flag, int wave, int seg, int nseg, int live,
                                         int P, int cp, ScanShared &sh, float4 *pre, float4 *all) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, par = wave & 1;
    float4 *row = agg + (int64_t)par * nseg * 32;
    if (warp == 0) {
        if (lane < P) __stcg(row + seg * 32 + cp, mine);
        __syncwarp();
        if (lane == 0) {
            __threadfence();
            asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(flag + seg), "r"((unsigned)(wave + 1)) : "memory");
        }
    }
    // Each run of threads folds its share of the wave's tiles.
    const int parts = kThreads / P, part = tid / P;
    const int lo = live * part / parts, hi = live * (part + 1) / parts;
    for (int s = lo; s < hi; ++s) wait_published(flag + s, (unsigned)(wave + 1), &sh.abort_flag);
    float4 fa = identity4(), fp = identity4();
#pragma unroll 4
    for (int s = lo; s < hi; ++s) {
        const float4 v = __ldcg(row + s * 32 + cp);
        if (s == seg) fp = fa;
        fa = compose(fa, v);
    }
    if (seg >= hi) fp = fa;             // (a share that lies after `seg` keeps the identity)
    fa = lane_scan<false>(fa, P, lane);
    // Before-parts compose in the same order: full shares, then the one that holds `seg`.
    fp = lane_scan<false>(fp, P, lane);
    if (lane >= 32 - P) {
        sh.all[par][warp][cp] = fa;
        sh.pre[par][warp][cp] = fp;
    }
    __syncthreads();
    float4 ta = identity4(), tp = identity4();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        ta = compose(ta, sh.all[par][w][cp]);
        tp = compose(tp, sh.pre[par][w][cp]);
    }
    *pre = tp;
    *all = ta;
}

template <typename T, bool kLeak>
__global__ void __launch_bounds__(kThreads, 2) k_scan_forward(const ScanArgs<T> a) {
    constexpr int S = kFwdRun<T>;
    using Raw = typename Pair<T>::Raw;
    __shared__ ScanShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int P = 1 << a.log2p, cp = tid & (P - 1), sc = tid >> a.log2p;
    const int chains = gridDim.x / a.nseg, seg = blockIdx.x / chains, chain = blockIdx.x - seg * chains;
    const int row = chain / a.groups, c = (chain - row * a.groups) * 2 * P + 2 * cp;
    const bool on = c < a.D;
    const int T_ = (kThreads >> a.log2p) * S;
    const int len = a.lengths ? min(max(a.lengths[row], 0), a.L) : a.L;
    if (tid == 0) sh.abort_flag = 0;
    const T *xp = a.x + row * a.x_b + c, *gp = a.g + row * a.g_b + c;
    T *yp = a.y + row * a.y_b + c;
    float2 carry = make_float2(0.f, 0.f);
    if (a.state_in && on) carry = *reinterpret_cast<const float2 *>(a.state_in + (int64_t)row * a.D + c);

    Raw xr[S], gr[S];
    auto load = [&](int tile) {
        const int t0 = tile * T_ + sc * S;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const bool ok = on && t0 + i < len;
            xr[i] = ok ? Pair<T>::load(xp + (int64_t)(t0 + i) * a.x_l) : Pair<T>::zero();
            gr[i] = ok ? Pair<T>::load(gp + (int64_t)(t0 + i) * a.g_l) : Pair<T>::zero();
        }
    };
    load(seg);
    __syncthreads();
    int wave = 0;
    for (int tile = seg; tile < a.ntiles; tile += a.nseg, ++wave) {
        const int t0 = tile * T_ + sc * S;
        Raw xs[S];
        float2 b[S];
        float4 f = identity4();
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const float2 g = Pair<T>::value(gr[i]);
            const bool ok = t0 + i < len;
            b[i] = ok ? make_float2(rest(g.x), rest(g.y)) : make_float2(0.f, 0.f);   // past the end: the identity
            xs[i] = xr[i];
            const float2 x = Pair<T>::value(xs[i]);
            f.x = fmaf(-b[i].x, f.x, f.x);
            f.y = fmaf(-b[i].y, f.y, f.y);
            f.z = kLeak ? fmaf(b[i].x, x.x - f.z, f.z) : fmaf(-b[i].x, f.z, f.z + x.x);
            f.w = kLeak ? fmaf(b[i].y, x.y - f.w, f.w) : fmaf(-b[i].y, f.w, f.w + x.y);
        }
        if (tile + a.nseg < a.ntiles) load(tile + a.nseg);
        const float4 incl = lane_scan<false>(f, P, lane);
        const float4 excl = lane_exclusive<false>(incl, P, lane);
        if (lane >= 32 - P) sh.run[wave & 1][warp][cp] = incl;
        __syncthreads();
        float4 before = identity4(), total = identity4();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) before = total;
            total = compose(total, sh.run[wave & 1][w][cp]);
        }
        before = compose(before, excl);
        float2 h;
        if (a.nseg > 1) {
            float4 pre, all;
            exchange(total, a.agg + (int64_t)chain * 2 * a.nseg * 32, a.flag + (int64_t)chain * a.nseg, wave, seg,
                     a.nseg, min(a.nseg, a.ntiles - wave * a.nseg), P, cp, sh, &pre, &all);
            h = apply(before, apply(pre, carry));
            carry = apply(all, carry);
        } else {
            h = apply(before, carry);
            carry = apply(total, carry);
        }
        if (a.saved && on && t0 % kChunk == 0 && t0 < a.L)
            *reinterpret_cast<float2 *>(a.saved + ((int64_t)row * a.nchunks + t0 / kChunk) * a.D + c) = h;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const float2 x = Pair<T>::value(xs[i]);
            h.x = kLeak ? fmaf(b[i].x, x.x - h.x, h.x) : fmaf(-b[i].x, h.x, h.x + x.x);
            h.y = kLeak ? fmaf(b[i].y, x.y - h.y, h.y) : fmaf(-b[i].y, h.y, h.y + x.y);
            if (on && t0 + i < a.L)
                Pair<T>::store(yp + (int64_t)(t0 + i) * a.y_l, t0 + i < len ? h : make_float2(0.f, 0.f));
        }
        if (tile == a.ntiles - 1 && a.state_out && on && sc == (kThreads >> a.log2p) - 1)
            *reinterpret_cast<float2 *>(a.state_out + (int64_t)row * a.D + c) = h;
    }
}

template <typename T, bool kLeak>
__global__ void __launch_bounds__(kThreads, 2) k_scan_backward(const ScanArgs<T> a) {
    constexpr int S = kBwdRun;
    using Raw = typename Pair<T>::Raw;
    __shared__ ScanShared sh;
    __shared__ float4 rev[2][kWarps][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int P = 1 << a.log2p, cp = tid & (P - 1), sc = tid >> a.log2p;
    const int chains = gridDim.x / a.nseg, seg = blockIdx.x / chains, chain = blockIdx.x - seg * chains;
    const int row = chain / a.groups, c = (chain - row * a.groups) * 2 * P + 2 * cp;
    const bool on = c < a.D;
    const int T_ = (kThreads >> a.log2p) * S;
    const int len = a.lengths ? min(max(a.lengths[row], 0), a.L) : a.L;
    if (tid == 0) sh.abort_flag = 0;
    const T *xp = a.x + row * a.x_b + c, *gp = a.g + row * a.g_b + c, *dyp = a.dy + row * a.dy_b + c;
    T *dxp = a.dx + row * a.dx_b + c, *dgp = a.dg + row * a.dg_b + c;
    float2 carry = make_float2(0.f, 0.f);       // C at the end of the wave
    if (a.state_in && on) carry = *reinterpret_cast<const float2 *>(a.state_in + (int64_t)row * a.D + c);
    // A chunk of saved-state distance is kChunk / S runs: 8 lanes-by-P of one warp or several warps.
    const int wpc = max(1, (kChunk / S) * P / 32);

    Raw xr[S], gr[S], dr[S];
    float2 hs;                                   // the saved state before the thread's chunk
    auto load = [&](int tile) {
        const int t0 = tile * T_ + sc * S;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const bool ok = on && t0 + i < len;
            xr[i] = ok ? Pair<T>::load(xp + (int64_t)(t0 + i) * a.x_l) : Pair<T>::zero();
            gr[i] = ok ? Pair<T>::load(gp + (int64_t)(t0 + i) * a.g_l) : Pair<T>::zero();
            dr[i] = ok ? Pair<T>::load(dyp + (int64_t)(t0 + i) * a.dy_l) : Pair<T>::zero();
        }
        hs = make_float2(0.f, 0.f);
        if (on && t0 < len)
            hs = __ldg(reinterpret_cast<const float2 *>(a.saved + ((int64_t)row * a.nchunks + t0 / kChunk) * a.D + c));
    };
    load(a.ntiles - 1 - seg);
    __syncthreads();
    int wave = 0;
    for (int back = seg; back < a.ntiles; back += a.nseg, ++wave) {
        const int tile = a.ntiles - 1 - back, t0 = tile * T_ + sc * S;
        Raw xs[S], ds[S];
        float2 b[S];
        float4 f = identity4(), r = identity4();
        float2 h = hs;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const float2 g = Pair<T>::value(gr[i]);
            const bool ok = t0 + i < len;
            b[i] = ok ? make_float2(rest(g.x), rest(g.y)) : make_float2(0.f, 0.f);
            xs[i] = xr[i];
            ds[i] = dr[i];
            const float2 x = Pair<T>::value(xs[i]);
            f.x = fmaf(-b[i].x, f.x, f.x);
            f.y = fmaf(-b[i].y, f.y, f.y);
            f.z = kLeak ? fmaf(b[i].x, x.x - f.z, f.z) : fmaf(-b[i].x, f.z, f.z + x.x);
            f.w = kLeak ? fmaf(b[i].y, x.y - f.w, f.w) : fmaf(-b[i].y, f.w, f.w + x.y);
        }
        r.x = f.x;
        r.y = f.y;
#pragma unroll
        for (int i = S - 1; i >= 0; --i) {
            const float2 d = Pair<T>::value(ds[i]);
            const float gx = d.x + r.z, gy = d.y + r.w;
            r.z = fmaf(-b[i].x, gx, gx);
            r.w = fmaf(-b[i].y, gy, gy);
        }
        if (back + a.nseg < a.ntiles) load(tile - a.nseg);
        // Forward runs since the chunk's start (within the warp: only lanes of the same chunk).
        float4 excl;
        {
            const int run = (lane >> a.log2p) & (kChunk / S - 1);      // place within the chunk's lanes
            float4 v = f;
            for (int d = 1; (d << a.log2p) < 32; d <<= 1) {
                const float4 o = shfl4(v, (lane - (d << a.log2p)) & 31);
                if (run >= d && lane >= (d << a.log2p)) v = compose(o, v);
            }
            const float4 o = shfl4(v, (lane - P) & 31);
            excl = run >= 1 && lane >= P ? o : identity4();
            if (lane >= 32 - P) sh.run[wave & 1][warp][cp] = v;
        }
        const float4 rincl = lane_scan<true>(r, P, lane);
        const float4 rexcl = lane_exclusive<true>(rincl, P, lane);
        if (lane < P) rev[wave & 1][warp][cp] = rincl;
        __syncthreads();
        float4 before = identity4();
        const int w0 = warp - warp % wpc;
        for (int w = w0; w < warp; ++w) before = compose(before, sh.run[wave & 1][w][cp]);
        h = apply(compose(before, excl), h);
        float4 after = identity4(), total = identity4();
#pragma unroll
        for (int w = kWarps - 1; w >= 0; --w) {
            if (w == warp) after = total;
            total = compose(total, rev[wave & 1][w][cp]);
        }
        after = compose(after, rexcl);
        float2 C;
        if (a.nseg > 1) {
            float4 pre, all;
            exchange(total, a.agg + (int64_t)chain * 2 * a.nseg * 32, a.flag + (int64_t)chain * a.nseg, wave, seg,
                     a.nseg, min(a.nseg, a.ntiles - wave * a.nseg), P, cp, sh, &pre, &all);
            C = apply(after, apply(pre, carry));
            carry = apply(all, carry);
        } else {
            C = apply(after, carry);
            carry = apply(total, carry);
        }
        float2 hp[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const float2 x = Pair<T>::value(xs[i]);
            hp[i] = h;
            h.x = kLeak ? fmaf(b[i].x, x.x - h.x, h.x) : fmaf(-b[i].x, h.x, h.x + x.x);
            h.y = kLeak ? fmaf(b[i].y, x.y - h.y, h.y) : fmaf(-b[i].y, h.y, h.y + x.y);
        }
#pragma unroll
        for (int i = S - 1; i >= 0; --i) {
            const float2 x = Pair<T>::value(xs[i]), d = Pair<T>::value(ds[i]);
            const float gx = d.x + C.x, gy = d.y + C.y;
            C.x = fmaf(-b[i].x, gx, gx);                // a G
            C.y = fmaf(-b[i].y, gy, gy);
            if (on && t0 + i < a.L) {
                const bool ok = t0 + i < len;
                const float2 zero = make_float2(0.f, 0.f);
                float2 vx, vg;
                vx.x = kLeak ? b[i].x * gx : gx;
                vx.y = kLeak ? b[i].y * gy : gy;
                vg.x = C.x * b[i].x * (kLeak ? hp[i].x - x.x : hp[i].x);
                vg.y = C.y * b[i].y * (kLeak ? hp[i].y - x.y : hp[i].y);
                Pair<T>::store(dxp + (int64_t)(t0 + i) * a.dx_l, ok ? vx : zero);
                Pair<T>::store(dgp + (int64_t)(t0 + i) * a.dg_l, ok ? vg : zero);
            }
        }
        if (tile == 0 && a.state_out && on && sc == 0)
            *reinterpret_cast<float2 *>(a.state_out + (int64_t)row * a.D + c) = C;
    }
}

// One token for each row: a thread per channel pair.  Bound by the launch up to a few
// hundred thousand channels, by the state's 8 bytes a channel beyond.
template <typename T, bool kLeak>
__global__ void __launch_bounds__(256) k_scan_step(const T *x, const T *g, T *y, int64_t x_b, int64_t g_b, int64_t y_b,
                                                   float *state, int half, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (i < n) {
        int64_t row;
        int c;
        if (n <= 0x7fffffff) {
            row = (unsigned)i / (unsigned)half;
            c = 2 * (int)((unsigned)i - (unsigned)row * half);
        } else {
            row = i / half;
            c = 2 * (int)(i - row * half);
        }
        // Plain loads: the previous kernel may still have been writing these when this one started.
        using Raw = typename Pair<T>::Raw;
        const float2 gv = Pair<T>::value(*reinterpret_cast<const Raw *>(g + row * g_b + c));
        const float2 xv = Pair<T>::value(*reinterpret_cast<const Raw *>(x + row * x_b + c));
        float2 *sp = reinterpret_cast<float2 *>(state) + i;
        float2 h = *sp;
        const float bx = rest(gv.x), by = rest(gv.y);
        h.x = kLeak ? fmaf(bx, xv.x - h.x, h.x) : fmaf(-bx, h.x, h.x + xv.x);
        h.y = kLeak ? fmaf(by, xv.y - h.y, h.y) : fmaf(-by, h.y, h.y + xv.y);
        *sp = h;
        Pair<T>::store(y + row * y_b + c, h);
    }
    asm volatile("griddepcontrol.launch_dependents;" :::);
}

struct ScanPlan {
    int log2p, groups, tile, ntiles, nseg;
    int64_t chains;
};

// Resident CTAs of the scan kernels: two per SM (their launch bounds).
ScanPlan scan_plan(int64_t B, int64_t L, int D, int run) {
    ScanPlan p;
    p.log2p = 2;
    while (p.log2p < 5 && (2 << p.log2p) < D) ++p.log2p;
    p.groups = (D + (2 << p.log2p) - 1) / (2 << p.log2p);
    p.tile = (kThreads >> p.log2p) * run;
    p.ntiles = (int)((L + p.tile - 1) / p.tile);
    p.chains = B * p.groups;
    // As many segments as keep every CTA resident, evened out over the waves.
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(p.ntiles, 2 * (int64_t)sm_count() / p.chains));
    const int waves = (int)((p.ntiles + most - 1) / most);
    p.nseg = (p.ntiles + waves - 1) / waves;
    return p;
}

size_t plan_ws_bytes(const ScanPlan &p) {
    if (p.nseg < 2) return 0;
    return (size_t)p.chains * p.nseg * (2 * 32 * sizeof(float4) + sizeof(unsigned));
}

int forward_run(rlm_dtype dt) { return dt == RLM_BF16 ? kFwdRun<__nv_bfloat16> : kFwdRun<float>; }

template <typename T>
cudaError_t launch_scan(void (*kernel)(const ScanArgs<T>), ScanArgs<T> &a, const ScanPlan &p, void *ws,
                        cudaStream_t st) {
    a.groups = p.groups;
    a.log2p = p.log2p;
    a.nseg = p.nseg;
    a.ntiles = p.ntiles;
    a.nchunks = (a.L + kChunk - 1) / kChunk;
    const dim3 grid((unsigned)(p.chains * p.nseg));
    count_launches(1);
    if (p.nseg < 2) {
        a.agg = nullptr;
        a.flag = nullptr;
        kernel<<<grid, kThreads, 0, st>>>(a);
        return cudaGetLastError();
    }
    a.agg = static_cast<float4 *>(ws);
    a.flag = reinterpret_cast<unsigned *>(a.agg + (size_t)p.chains * p.nseg * 2 * 32);
    cudaError_t e = cudaMemsetAsync(a.flag, 0, (size_t)p.chains * p.nseg * sizeof(unsigned), st);
    if (e != cudaSuccess) return e;
    void *args[] = {&a};
    return cudaLaunchCooperativeKernel(reinterpret_cast<const void *>(kernel), grid, dim3(kThreads), args, 0, st);
}

template <typename T>
cudaError_t forward_t(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak, const float *sin,
                      float *sout, float *saved, const int *lengths, void *ws, cudaStream_t st) {
    ScanArgs<T> a = {};
    a.x = static_cast<const T *>(x.ptr);
    a.g = static_cast<const T *>(g.ptr);
    a.y = static_cast<T *>(y.ptr);
    a.x_b = x.stride_b, a.x_l = x.stride_l, a.g_b = g.stride_b, a.g_l = g.stride_l;
    a.y_b = y.stride_b, a.y_l = y.stride_l;
    a.state_in = sin;
    a.state_out = sout;
    a.saved = saved;
    a.lengths = lengths;
    a.L = (int)x.L;
    a.D = (int)x.D;
    return launch_scan(leak ? k_scan_forward<T, true> : k_scan_forward<T, false>, a,
                       scan_plan(x.B, x.L, (int)x.D, kFwdRun<T>), ws, st);
}

template <typename T>
cudaError_t backward_t(const rlm_strided &dy, const rlm_strided &x, const rlm_strided &g, const float *saved, bool leak,
                       const float *dsout, const rlm_strided &dx, const rlm_strided &dg, float *dsin,
                       const int *lengths, void *ws, cudaStream_t st) {
    ScanArgs<T> a = {};
    a.x = static_cast<const T *>(x.ptr);
    a.g = static_cast<const T *>(g.ptr);
    a.dy = static_cast<const T *>(dy.ptr);
    a.dx = static_cast<T *>(dx.ptr);
    a.dg = static_cast<T *>(dg.ptr);
    a.x_b = x.stride_b, a.x_l = x.stride_l, a.g_b = g.stride_b, a.g_l = g.stride_l;
    a.dy_b = dy.stride_b, a.dy_l = dy.stride_l, a.dx_b = dx.stride_b, a.dx_l = dx.stride_l;
    a.dg_b = dg.stride_b, a.dg_l = dg.stride_l;
    a.state_in = dsout;
    a.state_out = dsin;
    a.saved = const_cast<float *>(saved);
    a.lengths = lengths;
    a.L = (int)x.L;
    a.D = (int)x.D;
    return launch_scan(leak ? k_scan_backward<T, true> : k_scan_backward<T, false>, a,
                       scan_plan(x.B, x.L, (int)x.D, kBwdRun), ws, st);
}

template <typename T>
cudaError_t step_t(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak, float *state,
                   cudaStream_t st) {
    const int half = (int)(x.D / 2);
    const int64_t n = x.B * half;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((n + 255) / 256));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launches(1);
    return cudaLaunchKernelEx(&cfg, leak ? k_scan_step<T, true> : k_scan_step<T, false>, static_cast<const T *>(x.ptr),
                              static_cast<const T *>(g.ptr), static_cast<T *>(y.ptr), x.stride_b, g.stride_b,
                              y.stride_b, state, half, n);
}

}  // namespace

size_t scan_ws_bytes(int64_t B, int64_t L, int D, rlm_dtype dt) {
    return std::max(plan_ws_bytes(scan_plan(B, L, D, forward_run(dt))), plan_ws_bytes(scan_plan(B, L, D, kBwdRun)));
}

cudaError_t scan_forward(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak,
                         const float *state_in, float *state_out, float *saved, const int *lengths, void *ws,
                         cudaStream_t st) {
    if (x.dtype == RLM_BF16)
        return forward_t<__nv_bfloat16>(x, g, y, leak, state_in, state_out, saved, lengths, ws, st);
    return forward_t<float>(x, g, y, leak, state_in, state_out, saved, lengths, ws, st);
}

cudaError_t scan_backward(const rlm_strided &dy, const rlm_strided &x, const rlm_strided &g, const float *saved,
                          bool leak, const float *d_state_out, const rlm_strided &dx, const rlm_strided &dg,
                          float *d_state_in, const int *lengths, void *ws, cudaStream_t st) {
    if (x.dtype == RLM_BF16)
        return backward_t<__nv_bfloat16>(dy, x, g, saved, leak, d_state_out, dx, dg, d_state_in, lengths, ws, st);
    return backward_t<float>(dy, x, g, saved, leak, d_state_out, dx, dg, d_state_in, lengths, ws, st);
}

cudaError_t scan_step(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak, float *state,
                      cudaStream_t st) {
    if (x.dtype == RLM_BF16) return step_t<__nv_bfloat16>(x, g, y, leak, state, st);
    return step_t<float>(x, g, y, leak, state, st);
}

cudaError_t read_and_clear_scan_status(int *status, cudaStream_t st) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(status, g_scan_status, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
    if (e != cudaSuccess) return e;
    if ((e = cudaStreamSynchronize(st)) != cudaSuccess) return e;
    if (*status == RLM_OK) return cudaSuccess;
    const int zero = 0;
    if ((e = cudaMemcpyToSymbolAsync(g_scan_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, st)) != cudaSuccess)
        return e;
    return cudaStreamSynchronize(st);
}

}  // namespace rlm
