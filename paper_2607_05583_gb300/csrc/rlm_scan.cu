// rlm_scan.cu -- the gated linear recurrence: sequence form, gradients, one step.
//
//   a_t = sigma(g_t),  h_t = a_t h_{t-1} + i_t,  i_t = (1 - a_t) x_t (leak) or x_t
//
// per channel.  The smaller of a and b = 1 - a is formed directly, b = 1 / (1 + e^g) where gates
// are open and a = e^g b where they are closed: as a difference from 1 either would lose its
// leading bits (2 % of the gradients at g = -15).  The kernels keep one number, q = -b or q = a,
// whose sign says which, and
//   a v = [q < 0] v + q v         b v = [q > 0] v - q v         a b = |q| (1 - |q|)
//   leak  h = [q < 0 ? h : x] + q (h - x)         unit  h = x + a h
// lose nothing at any gate, and keep and forget exactly where it saturates.  Where all gates of a
// warp's runs have a > 1 / 32, q is -b and the selections go: they are two thirds of a token's
// arithmetic (bf16, B = 4, L = 32768, D = 512, gates 2.5 + 1.5 N(0, 1): 86 and 132 us forward and
// backward; gates -2.5 + 1.5 N(0, 1), where no warp is without a closed one: 125 and 188 us).
//
// A run of tokens maps the state by h -> A h + H (A the product of its a, H its end
// state from zero), and runs compose: (A2, H2) o (A1, H1) = (A2 A1, A2 H1 + H2).
// The gradient is the same scan with time reversed: with C_t the gradient that
// reaches h_{t-1}, G_t = dy_t + C_{t+1} and C_t = a_t G_t; then
//   leak  dx = b G, dg = a b G (h_{t-1} - x)      unit  dx = G, dg = a b G h_{t-1}.
//
// Bound by memory: 3 fields move in the forward pass and 5 in the backward pass, and
// each is read once.  At the measured copy rate an SM has about 33 instructions for each
// bf16 element of the forward pass, so the arithmetic runs on channel pairs as packed
// fp32 (f32x2); the selections by q's sign go half by half.
//
// Tiles.  Eight data warps of a CTA cover P channel pairs (P = 4, 8, 16 or 32) by
// 256 / P runs of kS = 8 tokens, a thread per run and pair.  A warp copies the rows
// that its own threads need (16-byte cp.async, out-of-range rows and padding filled
// with zeros) into a private ring of kStages tiles, so no barrier guards the data.
// A thread composes its run (first pass), keeps q in registers, and once it knows the
// state at the run's start walks the run again for the outputs (second pass).
//
// Two more warps turn runs into states, a tile each in turn.  A lane holds one channel pair
// of 8 consecutive runs (64 tokens, one saved chunk): it composes them, scans across
// lanes, adds the carry (which one warp hands the other) and gives every run its start
// state.  The data warps work on other tiles meanwhile: the second pass of tile w follows
// the first pass of tile w + 1 (that of w + 2 costs more, by the code of a third tile: 49
// against 47 us in bf16 at B = 4, L = 32768, D = 256, 91 against 71 us without segments).  x,
// needed again then, and g, needed once, have rings of their own: two CTAs per SM in fp32 (73
// -> 66 us).  (One such warp took 3100 cycles a tile where a cluster shares a chain, half of
// them the exchange, and bounded the kernel: 54 us at B = 4, L = 32768, D = 256.)
//
// Segments.  Few channels would leave SMs idle, so a cluster of nseg CTAs (2, 4 or 8)
// shares a chain of tiles: in wave w CTA s takes tile w nseg + s and sends the tile's
// (A, H) into every member's shared memory (st.async, which also completes the
// receiver's mbarrier, so data and readiness arrive together).  Each member composes the
// entries before its own on top of the carry, and all of them for the next wave's carry.
// Nobody waits for a neighbour's output: a wave costs one exchange, whatever nseg is, and
// no field is read twice.  Every wait is bounded.  The order of all products and sums is
// fixed by the shape: results repeat bit for bit.
//
// Measured, forward and backward, gates 2.5 + 1.5 N(0, 1): bf16, B = 256, L = 512, D = 512, no
// segments, 71 and 110 us, 84 and 90 % of the copy rate; bf16, B = 4, L = 32768, 8 segments, 86
// and 132 us with D = 512 (69 and 75 %), 47 and 73 us with D = 256; fp32, D = 256, 64 and 111 us.  With
// segments the data warps' own latency bounds a wave (40 % of issue slots, a third of the
// stalls at the hand-over).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "rlm_device.cuh"
#include "rlm_internal.h"

namespace rlm {

__device__ int g_scan_status = 0;
static std::atomic<bool> g_scan_waits{false};        // whether a kernel that may set it was launched

namespace {

constexpr int kDataThreads = 256;
constexpr int kThreads = kDataThreads + 64;         // and the two warps that turn runs into states
constexpr int kS = 8;                               // tokens of a run
constexpr int kBarRuns = 1, kBarStates = 3, kBarCarry = 5;      // named barriers, two each by a tile's parity
constexpr int kHandOver = kDataThreads + 32;        // threads of the first two: the data warps and one state warp
constexpr int kChunk = RLM_SCAN_CHUNK;              // tokens between saved states
constexpr long long kWaitLimit = 4000000000ll;      // SM cycles: about 2 s

// Two neighbouring channels of a field, as loaded and as values.
template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
    using Raw = uint32_t;
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
    static __device__ __forceinline__ float2 value(Raw r) { return r; }
    static __device__ __forceinline__ void store(float *p, float2 v) { __stcs(reinterpret_cast<float2 *>(p), v); }
};

template <typename T>
struct ScanArgs {
    const T *x, *g, *dy;
    T *y, *dx, *dg;
    int64_t x_b, x_l, g_b, g_l, dy_b, dy_l, y_b, y_l, dx_b, dx_l, dg_b, dg_l;   // strides in elements
    const float *state_in;      // forward: h_{-1}; backward: dl/dh_{L-1}; nullable (zero)
    float *state_out;           // forward: h_{L-1}; backward: dl/dh_{-1}; nullable
    float *saved;               // [B][ceil(L / kChunk)][D]: h before each chunk (forward: nullable output)
    const int *lengths;         // nullable, [B]
    int L, D, groups, nseg, ntiles, nchunks;
};

constexpr f32x2 kOne = 0x3f8000003f800000ull, kMinus = 0xbf800000bf800000ull, kKeep = 0x8000000080000000ull;   // (q of a = 1)

// Gates whose b passes this (g below -3.43) count as closed.  b is within 2^-23 (1 + e and its
// reciprocal), so short of it v - b v is within 2^-18 of a v.
constexpr float kClosed = 31.f / 32.f;

// A run of two channels: h -> A h + H.
struct alignas(16) Run {
    f32x2 A, H;
};
__device__ __forceinline__ Run identity() { return {kOne, 0}; }
__device__ __forceinline__ f32x2 apply(Run f, f32x2 h) { return fma2(f.A, h, f.H); }
__device__ __forceinline__ Run compose(Run earlier, Run later) { return {mul2(later.A, earlier.A), apply(later, earlier.H)}; }
__device__ __forceinline__ Run shuffle(Run v, int src) { return {__shfl_sync(~0u, v.A, src), __shfl_sync(~0u, v.H, src)}; }

// Inclusive scan over the lanes of one channel pair (P apart); kRev: over those after.
template <bool kRev, int P>
__device__ __forceinline__ Run lane_scan(Run v, int lane) {
#pragma unroll
    for (int d = P; d < 32; d <<= 1) {
        const int src = kRev ? lane + d : lane - d;
        const Run o = shuffle(v, src & 31);
        if (kRev ? src < 32 : src >= 0) v = compose(o, v);
    }
    return v;
}
// The same, without this lane's own run.
template <bool kRev, int P>
__device__ __forceinline__ Run lane_exclusive(Run incl, int lane) {
    if (P == 32) return identity();
    const int src = kRev ? lane + P : lane - P;
    const Run o = shuffle(incl, src & 31);
    return (kRev ? src < 32 : src >= 0) ? o : identity();
}

template <int kCount = kHandOver>
__device__ __forceinline__ void bar_sync(int id) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kCount) : "memory");
}
template <int kCount = kHandOver>
__device__ __forceinline__ void bar_arrive(int id) {
    asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kCount) : "memory");
}

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

constexpr int kMaxSeg = 8;      // portable cluster size

// What a cluster's members send one another: tile runs, four waves' worth (see exchange()).
constexpr int kWaves = 4;
template <int P>
struct Peers {
    Run run[kWaves][kMaxSeg][P];
    unsigned long long full[kWaves];    // mbarriers: one arrival (this CTA's) and the entries' bytes
};

// Bounded wait; after a timeout (now or earlier) the kernel runs on with what is there.
__device__ __forceinline__ void wait_full(uint32_t bar, uint32_t parity, bool &gave_up) {
    long long t0 = 0;
    for (uint32_t it = 1;; ++it) {
        uint32_t ok;
        asm volatile(
            "{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok || gave_up) return;
        if ((it & 255u) == 0) {
            const long long now = clock64();
            if (t0 == 0) {
                t0 = now;
            } else if (now - t0 > kWaitLimit) {
                gave_up = true;
                atomicExch(&g_scan_status, (int)RLM_ERR_TIMEOUT);
            }
        }
    }
}

// One wave's exchange by its state warp: sends this tile's run `mine` (held by every lane of a
// pair) to all members and returns the composition of the tiles before it (*pre) and of the
// whole wave.  A member's warp sends wave w + 4 into the place of wave w after its own wave
// w + 2, which took this CTA's run of wave w + 2, sent by the warp that read wave w just before.
template <int P>
__device__ __forceinline__ void exchange(Run mine, Peers<P> &peers, int wave, int seg, int nseg, int cp, bool &gave_up,
                                         Run *pre, Run *all) {
    const int lane = threadIdx.x & 31, at = wave % kWaves;
    const uint32_t bar = smem_u32(&peers.full[at]), slot = smem_u32(&peers.run[at][seg][cp]);
    if (lane == 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(nseg * P * 16) : "memory");
    for (int s = lane / P; s < nseg; s += 32 / P) {
        uint32_t to, tb;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(slot), "r"(s));
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(tb) : "r"(bar), "r"(s));
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(to),
                     "l"(mine.A), "l"(mine.H), "r"(tb)
                     : "memory");
    }
    wait_full(bar, (wave / kWaves) & 1, gave_up);
    Run v[kMaxSeg];
#pragma unroll
    for (int s = 0; s < kMaxSeg; ++s) v[s] = s < nseg ? peers.run[at][s][cp] : identity();
    Run f = identity();
    *pre = f;
#pragma unroll
    for (int s = 0; s < kMaxSeg; ++s) {
        if (s == seg) *pre = f;
        f = compose(f, v[s]);
    }
    *all = f;
    __syncwarp();
}

// A state warp's share of a wave once its tile's run is known: exchange, the carry from the
// other state warp, the next wave's carry to it.  Returns the state before the tile.
template <int P>
__device__ __forceinline__ f32x2 carry_over(Run total, Peers<P> &peers, f32x2 (&carries)[2][32], f32x2 &carry, int wave, int n,
                                            int seg, int nseg, int cp, bool &gave_up) {
    Run pre = identity(), all = total;
    if (nseg > 1) exchange<P>(total, peers, wave, seg, nseg, cp, gave_up, &pre, &all);
    if (wave > 0) {
        bar_sync<64>(kBarCarry + ((wave - 1) & 1));
        carry = carries[(wave - 1) & 1][cp];
    }
    const f32x2 h = apply(pre, carry);
    carry = apply(all, carry);
    if (wave + 1 < n) {
        if ((threadIdx.x & 31) < P) carries[wave & 1][cp] = carry;
        bar_arrive<64>(kBarCarry + (wave & 1));
    }
    return h;
}

// Set-up and end of a cluster: no member sends before all have their barriers, none
// leaves while another may still send to it.
template <int P>
__device__ __forceinline__ void open_peers(Peers<P> &peers, int nseg) {
    if (nseg < 2) return;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kWaves; ++i)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&peers.full[i])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_sync();
}
__device__ __forceinline__ void close_peers(int nseg) {
    if (nseg > 1) cluster_sync();
}

// What the warps of one scan CTA share.
struct Where {
    int lane, warp, P, cp, sc, seg, row, c, tile_tokens, len, n;
    bool on;
};

template <int kLog2P, typename T>
__device__ __forceinline__ Where where(const ScanArgs<T> &a) {
    Where w;
    const int tid = threadIdx.x;
    w.lane = tid & 31;
    w.warp = tid >> 5;
    w.P = 1 << kLog2P;
    w.cp = tid & (w.P - 1);
    w.sc = tid >> kLog2P;
    const int chain = blockIdx.x / a.nseg;          // a cluster is one chain
    w.seg = blockIdx.x - chain * a.nseg;
    w.row = chain / a.groups;
    w.c = (chain - w.row * a.groups) * 2 * w.P + 2 * w.cp;
    w.on = w.c < a.D;
    w.tile_tokens = (kDataThreads >> kLog2P) * kS;
    w.n = (a.ntiles + a.nseg - 1) / a.nseg;         // waves (in the last one, tiles past the end do nothing)
    return w;
}

// A warp's ring of tiles: kFields fields, 32 / P runs of kS rows, each run a row's size
// further on so that the runs' rows fall into different banks.
template <typename T, int kFields, int kStages, int kLog2P>
struct Ring {
    static constexpr int kRowBytes = 2 * (int)sizeof(T) << kLog2P;
    static constexpr int kRunBytes = (kS + 1) * kRowBytes;
    static constexpr int kFieldBytes = (32 >> kLog2P) * kRunBytes - kRowBytes;      // (no row after the last run)
    static constexpr int kStageBytes = kFields * kFieldBytes;
    static constexpr int kWarpBytes = kStages * kStageBytes;
    static constexpr int kBytes = kWarpBytes * (kDataThreads / 32);
    static constexpr int kPerRow = kRowBytes / 16;          // 16-byte copies a row
    static constexpr int kRows = (32 >> kLog2P) * kS;       // a warp's rows (tokens) of a tile
    static constexpr int kCopies = kRows * kPerRow / 32;    // copies a lane, a field
    static constexpr int kApart = 32 / kPerRow;             // rows between a lane's copies
    uint32_t base, dst, own;    // shared addresses: the warp's ring; a lane's first copy, its own values in a field
    int row, c;                 // row and channel of a lane's first copy

    __device__ __forceinline__ Ring(const Where &w, const void *smem) {
        base = (uint32_t)__cvta_generic_to_shared(smem) + w.warp * kWarpBytes;
        const int r = w.lane / kPerRow, col = w.lane % kPerRow;
        dst = base + place(r) + col * 16;
        row = w.warp * kRows + r;
        c = w.c - 2 * w.cp + col * (16 / (int)sizeof(T));
        own = base + (w.lane >> kLog2P) * kRunBytes + w.cp * 2 * (int)sizeof(T);
    }
    static __host__ __device__ constexpr int place(int r) { return (r / kS) * kRunBytes + (r % kS) * kRowBytes; }
    // Copies one field of the tile from token t0 on; p: the batch row's token 0 at the lane's channel.
    __device__ __forceinline__ void copy(int stage, int f, const T *p, int64_t stride, int t0, int tokens, int len,
                                         bool on) const {
        const uint32_t to = dst + stage * kStageBytes + f * kFieldBytes;
        const T *src = p + (int64_t)(t0 + row) * stride;
        if (on && t0 >= 0 && t0 + tokens <= len) {
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + place(k * kApart)), "l"(src)
                             : "memory");
                src += kApart * stride;
            }
        } else {
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
                const int t = t0 + row + k * kApart;
                const bool ok = on && t >= 0 && t < len;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + place(k * kApart)),
                             "l"(ok ? src : p), "r"(ok ? 16 : 0)
                             : "memory");
                src += kApart * stride;
            }
        }
    }
    // A thread's channel pair of token i of its run.
    __device__ __forceinline__ f32x2 value(int stage, int f, int i) const {
        const uint32_t at = own + stage * kStageBytes;
        const int off = f * kFieldBytes + i * kRowBytes;
        if constexpr (sizeof(T) == 2) {
            uint32_t r;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(at + off));
            return pack(Pair<T>::value(r));
        } else {
            f32x2 r;
            asm volatile("ld.shared.b64 %0, [%1];" : "=l"(r) : "r"(at + off));
            return r;
        }
    }
};
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncwarp();
}

__device__ __forceinline__ float exp2_approx(float v) {
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
    return e;
}
__device__ __forceinline__ float reciprocal_approx(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
constexpr f32x2 kLog2e = 0x3fb8aa3b3fb8aa3bull;

template <typename T>
__device__ __forceinline__ f32x2 exponential(f32x2 g) {
    if constexpr (sizeof(T) == 2) {
        const float2 p = unpack(mul2(g, kLog2e));
        return pack(make_float2(exp2_approx(p.x), exp2_approx(p.y)));
    }
    const float2 p = unpack(g);
    return pack(make_float2(expf(p.x), expf(p.y)));
}
// -b = -1 / (1 + e), e = e^g: q where gates are not closed; g = +inf gives -0.
__device__ __forceinline__ f32x2 minus_rest(f32x2 e) {
    const float2 d = unpack(fma2(e, kMinus, kMinus));
    return pack(make_float2(reciprocal_approx(d.x), reciprocal_approx(d.y)));
}
// q of any gate: a = e b where b > 1 / 2 (g = -inf gives +0; a below 2^-126 is 0), else -b.
__device__ __forceinline__ f32x2 smaller(f32x2 e, f32x2 minus_b) {
    f32x2 s;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(s) : "l"(e), "l"(minus_b ^ kKeep));
    const float2 a = unpack(s), r = unpack(minus_b);
    return pack(make_float2(r.x < -0.5f ? a.x : r.x, r.y < -0.5f ? a.y : r.y));
}

// A run's q, and whether all of the warp's runs are free of closed gates.
struct Gates {
    f32x2 q[kS];
    bool open;
};
template <typename T, typename Value>
__device__ __forceinline__ void gates_of(Gates &t, Value g) {
    float low = 0.f;
#pragma unroll
    for (int i = 0; i < kS; ++i) {
        t.q[i] = minus_rest(exponential<T>(g(i)));
        const float2 v = unpack(t.q[i]);
        low = fminf(low, fminf(v.x, v.y));
    }
    t.open = !__any_sync(~0u, low < -kClosed);
    if (!t.open) {
#pragma unroll
        for (int i = 0; i < kS; ++i) t.q[i] = smaller(exponential<T>(g(i)), t.q[i]);
    }
}

// Half by half: v where q < 0 (-0 among them), else o.
__device__ __forceinline__ f32x2 where_open(f32x2 q, f32x2 v, f32x2 o) {
    const float2 s = unpack(q), a = unpack(v), b = unpack(o);
    return pack(make_float2(__float_as_int(s.x) < 0 ? a.x : b.x, __float_as_int(s.y) < 0 ? a.y : b.y));
}
// a v; kOpen: q is -b throughout.
template <bool kOpen>
__device__ __forceinline__ f32x2 decayed(f32x2 q, f32x2 v) { return fma2(q, v, kOpen ? v : where_open(q, v, 0)); }
// One token.
template <bool kLeak, bool kOpen>
__device__ __forceinline__ f32x2 advance(f32x2 h, f32x2 q, f32x2 x) {
    if (kLeak) return fma2(q, fma2(x, kMinus, h), kOpen ? h : where_open(q, h, x));
    return fma2(q, h, add2(x, kOpen ? h : where_open(q, h, 0)));
}
template <bool kOpen>
using Open = std::integral_constant<bool, kOpen>;

// first(0), first(1), second(0), first(2), second(1), ...: each pass's q in one of two
// register arrays.
template <typename First, typename Second>
__device__ __forceinline__ void two_passes(int n, First first, Second second) {
    Gates even, odd;
    first(0, even);
    for (int k = 1;; k += 2) {
        if (k < n) first(k, odd);
        second(k - 1, even);
        if (k >= n) return;
        if (k + 1 < n) first(k + 1, even);
        second(k, odd);
        if (k + 1 >= n) return;
    }
}

// Resident CTAs per SM: what the rings leave room for.
template <typename T>
constexpr int kBwdPerSm = sizeof(T) == 2 ? 2 : 1;

// ----------------------------------------------------------------- forward
// Tiles of g (needed until the first pass) and of x (until the second, a tile later) in the ring.
template <typename T>
constexpr int kGStages = sizeof(T) == 2 ? 3 : 2;
template <typename T>
constexpr int kXStages = kGStages<T> + 1;
template <typename T, int kLog2P>
using XRing = Ring<T, 1, kXStages<T>, kLog2P>;
template <typename T, int kLog2P>
using GRing = Ring<T, 1, kGStages<T>, kLog2P>;

template <typename T, bool kLeak, int kLog2P>
__global__ void __launch_bounds__(kThreads, 2) k_scan_forward(const ScanArgs<T> a) {
    extern __shared__ __align__(16) unsigned char ring_mem[];
    __shared__ Peers<1 << kLog2P> peers;
    constexpr int X = kXStages<T>, G = kGStages<T>;
    __shared__ Run runs[2][kDataThreads];
    __shared__ f32x2 states[2][kDataThreads], carries[2][32];
    constexpr int P = 1 << kLog2P;
    Where w = where<kLog2P>(a);
    open_peers(peers, a.nseg);
    wait_for_previous();
    w.len = a.lengths ? min(max(a.lengths[w.row], 0), a.L) : a.L;

    if (w.warp >= kDataThreads / 32) {
        // Runs to states, the two warps in turn: lane (part, cp) holds runs 8 part .. 8 part + 7.
        const int first = (w.lane / P) * 8 * P + w.cp, me = w.warp - kDataThreads / 32;
        f32x2 carry = 0;
        if (a.state_in && w.on) carry = pack(*reinterpret_cast<const float2 *>(a.state_in + (int64_t)w.row * a.D + w.c));
        bool gave_up = false;
        for (int k = me; k < w.n; k += 2) {
            const int par = k & 1, tile = k * a.nseg + w.seg;
            bar_sync(kBarRuns + par);
            Run f = identity();
#pragma unroll
            for (int j = 0; j < 8; ++j) f = compose(f, runs[par][first + j * P]);
            const Run incl = lane_scan<false, P>(f, w.lane), excl = lane_exclusive<false, P>(incl, w.lane);
            const Run total = P == 32 ? incl : shuffle(incl, 32 - P + w.cp);
            f32x2 h = carry_over<P>(total, peers, carries, carry, k, w.n, w.seg, a.nseg, w.cp, gave_up);
            h = apply(excl, h);
            const int t0 = tile * w.tile_tokens + (w.lane / P) * kChunk;
            if (a.saved && w.on && t0 < a.L)
                *reinterpret_cast<float2 *>(a.saved + ((int64_t)w.row * a.nchunks + t0 / kChunk) * a.D + w.c) = unpack(h);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                states[par][first + j * P] = h;
                h = apply(runs[par][first + j * P], h);
            }
            bar_arrive(kBarStates + par);
        }
        // Every member holds the same carry.  state_out may be state_in: all members have read it.
        close_peers(a.nseg);
        if (a.state_out && w.on && w.lane < P && w.seg == 0 && me == ((w.n - 1) & 1))
            *reinterpret_cast<float2 *>(a.state_out + (int64_t)w.row * a.D + w.c) = unpack(carry);
        return;
    }

    const XRing<T, kLog2P> xs(w, ring_mem);
    const GRing<T, kLog2P> gs(w, ring_mem + XRing<T, kLog2P>::kBytes);
    const bool on = xs.c < a.D;
    const T *xp = a.x + w.row * a.x_b + (on ? xs.c : 0), *gp = a.g + w.row * a.g_b + (on ? xs.c : 0);
    T *yp = a.y + w.row * a.y_b + w.c;
    auto copy = [&](int k) {
        if (k < w.n) {
            const int t0 = (k * a.nseg + w.seg) * w.tile_tokens;
            xs.copy(k % X, 0, xp, a.x_l, t0, w.tile_tokens, w.len, on);
            gs.copy(k % G, 0, gp, a.g_l, t0, w.tile_tokens, w.len, on);
        }
        copies_commit();
    };
#pragma unroll
    for (int k = 0; k < G; ++k) copy(k);
    auto first = [&](int k, Gates &t) {
        // Copies are one group a tile, asked for G at the start, one after the first tile's first pass and
        // then one after each second pass: always G are open or to come, tile k the first.
        copies_wait<G - 1>();
        const int t0 = (k * a.nseg + w.seg) * w.tile_tokens + w.sc * kS;
        gates_of<T>(t, [&](int i) { return gs.value(k % G, 0, i); });
        if (t0 + kS > w.len) {                          // past the end: the identity (x is 0 there)
#pragma unroll
            for (int i = 0; i < kS; ++i)
                if (t0 + i >= w.len) t.q[i] = kKeep;
        }
        f32x2 A = kOne, H = 0;
        auto run = [&](auto open) {
            constexpr bool kOpen = decltype(open)::value;
#pragma unroll
            for (int i = 0; i < kS; ++i) {
                A = decayed<kOpen>(t.q[i], A);
                H = advance<kLeak, kOpen>(H, t.q[i], xs.value(k % X, 0, i));
            }
        };
        if (t.open) run(Open<true>{}); else run(Open<false>{});
        runs[k & 1][threadIdx.x] = {A, H};
        bar_arrive(kBarRuns + (k & 1));
        if (k == 0) {
            __syncwarp();
            copy(G);
        }
    };
    auto second = [&](int k, const Gates &t) {
        const int t0 = (k * a.nseg + w.seg) * w.tile_tokens + w.sc * kS;
        bar_sync(kBarStates + (k & 1));
        f32x2 h = states[k & 1][threadIdx.x];
        T *out = yp + (int64_t)t0 * a.y_l;
        if (t.open && t0 + kS <= w.len) {
            if (w.on) {
#pragma unroll
                for (int i = 0; i < kS; ++i) {
                    h = advance<kLeak, true>(h, t.q[i], xs.value(k % X, 0, i));
                    Pair<T>::store(out, unpack(h));
                    out += a.y_l;
                }
            }
        } else if (w.on) {
#pragma unroll
            for (int i = 0; i < kS; ++i) {
                h = advance<kLeak, false>(h, t.q[i], xs.value(k % X, 0, i));
                if (t0 + i < a.L) Pair<T>::store(out, t0 + i < w.len ? unpack(h) : make_float2(0.f, 0.f));
                out += a.y_l;
            }
        }
        __syncwarp();
        copy(k + X);            // x into the stage that this pass has just left
    };
    two_passes(w.n, first, second);
    close_peers(a.nseg);
}

// ---------------------------------------------------------------- backward
template <typename T>
constexpr int kBwdStages = 3;
template <typename T, int kLog2P>
using BwdRing = Ring<T, 3, kBwdStages<T>, kLog2P>;          // fields: x, g, dy

template <typename T, bool kLeak, int kLog2P>
__global__ void __launch_bounds__(kThreads, kBwdPerSm<T>) k_scan_backward(const ScanArgs<T> a) {
    extern __shared__ __align__(16) unsigned char ring_mem[];
    // Gradients are carried negated: the signs of b G and of a b G then fall into the fma.
    __shared__ Peers<1 << kLog2P> peers;
    __shared__ Run runs[2][kDataThreads];
    __shared__ f32x2 ends[2][kDataThreads];         // a run's -C from a zero C after it; then its -C
    __shared__ f32x2 states[2][kDataThreads], carries[2][32];
    constexpr int P = 1 << kLog2P;
    Where w = where<kLog2P>(a);
    constexpr int ST = kBwdStages<T>;
    open_peers(peers, a.nseg);
    wait_for_previous();
    w.len = a.lengths ? min(max(a.lengths[w.row], 0), a.L) : a.L;

    if (w.warp >= kDataThreads / 32) {
        // A lane's 8 runs are one chunk: their states follow from the chunk's saved state.
        const int part = w.lane / P, first = part * 8 * P + w.cp, me = w.warp - kDataThreads / 32;
        f32x2 carry = 0;                            // -C after the wave
        if (a.state_in && w.on)
            carry = mul2(pack(*reinterpret_cast<const float2 *>(a.state_in + (int64_t)w.row * a.D + w.c)), kMinus);
        auto saved_at = [&](int k) {
            const int t0 = (a.ntiles - 1 - (k * a.nseg + w.seg)) * w.tile_tokens + part * kChunk;
            if (k >= w.n || !w.on || t0 < 0 || t0 >= w.len) return make_float2(0.f, 0.f);
            return *reinterpret_cast<const float2 *>(a.saved + ((int64_t)w.row * a.nchunks + t0 / kChunk) * a.D + w.c);
        };
        bool gave_up = false;
        float2 next = saved_at(me);
        for (int k = me; k < w.n; k += 2) {
            const int par = k & 1;
            f32x2 h = pack(next);
            next = saved_at(k + 2);
            bar_sync(kBarRuns + par);
            auto reverse_run = [&](int j) { return Run{runs[par][first + j * P].A, ends[par][first + j * P]}; };
            Run f = identity();
#pragma unroll
            for (int j = 7; j >= 0; --j) f = compose(f, reverse_run(j));
            const Run incl = lane_scan<true, P>(f, w.lane), excl = lane_exclusive<true, P>(incl, w.lane);
            const Run total = P == 32 ? incl : shuffle(incl, w.cp);
            f32x2 C = carry_over<P>(total, peers, carries, carry, k, w.n, w.seg, a.nseg, w.cp, gave_up);
            C = apply(excl, C);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                states[par][first + j * P] = h;
                h = apply(runs[par][first + j * P], h);
            }
#pragma unroll
            for (int j = 7; j >= 0; --j) {
                const Run r = reverse_run(j);
                ends[par][first + j * P] = C;
                C = apply(r, C);
            }
            bar_arrive(kBarStates + par);
        }
        close_peers(a.nseg);
        if (a.state_out && w.on && w.lane < P && w.seg == 0 && me == ((w.n - 1) & 1))
            *reinterpret_cast<float2 *>(a.state_out + (int64_t)w.row * a.D + w.c) = unpack(mul2(carry, kMinus));
        return;
    }

    const BwdRing<T, kLog2P> ring(w, ring_mem);
    const bool on = ring.c < a.D;
    const int cc = on ? ring.c : 0;
    const T *xp = a.x + w.row * a.x_b + cc, *gp = a.g + w.row * a.g_b + cc, *dp = a.dy + w.row * a.dy_b + cc;
    T *dxp = a.dx + w.row * a.dx_b + w.c, *dgp = a.dg + w.row * a.dg_b + w.c;
    auto copy = [&](int k) {
        if (k < w.n) {
            const int t0 = (a.ntiles - 1 - (k * a.nseg + w.seg)) * w.tile_tokens;
            ring.copy(k % ST, 0, xp, a.x_l, t0, w.tile_tokens, w.len, on);
            ring.copy(k % ST, 1, gp, a.g_l, t0, w.tile_tokens, w.len, on);
            ring.copy(k % ST, 2, dp, a.dy_l, t0, w.tile_tokens, w.len, on);
        }
        copies_commit();
    };
#pragma unroll
    for (int k = 0; k < ST; ++k) copy(k);
    auto first = [&](int k, Gates &t) {
        if (k == 0) copies_wait<ST - 1>(); else copies_wait<ST - 2>();
        const int st = k % ST, t0 = (a.ntiles - 1 - (k * a.nseg + w.seg)) * w.tile_tokens + w.sc * kS;
        gates_of<T>(t, [&](int i) { return ring.value(st, 1, i); });
        if (t0 < 0 || t0 + kS > w.len) {
#pragma unroll
            for (int i = 0; i < kS; ++i)
                if (t0 < 0 || t0 + i >= w.len) t.q[i] = kKeep;
        }
        f32x2 A = kOne, H = 0, R = 0;
        auto run = [&](auto open) {
            constexpr bool kOpen = decltype(open)::value;
#pragma unroll
            for (int i = 0; i < kS; ++i) {
                A = decayed<kOpen>(t.q[i], A);
                H = advance<kLeak, kOpen>(H, t.q[i], ring.value(st, 0, i));
            }
#pragma unroll
            for (int i = kS - 1; i >= 0; --i) R = decayed<kOpen>(t.q[i], fma2(ring.value(st, 2, i), kMinus, R));
        };
        if (t.open) run(Open<true>{}); else run(Open<false>{});
        runs[k & 1][threadIdx.x] = {A, H};
        ends[k & 1][threadIdx.x] = R;
        bar_arrive(kBarRuns + (k & 1));
    };
    auto second = [&](int k, const Gates &t) {
        const int st = k % ST, t0 = (a.ntiles - 1 - (k * a.nseg + w.seg)) * w.tile_tokens + w.sc * kS;
        bar_sync(kBarStates + (k & 1));
        f32x2 h = states[k & 1][threadIdx.x], C = ends[k & 1][threadIdx.x];
        T *ox = dxp + (int64_t)(t0 + kS - 1) * a.dx_l, *og = dgp + (int64_t)(t0 + kS - 1) * a.dg_l;
        auto run = [&](auto open) {
            constexpr bool kOpen = decltype(open)::value;
            f32x2 v[kS];                                // h_{t-1} - x or h_{t-1}
#pragma unroll
            for (int i = 0; i < kS; ++i) {
                const f32x2 x = ring.value(st, 0, i);
                v[i] = kLeak ? fma2(x, kMinus, h) : h;
                h = advance<kLeak, kOpen>(h, t.q[i], x);
            }
            auto token = [&](int i, float2 &vx, float2 &vg) {
                const f32x2 q = t.q[i], G = fma2(ring.value(st, 2, i), kMinus, C);
                if (kOpen) {
                    C = fma2(q, G, G);                  // a G
                    vx = unpack(mul2(kLeak ? q : kMinus, G));
                    vg = unpack(mul2(mul2(C, q), v[i]));
                } else {
                    const f32x2 kept = where_open(q, G, 0);
                    C = fma2(q, G, kept);
                    vx = unpack(kLeak ? fma2(q, G, fma2(G, kMinus, kept)) : mul2(G, kMinus));
                    const f32x2 less = q | kKeep, n = mul2(less, mul2(G, v[i]));        // -|q|
                    vg = unpack(fma2(less, n, n));
                }
            };
            if (w.on && t0 >= 0 && t0 + kS <= w.len) {
#pragma unroll
                for (int i = kS - 1; i >= 0; --i) {
                    float2 vx, vg;
                    token(i, vx, vg);
                    Pair<T>::store(ox, vx);
                    Pair<T>::store(og, vg);
                    ox -= a.dx_l;
                    og -= a.dg_l;
                }
            } else if (w.on && t0 >= 0) {
#pragma unroll
                for (int i = kS - 1; i >= 0; --i) {
                    float2 vx, vg;
                    token(i, vx, vg);
                    if (t0 + i >= w.len) vx = vg = make_float2(0.f, 0.f);
                    if (t0 + i < a.L) {
                        Pair<T>::store(ox, vx);
                        Pair<T>::store(og, vg);
                    }
                    ox -= a.dx_l;
                    og -= a.dg_l;
                }
            }
        };
        if (t.open) run(Open<true>{}); else run(Open<false>{});
        __syncwarp();
        copy(k + ST);
    };
    two_passes(w.n, first, second);
    close_peers(a.nseg);
}

// One token for each row: a thread per channel pair.  Bound by the launch up to a few
// hundred thousand channels, by the state's 8 bytes a channel beyond.
template <typename T, bool kLeak>
__global__ void __launch_bounds__(256) k_scan_step(const T *x, const T *g, T *y, int64_t x_b, int64_t g_b, int64_t y_b,
                                                   float *state, int half, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    wait_for_previous();
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
        using Raw = typename Pair<T>::Raw;
        const float2 gv = Pair<T>::value(*reinterpret_cast<const Raw *>(g + row * g_b + c));
        const float2 xv = Pair<T>::value(*reinterpret_cast<const Raw *>(x + row * x_b + c));
        float2 *sp = reinterpret_cast<float2 *>(state) + i;
        const f32x2 e = exponential<T>(pack(gv)), q = smaller(e, minus_rest(e));
        const float2 h = unpack(advance<kLeak, false>(pack(*sp), q, pack(xv)));
        *sp = h;
        Pair<T>::store(y + row * y_b + c, h);
    }
}

template <typename T>
struct ScanKernel {
    void (*fn)(const ScanArgs<T>);
    int smem;
};
template <typename T, bool kLeak, int kLog2P>
ScanKernel<T> kernel_of(bool backward) {
    if (backward) return {k_scan_backward<T, kLeak, kLog2P>, BwdRing<T, kLog2P>::kBytes};
    return {k_scan_forward<T, kLeak, kLog2P>, XRing<T, kLog2P>::kBytes + GRing<T, kLog2P>::kBytes};
}
template <typename T, bool kLeak>
ScanKernel<T> kernel_of(bool backward, int log2p) {
    switch (log2p) {
        case 2: return kernel_of<T, kLeak, 2>(backward);
        case 3: return kernel_of<T, kLeak, 3>(backward);
        case 4: return kernel_of<T, kLeak, 4>(backward);
        default: return kernel_of<T, kLeak, 5>(backward);
    }
}

// Relative cost of a byte with rows of 4, 8, 16 and 32 channel pairs.
constexpr double kRowCost[4] = {1.6, 1.25, 1.02, 1.0};

struct ScanPlan {
    int log2p, groups, ntiles, nseg;
    int64_t chains;
};

// Resident CTAs of a kernel on the current device in clusters of nseg (a cluster's CTAs
// sit in one GPC, so large ones do not fill every SM).  Asked once for each kernel, whose shared
// memory size it sets.
template <typename T>
int64_t resident(const ScanKernel<T> &k, int nseg, std::atomic<int> &known) {
    const int ctas = known.load(std::memory_order_relaxed);
    if (ctas > 0) return ctas;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)nseg);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)k.smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)nseg;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, k.fn, &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    known.store(n * nseg, std::memory_order_relaxed);
    return (int64_t)n * nseg;
}

// With lengths, rounds after the first count for less: a CTA walks all waves of L whatever its
// row's length, but those past the row's end without memory, so short rows make some room.  A
// figure fitted to one shape: 0.35 + 0.65 rounds in place of rounds, forward and backward of
// bf16 B = 32, L = 1500, D = 320, lengths of 0 to L: 30.8 -> 24.7 and 56.4 -> 36.8 us (27 and 34
// now); the order of the rows by length changed either by 4 % at most.
constexpr double kFirstRound = 0.35;

// Channel pairs per CTA and segments per chain: the least of rounds of resident CTAs times
// a CTA's waves, with a few waves' worth for its start and end.
template <typename T>
ScanPlan scan_plan(int64_t B, int64_t L, int D, bool backward, bool leak, bool ragged) {
    static std::atomic<int> known[64][2][2][4][4];          // resident CTAs: device, direction, leak, pairs, segments
    int dev = 0;
    cudaGetDevice(&dev);
    ScanPlan best = {};
    double best_cost = 0;
    for (int lp = 5; lp >= 2; --lp) {
        if (lp > 2 && (2 << (lp - 1)) >= D) continue;       // a narrower group already holds the row
        const ScanKernel<T> k = leak ? kernel_of<T, true>(backward, lp) : kernel_of<T, false>(backward, lp);
        ScanPlan p;
        p.log2p = lp;
        p.groups = (D + (2 << lp) - 1) / (2 << lp);
        p.chains = B * p.groups;
        const int tile = (kDataThreads >> lp) * kS;
        p.ntiles = (int)((L + tile - 1) / tile);
        int at = 0;
        for (p.nseg = 1; p.nseg <= kMaxSeg && p.nseg <= p.ntiles; p.nseg *= 2, ++at) {
            const int64_t room = resident(k, p.nseg, known[dev & 63][backward][leak][lp - 2][at]);
            if (room < 1) continue;
            double rounds = (double)((p.chains * p.nseg + room - 1) / room);
            if (ragged) rounds = kFirstRound + (1 - kFirstRound) * rounds;
            const int waves = (p.ntiles + p.nseg - 1) / p.nseg;
            const double cost = rounds * (waves + 4) * kRowCost[lp - 2];
            if (best_cost == 0 || cost < best_cost * 0.999) {
                best_cost = cost;
                best = p;
            }
        }
    }
    return best;
}

template <typename T>
cudaError_t launch_scan(bool backward, bool leak, ScanArgs<T> &a, int64_t B, cudaStream_t st) {
    const ScanPlan p = scan_plan<T>(B, a.L, a.D, backward, leak, a.lengths != nullptr);
    if (p.nseg < 1) return cudaErrorInvalidConfiguration;
    const ScanKernel<T> k = leak ? kernel_of<T, true>(backward, p.log2p) : kernel_of<T, false>(backward, p.log2p);
    a.groups = p.groups;
    a.nseg = p.nseg;
    a.ntiles = p.ntiles;
    a.nchunks = (a.L + kChunk - 1) / kChunk;
    if (p.nseg > 1) g_scan_waits.store(true, std::memory_order_relaxed);
    // (resident() has set the kernel's shared memory size.)
    return launch_dependent(k.fn, dim3((unsigned)(p.chains * p.nseg)), kThreads, (size_t)k.smem, st, p.nseg, a);
}

template <typename T>
cudaError_t forward_t(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak, const float *sin,
                      float *sout, float *saved, const int *lengths, cudaStream_t st) {
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
    return launch_scan(false, leak, a, x.B, st);
}

template <typename T>
cudaError_t backward_t(const rlm_strided &dy, const rlm_strided &x, const rlm_strided &g, const float *saved, bool leak,
                       const float *dsout, const rlm_strided &dx, const rlm_strided &dg, float *dsin,
                       const int *lengths, cudaStream_t st) {
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
    return launch_scan(true, leak, a, x.B, st);
}

template <typename T>
cudaError_t step_t(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak, float *state,
                   cudaStream_t st) {
    const int half = (int)(x.D / 2);
    const int64_t n = x.B * half;
    return launch_dependent(leak ? k_scan_step<T, true> : k_scan_step<T, false>, dim3((unsigned)((n + 255) / 256)), 256, 0, st, 1,
                            static_cast<const T *>(x.ptr), static_cast<const T *>(g.ptr), static_cast<T *>(y.ptr), x.stride_b,
                            g.stride_b, y.stride_b, state, half, n);
}

}  // namespace

cudaError_t scan_forward(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak,
                         const float *state_in, float *state_out, float *saved, const int *lengths,
                         cudaStream_t st) {
    if (x.dtype == RLM_BF16)
        return forward_t<__nv_bfloat16>(x, g, y, leak, state_in, state_out, saved, lengths, st);
    return forward_t<float>(x, g, y, leak, state_in, state_out, saved, lengths, st);
}

cudaError_t scan_backward(const rlm_strided &dy, const rlm_strided &x, const rlm_strided &g, const float *saved,
                          bool leak, const float *d_state_out, const rlm_strided &dx, const rlm_strided &dg,
                          float *d_state_in, const int *lengths, cudaStream_t st) {
    if (x.dtype == RLM_BF16)
        return backward_t<__nv_bfloat16>(dy, x, g, saved, leak, d_state_out, dx, dg, d_state_in, lengths, st);
    return backward_t<float>(dy, x, g, saved, leak, d_state_out, dx, dg, d_state_in, lengths, st);
}

cudaError_t scan_step(const rlm_strided &x, const rlm_strided &g, const rlm_strided &y, bool leak, float *state,
                      cudaStream_t st) {
    if (x.dtype == RLM_BF16) return step_t<__nv_bfloat16>(x, g, y, leak, state, st);
    return step_t<float>(x, g, y, leak, state, st);
}

cudaError_t read_and_clear_scan_status(int *status, cudaStream_t st) {
    *status = RLM_OK;
    if (!g_scan_waits.load(std::memory_order_relaxed)) return cudaSuccess;
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
