// rlm_ssm_backward.cu -- gradients of the selective state space scan (mathematics and layout in rlm_ssm.cuh).
//
//   do = dy silu(z),  dz = dy o silu'(z),  G_t = C_t do_t + a_{t+1} G_{t+1}
//   dC_t = sum_d do_t h_t,  dB_t = sum_d G_t D_t x_t,  dx = skip do + D sum_n G B
//   dD = sum_n G (x B + A a h_{t-1}),  ddt = dD sigma(dt + bias),  dA = sum_t G D a h_{t-1}
//
// A thread owns 4 channels and 4 of their states, as in the forward pass; a block 64 channels.  Tiles are walked from
// the last to the first, each in runs of kRun tokens.  The forward pass kept the state before every tile: a first
// walk forms it again at the later runs' starts, then for each run, from the last, its states once more, which
// stay in registers until the walk back through the run has used them.  (Kept in shared memory for a tile of 32
// tokens, with one channel a thread, they left 4 warps on an SM: 657 us at B = 4, L = 4096, D = 1024, N = 16 in bf16,
// against 325.  With 2 channels a thread and runs of 8, 407: bound by shared memory's 128 bytes a clock.  Tiles of
// 32 tokens leave room for half the blocks; what the states between tiles of 16 move more is nothing beside the
// arithmetic.)  The G that reaches the tile before is the only thing carried.  Putting it right by the decays' product
// is 8 % of the time (351 us; N = 8, B = 16: 1.21 ms for 1.05).
//
// Sums over the state's n are left in shared memory as P shares a channel and added where they are used.  Sums over
// channels (dB, dC: 4 values each a thread and token) go over the thread's 4, then over the lanes of a warp that hold
// the same n by exchanging halves.  So that no value has to be selected for that, lanes hold their 4 states in an order
// of their own: index j is state j ^ q, q two bits of the lane, and what a lane sends is always the same
// registers' contents.  Then over the block's warps, and over the blocks by a second kernel, which also adds the
// parameters' gradients over batch rows and segments.  Every order is fixed by the shape.
//
// Segments as in the forward pass: k_reverse_ends forms what every segment but the first adds to the G
// before it, from a zero G behind it, and G's factor e^(A S).
#include <algorithm>

#include "rlm_ssm.cuh"

namespace rlm {
namespace ssm {
namespace {

template <typename T>
__device__ __forceinline__ float4 gated(const Four<T> &dy, const Four<T> &z, bool gate) {
    float4 d = dy.values();
    if (gate) {
        const float4 g = z.values();
        d.x *= g.x * sigma(g.x), d.y *= g.y * sigma(g.y), d.z *= g.z * sigma(g.z), d.w *= g.w * sigma(g.w);
    }
    return d;
}

// What G is before a segment when it is zero behind it: sum over its tokens of e^(A (sum of D up to t)) C_t do_t.
template <typename T, int N, bool kGate>
__global__ void __launch_bounds__(kThreads) k_reverse_ends(Args<T> a) {
    using S = Block<N>;
    __shared__ __align__(16) float4 delta[S::kTok * S::kGroups], dout[S::kTok * S::kGroups], cs[S::kTok * S::P];
    wait_for_previous();
    const Place<T, N> w(a);
    const int64_t end = (int64_t)w.b * a.nseg + w.seg;
    Quad G[4], a2[4];
    if (w.seg == 0) {               // the first one's place holds the final state's gradient, which d_state_in may overwrite
        w.load_states(G, a.d_state_out ? a.d_state_out + w.state(a, w.b) : nullptr);
        w.store_states(G, a.end_state + w.state(a, end));
        return;
    }
    const T *dy = a.dy + w.b * a.dy_b, *dt = a.dt + w.b * a.dt_b, *c = a.c + w.b * a.c_b;
    const T *z = kGate ? a.z + w.b * a.z_b : nullptr;
    const Quad bias = quad(four_of(a.bias, w.cu, w.on_u));
    w.load_decays(a2, a);
    w.load_states(G, nullptr);
    Quad minus = {0, 0};
    Passed passed;
    passed.clear();
    Four<T> ry[S::kUnits], rd[S::kUnits], rz[S::kUnits], rc[S::kRows];
    auto fetch = [&](int t0) {
        w.load(ry, dy, a.dy_l, t0);
        w.load(rd, dt, a.dt_l, t0);
        if (kGate) w.load(rz, z, a.z_l, t0);
        w.load_row(rc, c, a.c_l, t0);
    };
    const int last = min(w.last, (w.len + S::kTok - 1) / S::kTok);
    const int mine = threadIdx.x / S::P, p = w.p;
    if (w.first < last) fetch((last - 1) * S::kTok);
    for (int tile = last - 1; tile >= w.first; --tile) {
#pragma unroll
        for (int k = 0; k < S::kUnits; ++k) {
            delta[w.unit(k)] = unquad(step_of(rd[k].values(), bias, a.softplus, tile * S::kTok + w.token(k) < w.len));
            dout[w.unit(k)] = gated<T>(ry[k], rz[k], kGate);
        }
        w.store_row(cs, rc);
        __syncthreads();
        if (tile > w.first) fetch((tile - 1) * S::kTok);
#pragma unroll 4
        for (int t = S::kTok - 1; t >= 0; --t) {
            const float4 d = delta[t * S::kGroups + mine], g = dout[t * S::kGroups + mine];
            const Quad C = quad(cs[t * S::P + p]);
            passed.add(quad(d));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2 di = both(at(d, i));
                const Quad decays = {decay(di, a2[i].lo), decay(di, a2[i].hi)};
                G[i] = mul4(decays, fma4(both(at(g, i)), C, G[i]));
                passed.product[i] = mul4(decays, passed.product[i]);
            }
        }
        if (tile * S::kTok % kPeriod == 0 || tile == w.first) {
            put_right(G, a2, passed);
            minus = {add2(minus.lo, passed.minus.lo), add2(minus.hi, passed.minus.hi)};
            passed.clear();
        }
        __syncthreads();
    }
    w.store_states(G, a.end_state + w.state(a, end));
    if (w.on && p == 0) *reinterpret_cast<float4 *>(a.end_delta + end * a.D + w.c) = unquad(mul4(both(-1.f), minus));
}

constexpr int kWide = 64;       // channels of a block of the main kernel
constexpr int kRun = 4;         // tokens whose states are in registers

template <int N>
struct Shared {
    static constexpr int P = N / 4, kThreads = kWide / 4 * P;
    float4 delta[kTile][kWide / 4], drive[kTile][kWide / 4], dout[kTile][kWide / 4];    // D, D x, do of 4 channels
    float4 b[2][kTile][P], c[2][kTile][P];  // [1]: neighbours swapped
    union {
        struct {
            // Shares of sums over n, a thread's 4 channels each, one more every P to keep the banks apart.
            float4 o[kRun][kThreads + kWide / 4], gb[kRun][kThreads + kWide / 4], ga[kRun][kThreads + kWide / 4];   // of C h, G B, G a h A
            float bc[kRun][kThreads / 32][2 * N];       // a warp's sums over its channels of dB and dC
        };
        float col[kThreads][8];             // at the end: threads' sums of dskip and dbias
    };
    Quad mid[kTile / kRun][4][kThreads];    // states at the runs' starts; the last run's place then holds the decays' product
};

// Four states of four channels; index j is state j ^ q.
struct States {
    Quad v[4];
};
__device__ __forceinline__ float4 permuted(float4 f, int q) {
    if (q & 2) f = make_float4(f.z, f.w, f.x, f.y);
    if (q & 1) f = make_float4(f.y, f.x, f.w, f.z);
    return f;
}
// The channels' rows lie N floats apart.
template <int N>
__device__ __forceinline__ States load_states(const float *p, int q) {
    States s;
#pragma unroll
    for (int i = 0; i < 4; ++i) s.v[i] = quad(permuted(*reinterpret_cast<const float4 *>(p + i * N), q));
    return s;
}
template <int N>
__device__ __forceinline__ void store_states(float *p, const States &s, int q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(p + i * N) = permuted(unquad(s.v[i]), q);
}
__device__ __forceinline__ Quad decays(f32x2 delta, Quad a2) { return {decay(delta, a2.lo), decay(delta, a2.hi)}; }
// A token's four values in a lane's order: the halves' order is that of the addresses.
__device__ __forceinline__ Quad in_order(const float4 *p, int half) {
    const f32x2 *v = reinterpret_cast<const f32x2 *>(p);
    return {v[half], v[half ^ 1]};
}
// The sum of v's index j over the lanes that share lane % P; a lane is left with that of state q.
template <int P>
__device__ __forceinline__ float sum_channels(Quad v) {
    float4 f = unquad(v);
    f.x += __shfl_xor_sync(~0u, f.z, 16);
    f.y += __shfl_xor_sync(~0u, f.w, 16);
    f.x += __shfl_xor_sync(~0u, f.y, 8);
#pragma unroll
    for (int m = 4; m >= P; m >>= 1) f.x += __shfl_xor_sync(~0u, f.x, m);
    return f.x;
}
// Channels 4 u .. 4 u + 3 of a token's shares.
template <int P>
__device__ __forceinline__ float4 sum_shares(const float4 *p, int u) {
    Quad v = quad(p[u * (P + 1)]);
#pragma unroll
    for (int i = 1; i < P; ++i) {
        const Quad r = quad(p[u * (P + 1) + i]);
        v = {add2(v.lo, r.lo), add2(v.hi, r.hi)};
    }
    return unquad(v);
}

template <typename T, int N, bool kGate>
__global__ void __launch_bounds__(4 * N) k_backward(Args<T> a) {
    constexpr int P = N / 4, kThreads = Shared<N>::kThreads, kUnits = kTile * (kWide / 4) / kThreads;
    constexpr int kRunUnits = (kRun * (kWide / 4) + kThreads - 1) / kThreads;       // groups of 4 channels of a run, a thread
    static_assert(kThreads == 4 * N);
    extern __shared__ __align__(16) char smem[];
    Shared<N> &s = *reinterpret_cast<Shared<N> *>(smem);
    wait_for_previous();
    const int groups = (a.D + kWide - 1) / kWide, seg = blockIdx.x % a.nseg, row = blockIdx.x / a.nseg, bi = row / groups;
    const int group = row % groups, c0 = group * kWide;
    const int first = min(seg * a.per, a.ntiles), past = min(first + a.per, a.ntiles);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, p = tid % P, mine = tid / P, c = c0 + 4 * mine;
    const int q = lane >> 3, half = q >> 1;                         // the lane's order of states
    const int len = length_of(a, bi);
    const bool on = c < a.D;
    const int u = tid % (kWide / 4), cu = c0 + 4 * u;               // staging: a thread's group of channels
    const bool on_u = cu < a.D;
    const T *x = a.x + bi * a.x_b + cu, *dt = a.dt + bi * a.dt_b + cu, *dy = a.dy + bi * a.dy_b + cu;
    const T *z = kGate ? a.z + bi * a.z_b + cu : nullptr, *b = a.b + bi * a.b_b, *cc = a.c + bi * a.c_b;
    T *dx = a.dx + bi * a.dx_b + cu, *ddt = a.ddt + bi * a.ddt_b + cu, *dz = kGate ? a.dz + bi * a.dz_b + cu : nullptr;
    const float4 bias = four_of(a.bias, cu, on_u), skip = four_of(a.skip, cu, on_u);
    auto state = [&](int64_t r) { return (r * a.D + c) * N + 4 * p; };      // the thread's place in row r of [..][D][N]
    States a2 = {}, G = {}, dA = {};
    if (on) {
        a2 = load_states<N>(a.A + (int64_t)c * N + 4 * p, q);
#pragma unroll
        for (int j = 0; j < 4; ++j) a2.v[j] = mul4(both(kLog2e), a2.v[j]);
        if (a.nseg > 1) {
            const int64_t end = (int64_t)bi * a.nseg;
            auto load = [&](int k, Quad (&E)[4]) {
                const States e = load_states<N>(a.end_state + state(end + k), q);
#pragma unroll
                for (int j = 0; j < 4; ++j) E[j] = e.v[j];
            };
            through_segments(
                G.v, a2.v, a.nseg - 1 - seg, [&](Quad (&E)[4]) { load(0, E); },
                [&](int k, float4 &S, Quad (&E)[4]) {
                    load(a.nseg - 1 - k, E), S = *reinterpret_cast<const float4 *>(a.end_delta + (end + a.nseg - 1 - k) * a.D + c);
                });
        } else if (a.d_state_out) {
            G = load_states<N>(a.d_state_out + state(bi), q);
        }
    }
    float dskip[4] = {}, dbias[4] = {};
    auto bc_row = [&](int t) { return a.part_bc + (((int64_t)bi * a.L + t) * groups + group) * 2 * N; };
    const int last = min(past, (len + kTile - 1) / kTile);
    for (int tile = past - 1; tile >= max(first, last); --tile) {       // padding
        for (int i = tid; i < kTile * (kWide / 4); i += kThreads) {
            const int to = tile * kTile + i / (kWide / 4);
            if (!on_u || to >= a.L) continue;
            const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
            Four<T>::store(dx + (int64_t)to * a.dx_l, none);
            Four<T>::store(ddt + (int64_t)to * a.ddt_l, none);
            if (kGate) Four<T>::store(dz + (int64_t)to * a.dz_l, none);
        }
        for (int i = tid; i < kTile * 2 * N; i += kThreads) {
            const int to = tile * kTile + i / (2 * N);
            if (to < a.L) bc_row(to)[i % (2 * N)] = 0.f;
        }
    }
    const float4 *brow = &s.b[q & 1][0][p], *crow = &s.c[q & 1][0][p];
    const int share = tid + mine;
    for (int tile = last - 1; tile >= first; --tile) {
        const int t0 = tile * kTile;
        const float *saved = a.saved + state((int64_t)bi * a.ntiles + tile);
        States h = {};
        if (on) h = load_states<N>(saved, q);
        // Staging, as many of a thread's groups at a time as registers hold.
        constexpr int kHalf = kUnits * sizeof(T) <= 8 ? kUnits : kUnits / 2;
#pragma unroll
        for (int k0 = 0; k0 < kUnits; k0 += kHalf) {
            Four<T> rx[kHalf], rd[kHalf], ry[kHalf], rz[kHalf];
#pragma unroll
            for (int k = 0; k < kHalf; ++k) {
                const int to = t0 + (tid + (k0 + k) * kThreads) / (kWide / 4);
                rx[k].clear(), rd[k].clear(), ry[k].clear(), rz[k].clear();
                if (on_u && to < len) {
                    rx[k].load(x + (int64_t)to * a.x_l);
                    rd[k].load(dt + (int64_t)to * a.dt_l);
                    ry[k].load(dy + (int64_t)to * a.dy_l);
                    if (kGate) rz[k].load(z + (int64_t)to * a.z_l);
                }
            }
#pragma unroll
            for (int k = 0; k < kHalf; ++k) {
                const int t = (tid + (k0 + k) * kThreads) / (kWide / 4);
                const Quad d = step_of(rd[k].values(), quad(bias), a.softplus, t0 + t < len);
                s.delta[t][u] = unquad(d);
                s.drive[t][u] = unquad(mul4(d, quad(rx[k].values())));
                s.dout[t][u] = gated<T>(ry[k], rz[k], kGate);
            }
        }
        for (int i = tid; i < kTile * P; i += kThreads) {
            const int t = i / P, n = i % P;
            Four<T> rb, rc;
            rb.clear(), rc.clear();
            if (t0 + t < len) {
                rb.load(b + (int64_t)(t0 + t) * a.b_l + 4 * n);
                rc.load(cc + (int64_t)(t0 + t) * a.c_l + 4 * n);
            }
            s.b[0][t][n] = rb.values();
            s.b[1][t][n] = permuted(rb.values(), 1);
            s.c[0][t][n] = rc.values();
            s.c[1][t][n] = permuted(rc.values(), 1);
        }
        __syncthreads();
        if (tile > first && on_u) {         // the next tile into L2
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const int64_t to = t0 - kTile + (tid + k * kThreads) / (kWide / 4);
                asm volatile("prefetch.global.L2 [%0];" ::"l"(x + to * a.x_l));
                asm volatile("prefetch.global.L2 [%0];" ::"l"(dt + to * a.dt_l));
                asm volatile("prefetch.global.L2 [%0];" ::"l"(dy + to * a.dy_l));
                if (kGate) asm volatile("prefetch.global.L2 [%0];" ::"l"(z + to * a.z_l));
            }
        }
        if (tile > first && on) {
#pragma unroll
            for (int i = 0; i < 4; ++i) asm volatile("prefetch.global.L2 [%0];" ::"l"(saved - (int64_t)a.D * N + i * N));
        }
        // The states at the runs' starts.
#pragma unroll 1
        for (int run = 0; run < kTile / kRun; ++run) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s.mid[run][j][tid] = h.v[j];
            if (run == kTile / kRun - 1) break;
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                const int t = run * kRun + i;
                const float4 d = s.delta[t][mine], v = s.drive[t][mine];
                const Quad B = in_order(brow + t * P, half);
                const Quad w[4] = {mul4(both(v.x), B), mul4(both(v.y), B), mul4(both(v.z), B), mul4(both(v.w), B)};
                advance(h.v, a2.v, d, w);
            }
        }
#pragma unroll 1
        for (int run = kTile / kRun - 1; run >= 0; --run) {
            States h0;
#pragma unroll
            for (int j = 0; j < 4; ++j) h0.v[j] = s.mid[run][j][tid];
            // What the run's field gradients need again, loaded (out of L2) while the run is walked.
            Four<T> rx[kRunUnits], rd[kRunUnits], ry[kRunUnits], rz[kRunUnits];
#pragma unroll
            for (int k = 0; k < kRunUnits; ++k) {
                const int i = (tid + k * kThreads) / (kWide / 4), to = t0 + run * kRun + i;
                rx[k].clear(), rd[k].clear(), ry[k].clear(), rz[k].clear();
                if (i < kRun && on_u && to < len) {
                    rx[k].load(x + (int64_t)to * a.x_l);
                    rd[k].load(dt + (int64_t)to * a.dt_l);
                    ry[k].load(dy + (int64_t)to * a.dy_l);
                    if (kGate) rz[k].load(z + (int64_t)to * a.z_l);
                }
            }
            // The run's states, and its decays' product.
            Passed passed;
            passed.clear();
            States hs[kRun];
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                const int t = run * kRun + i;
                const float4 d = s.delta[t][mine], v = s.drive[t][mine];
                const Quad B = in_order(brow + t * P, half);
                const Quad w[4] = {mul4(both(v.x), B), mul4(both(v.y), B), mul4(both(v.z), B), mul4(both(v.w), B)};
                hs[i] = i ? hs[i ? i - 1 : 0] : h0;
                advance(hs[i].v, a2.v, d, w, passed);
                if (kGate) {
                    const Quad C = in_order(crow + t * P, half);
                    s.o[i][share] = make_float4(dot4(C, hs[i].v[0]), dot4(C, hs[i].v[1]), dot4(C, hs[i].v[2]), dot4(C, hs[i].v[3]));
                }
            }
            Quad(&product)[4][kThreads] = s.mid[kTile / kRun - 1];          // (the last run has taken its states from there)
            if (run < kTile / kRun - 1) {
#pragma unroll
                for (int j = 0; j < 4; ++j) passed.product[j] = mul4(product[j][tid], passed.product[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) product[j][tid] = passed.product[j];
            // The gradient, token by token backwards.
#pragma unroll
            for (int i = kRun - 1; i >= 0; --i) {
                const int t = run * kRun + i;
                const float4 d = s.delta[t][mine], v = s.drive[t][mine], w = s.dout[t][mine];
                const Quad B = in_order(brow + t * P, half), C = in_order(crow + t * P, half);
                Quad db, dc;
                float gb[4], ga[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x2 delta = both(at(d, j)), drive = both(at(v, j)), dout = both(at(w, j));
                    Quad &g = G.v[j];
                    g = fma4(dout, C, g);
                    db = j ? fma4(drive, g, db) : mul4(drive, g);
                    dc = j ? fma4(dout, hs[i].v[j], dc) : mul4(dout, hs[i].v[j]);
                    gb[j] = dot4(g, B);
                    g = mul4(decays(delta, a2.v[j]), g);
                    const Quad k = mul4(g, i ? hs[i ? i - 1 : 0].v[j] : h0.v[j]);       // G a h_{t-1}
                    ga[j] = dot4(k, a2.v[j]);
                    dA.v[j] = fma4(delta, k, dA.v[j]);
                }
                s.gb[i][share] = make_float4(gb[0], gb[1], gb[2], gb[3]);
                s.ga[i][share] = make_float4(ga[0], ga[1], ga[2], ga[3]);
                const float sb = sum_channels<P>(db), sc = sum_channels<P>(dc);
                if (P == 8 || (lane & 7) < P) {
                    s.bc[i][warp][4 * p + q] = sb;
                    s.bc[i][warp][N + 4 * p + q] = sc;
                }
            }
            __syncthreads();
            // The fields' gradients, 4 channels a thread.
#pragma unroll
            for (int k = 0; k < kRunUnits; ++k) {
                const int i = (tid + k * kThreads) / (kWide / 4), t = run * kRun + i, to = t0 + t;
                if (i >= kRun || !on_u || to >= a.L) continue;
                const float4 xv = rx[k].values(), dv = rd[k].values(), yv = ry[k].values(), zv = rz[k].values();
                const float4 delta = s.delta[t][u], v = s.dout[t][u];
                const float4 gb = sum_shares<P>(s.gb[i], u), ga = sum_shares<P>(s.ga[i], u);
                const float4 o = kGate ? sum_shares<P>(s.o[i], u) : make_float4(0.f, 0.f, 0.f, 0.f);
                float fx[4], fd[4], fz[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    fx[e] = fmaf(at(delta, e), at(gb, e), at(skip, e) * at(v, e));
                    fd[e] = fmaf(kLn2, at(ga, e), at(xv, e) * at(gb, e));
                    if (a.softplus) fd[e] *= sigma(at(dv, e) + at(bias, e));
                    if (kGate) {
                        const float g = at(zv, e), sg = sigma(g);
                        fz[e] = at(yv, e) * fmaf(at(skip, e), at(xv, e), at(o, e)) * sg * fmaf(g, 1.f - sg, 1.f);
                    }
                    if (to >= len) fx[e] = fd[e] = fz[e] = 0.f;
                    dskip[e] = fmaf(at(v, e), at(xv, e), dskip[e]);
                    dbias[e] += fd[e];
                }
                Four<T>::store(dx + (int64_t)to * a.dx_l, make_float4(fx[0], fx[1], fx[2], fx[3]));
                Four<T>::store(ddt + (int64_t)to * a.ddt_l, make_float4(fd[0], fd[1], fd[2], fd[3]));
                if (kGate) Four<T>::store(dz + (int64_t)to * a.dz_l, make_float4(fz[0], fz[1], fz[2], fz[3]));
            }
#pragma unroll
            for (int k = tid; k < kRun * 2 * N; k += kThreads) {
                const int i = k / (2 * N), n = k % (2 * N), to = t0 + run * kRun + i;
                float v = 0.f;
#pragma unroll
                for (int m = 0; m < kThreads / 32; ++m) v += s.bc[i][m][n];
                if (to < a.L) bc_row(to)[n] = to < len ? v : 0.f;
            }
            __syncthreads();
        }
        // After every tile: there is no room for the product over a longer time (in a place of its own it costs N = 8 a block
        // of the SM's 7).
        Passed passed;
        passed.clear();
#pragma unroll
        for (int j = 0; j < 4; ++j) passed.product[j] = s.mid[kTile / kRun - 1][j][tid];
#pragma unroll
        for (int t = 0; t < kTile; ++t) passed.add(quad(s.delta[t][mine]));
        put_right(G.v, a2.v, passed);
        __syncthreads();            // (the next tile's D)
    }
    const int64_t part = (int64_t)bi * a.nseg + seg;
    if (on) {
        store_states<N>(a.part_A + state(part), dA, q);
        if (a.d_state_in && seg == 0) store_states<N>(a.d_state_in + state(bi), G, q);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s.col[tid][i] = dskip[i], s.col[tid][4 + i] = dbias[i];
    __syncthreads();
    for (int i = tid; i < 2 * kWide; i += kThreads) {                   // dskip of the channels, then dbias
        const int k = i / kWide, d = i % kWide;
        float v = 0.f;
        for (int m = d / 4; m < kThreads; m += kWide / 4) v += s.col[m][4 * k + d % 4];
        if (c0 + d < a.D) a.part_d[(part * 2 + k) * a.D + c0 + d] = v;
    }
}

// The blocks' shares: dB and dC over groups of channels (blocks below `fields`), then dA, dskip and
// dbias over batch rows and segments.
constexpr int kSumThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kSumThreads) k_sums(Args<T> a, int64_t tokens, int N, int64_t fields, int rows, float *dA, float *dskip,
                                                      float *dbias) {
    __shared__ float share[8][33];
    wait_for_previous();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if ((int64_t)blockIdx.x < fields) {
        const int width = 2 * N, groups = (a.D + kWide - 1) / kWide;
        const int64_t i = (int64_t)blockIdx.x * kSumThreads + tid, t = i / width;
        const int n = (int)(i - t * width);
        if (t >= tokens) return;
        const float *q = a.part_bc + t * groups * width + n;
        float v = 0.f;
#pragma unroll 8
        for (int g = 0; g < groups; ++g) v += q[(int64_t)g * width];
        const int64_t b = t / a.L, l = t - b * a.L;
        st_elem(n < N ? a.db + b * a.db_b + l * a.db_l + n : a.dc + b * a.dc_b + l * a.dc_l + n - N, v);
        return;
    }
    // 32 values a block, their parts in 8 runs.
    const int64_t DN = (int64_t)a.D * N, i = ((int64_t)blockIdx.x - fields) * 32 + lane, end = DN + 2 * (int64_t)a.D;
    const float *q = i < DN ? a.part_A + i : a.part_d + (i - DN);
    const int64_t pitch = i < DN ? DN : 2 * (int64_t)a.D;
    const int per = (rows + 7) / 8, r0 = min(warp * per, rows), r1 = min(r0 + per, rows);
    float v = 0.f;
    if (i < end)
#pragma unroll 8
        for (int r = r0; r < r1; ++r) v += q[r * pitch];
    share[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || i >= end) return;
    v = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) v += share[r][lane];
    float *to = i < DN ? dA + i : i < DN + a.D ? (dskip ? dskip + (i - DN) : nullptr) : (dbias ? dbias + (i - DN - a.D) : nullptr);
    if (to) *to = v;
}

struct Plan {
    int ntiles, nseg, per;
    size_t end_delta, part_bc, part_A, part_d, bytes;
};
Plan plan(int64_t B, int64_t L, int D, int N) {
    Plan p;
    const int groups = (D + kWide - 1) / kWide;
    p.ntiles = (int)((L + kTile - 1) / kTile);
    const int want = segments(B * groups, p.ntiles, 64 / N, 1.2);
    p.per = (p.ntiles + want - 1) / want;
    p.nseg = (p.ntiles + p.per - 1) / p.per;
    size_t at = 0;
    auto take = [&](size_t floats) {
        const size_t here = at;
        at += (floats * sizeof(float) + 255) / 256 * 256;
        return here;
    };
    const size_t rows = (size_t)B * p.nseg;
    take(p.nseg > 1 ? rows * D * N : 0);        // end states, from the workspace's first byte on
    p.end_delta = take(p.nseg > 1 ? rows * D : 0);
    p.part_bc = take((size_t)B * L * groups * 2 * N);
    p.part_A = take(rows * D * N);
    p.part_d = take(rows * 2 * D);
    p.bytes = at;
    return p;
}

template <typename T, int N, bool kGate>
cudaError_t launch(Args<T> &a, int64_t B, const rlm_ssm_grads &d, cudaStream_t st) {
    const int64_t blocks = B * ((a.D + kWide - 1) / kWide) * a.nseg;
    cudaError_t e = cudaSuccess;
    if (a.nseg > 1)
        e = launch_dependent(k_reverse_ends<T, N, kGate>, dim3((unsigned)Block<N>::blocks_of(B, a.D, a.nseg)), kThreads, 0, st, 1, a);
    if (e != cudaSuccess) return e;
    constexpr int kBytes = (int)sizeof(Shared<N>);
    e = cudaFuncSetAttribute(k_backward<T, N, kGate>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    e = launch_dependent(k_backward<T, N, kGate>, dim3((unsigned)blocks), 4 * N, kBytes, st, 1, a);
    if (e != cudaSuccess) return e;
    const int64_t tokens = B * a.L, fields = (tokens * 2 * N + kSumThreads - 1) / kSumThreads;
    const int64_t params = ((int64_t)a.D * (N + 2) + 31) / 32;
    return launch_dependent(k_sums<T>, dim3((unsigned)(fields + params)), kSumThreads, 0, st, 1, a, tokens, N, fields, (int)(B * a.nseg), d.A,
                            d.skip, d.dt_bias);
}

template <typename T, bool kGate>
cudaError_t launch_n(Args<T> &a, int64_t B, int N, const rlm_ssm_grads &d, cudaStream_t st) {
    return N == 8 ? launch<T, 8, kGate>(a, B, d, st) : N == 16 ? launch<T, 16, kGate>(a, B, d, st) : launch<T, 32, kGate>(a, B, d, st);
}

template <typename T>
cudaError_t backward(const SsmBackward &g, void *ws, cudaStream_t st) {
    const rlm_ssm_params &p = *g.params;
    const Plan q = plan(g.x->B, g.x->L, p.D, p.N);
    Args<T> a = {};
    auto in = [](const rlm_strided &f, const T *&v, int64_t &sb, int64_t &sl) { v = static_cast<const T *>(f.ptr), sb = f.stride_b, sl = f.stride_l; };
    auto out = [](const rlm_strided &f, T *&v, int64_t &sb, int64_t &sl) { v = static_cast<T *>(f.ptr), sb = f.stride_b, sl = f.stride_l; };
    in(*g.x, a.x, a.x_b, a.x_l);
    in(*g.dt, a.dt, a.dt_b, a.dt_l);
    in(*g.b, a.b, a.b_b, a.b_l);
    in(*g.c, a.c, a.c_b, a.c_l);
    in(*g.dy, a.dy, a.dy_b, a.dy_l);
    out(*g.dx, a.dx, a.dx_b, a.dx_l);
    out(*g.ddt, a.ddt, a.ddt_b, a.ddt_l);
    out(*g.db, a.db, a.db_b, a.db_l);
    out(*g.dc, a.dc, a.dc_b, a.dc_l);
    if (g.z) {
        in(*g.z, a.z, a.z_b, a.z_l);
        out(*g.dz, a.dz, a.dz_b, a.dz_l);
    }
    a.A = p.A, a.skip = p.skip, a.bias = p.dt_bias, a.softplus = p.softplus;
    a.saved = const_cast<float *>(g.saved), a.lengths = g.lengths, a.d_state_out = g.d_state_out, a.d_state_in = g.d_state_in;
    a.L = (int)g.x->L, a.D = p.D, a.ntiles = q.ntiles, a.nseg = q.nseg, a.per = q.per;
    auto at = [&](size_t o) { return reinterpret_cast<float *>(static_cast<char *>(ws) + o); };
    a.end_state = at(0), a.end_delta = at(q.end_delta), a.part_bc = at(q.part_bc), a.part_A = at(q.part_A), a.part_d = at(q.part_d);
    return g.z ? launch_n<T, true>(a, g.x->B, p.N, *g.grads, st) : launch_n<T, false>(a, g.x->B, p.N, *g.grads, st);
}

}  // namespace
}  // namespace ssm

size_t ssm_backward_ws_bytes(int64_t B, int64_t L, int D, int N) { return ssm::plan(B, L, D, N).bytes; }

cudaError_t ssm_backward(const SsmBackward &g, void *ws, cudaStream_t st) {
    return g.x->dtype == RLM_BF16 ? ssm::backward<__nv_bfloat16>(g, ws, st) : ssm::backward<float>(g, ws, st);
}

}  // namespace rlm
