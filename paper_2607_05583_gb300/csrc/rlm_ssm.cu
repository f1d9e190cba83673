// rlm_ssm.cu -- the selective state space scan over a sequence, and one token of it (mathematics and
// layout in rlm_ssm.cuh, gradients in rlm_ssm_backward.cu).
//
// A token, channel and state cost one ex2 and four multiply-adds; an SM has units for 32 of the former and 128
// of the latter a clock (measured: 62.6 and 243 a nanosecond), so N states bound a token and channel by N / 32 clocks
// of an SM, against 8 bytes of memory (bf16): above N = 8 or so the kernel is bound by arithmetic, in
// practice by the issue of its instructions (31 a warp's 32 x 4 states and token: 10 of them for staging and output, 3 for
// keeping the decays' product and putting the states right by it).  B = 4, L = 4096, D = 1024, N = 16: 103 us in bf16, 115 in
// fp32, and 66 for the segments' ends.  The registers are bounded for 6 blocks on an SM, which k_forward needs no spills of
// more than a few bytes for; z is loaded before a tile's tokens and used behind them, where x and dt are a tile ahead (a
// tile ahead too, z takes registers that fp32 has not got: 128 us; 5 blocks an SM without a bound: 130).
//
// Segments.  Where rows and channels give too few warps the sequence is cut into nseg runs of tiles.
// A run maps its first state to its last by h -> e^(A S) h + H, S the sum of its D and H its end state
// from zero: k_ends forms (S, H) of all runs but the last, and every block of the main kernel composes
// those before its own.  That is two launches and, without C and y, about 0.75 more of the arithmetic;
// nobody waits for anybody within a kernel.
#include <algorithm>

#include "rlm_ssm.cuh"

namespace rlm {
namespace ssm {

int segments(int64_t blocks, int ntiles, int resident, double ends) {
    const int64_t slots = (int64_t)sm_count() * resident;
    int best = 1;
    double least = 0;
    for (int n = 1; n <= 128 && n <= ntiles; ++n) {
        const int64_t rounds = (blocks * n + slots - 1) / slots;
        const double cost = (double)rounds * ((ntiles + n - 1) / n + 1) * (n > 1 ? ends : 1.0);
        if (n == 1 || cost < least) best = n, least = cost;
    }
    return best;
}

namespace {

// End state and sum of D of a segment, from a zero state.
template <typename T, int N>
__global__ void __launch_bounds__(kThreads) k_ends(Args<T> a) {
    using S = Block<N>;
    __shared__ __align__(16) float4 delta[S::kTok * S::kGroups], drive[S::kTok * S::kGroups], bs[S::kTok * S::P];
    wait_for_previous();
    const Place<T, N> w(a);
    const int64_t end = (int64_t)w.b * a.nseg + w.seg;
    Quad h[4], a2[4];
    if (w.seg == a.nseg - 1) {      // the last one's place holds the initial state, which state_out may overwrite
        w.load_states(h, a.state_in ? a.state_in + w.state(a, w.b) : nullptr);
        w.store_states(h, a.end_state + w.state(a, end));
        return;
    }
    const T *x = a.x + w.b * a.x_b, *dt = a.dt + w.b * a.dt_b, *b = a.b + w.b * a.b_b;
    const Quad bias = quad(four_of(a.bias, w.cu, w.on_u));
    w.load_decays(a2, a);
    w.load_states(h, nullptr);
    Quad minus = {0, 0};
    Passed passed;
    passed.clear();
    Four<T> rx[S::kUnits], rd[S::kUnits], rb[S::kRows];
    auto fetch = [&](int t0) {
        w.load(rx, x, a.x_l, t0);
        w.load(rd, dt, a.dt_l, t0);
        w.load_row(rb, b, a.b_l, t0);
    };
    const int last = min(w.last, (w.len + S::kTok - 1) / S::kTok);
    const int mine = threadIdx.x / S::P, p = w.p;
    if (w.first < last) fetch(w.first * S::kTok);
    for (int tile = w.first; tile < last; ++tile) {
#pragma unroll
        for (int k = 0; k < S::kUnits; ++k) {
            const Quad d = step_of(rd[k].values(), bias, a.softplus, tile * S::kTok + w.token(k) < w.len);
            delta[w.unit(k)] = unquad(d);
            drive[w.unit(k)] = unquad(mul4(d, quad(rx[k].values())));
        }
        w.store_row(bs, rb);
        __syncthreads();
        if (tile + 1 < last) fetch((tile + 1) * S::kTok);
#pragma unroll 8
        for (int t = 0; t < S::kTok; ++t) {
            const float4 d = delta[t * S::kGroups + mine], u = drive[t * S::kGroups + mine];
            const Quad B = quad(bs[t * S::P + p]), v[4] = {mul4(both(u.x), B), mul4(both(u.y), B), mul4(both(u.z), B), mul4(both(u.w), B)};
            advance(h, a2, d, v, passed);
        }
        if ((tile + 1) * S::kTok % kPeriod == 0 || tile + 1 == last) {
            put_right(h, a2, passed);
            minus = {add2(minus.lo, passed.minus.lo), add2(minus.hi, passed.minus.hi)};
            passed.clear();
        }
        __syncthreads();
    }
    w.store_states(h, a.end_state + w.state(a, end));
    if (w.on && p == 0) *reinterpret_cast<float4 *>(a.end_delta + end * a.D + w.c) = unquad(mul4(both(-1.f), minus));
}

template <typename T, int N, bool kGate>
__global__ void __launch_bounds__(kThreads, 6) k_forward(Args<T> a) {
    using S = Block<N>;
    __shared__ __align__(16) float4 delta[S::kTok * S::kGroups], drive[S::kTok * S::kGroups], bs[S::kTok * S::P], cs[S::kTok * S::P];
    __shared__ __align__(16) float4 share[S::kTok][kThreads + S::kGroups];     // of o: P a group, one more to keep the banks apart
    wait_for_previous();
    const Place<T, N> w(a);
    const T *x = a.x + w.b * a.x_b, *dt = a.dt + w.b * a.dt_b, *b = a.b + w.b * a.b_b, *c = a.c + w.b * a.c_b;
    const T *z = kGate ? a.z + w.b * a.z_b : nullptr;
    T *y = a.y + w.b * a.y_b + w.cu;
    const Quad bias = quad(four_of(a.bias, w.cu, w.on_u)), skip = quad(four_of(a.skip, w.cu, w.on_u));
    Quad h[4], a2[4];
    w.load_decays(a2, a);
    if (a.nseg > 1) {
        const int64_t end = (int64_t)w.b * a.nseg;
        auto load = [&](int s, Quad (&H)[4]) { w.load_states(H, a.end_state + w.state(a, end + s)); };
        through_segments(
            h, a2, w.seg, [&](Quad (&H)[4]) { load(a.nseg - 1, H); },
            [&](int s, float4 &S, Quad (&H)[4]) { load(s, H), S = four_of(a.end_delta + (end + s) * a.D, w.c, w.on); });
    } else {
        w.load_states(h, a.state_in ? a.state_in + w.state(a, w.b) : nullptr);
    }
    Four<T> rx[S::kUnits], rz[S::kUnits], nx[S::kUnits], nd[S::kUnits], nb[S::kRows], nc[S::kRows];
    auto fetch = [&](int t0) {
        w.load(nx, x, a.x_l, t0);
        w.load(nd, dt, a.dt_l, t0);
        w.load_row(nb, b, a.b_l, t0);
        w.load_row(nc, c, a.c_l, t0);
    };
    const int last = min(w.last, (w.len + S::kTok - 1) / S::kTok);
    const int mine = threadIdx.x / S::P, p = w.p;
    Passed passed;
    passed.clear();
    if (w.first < last) fetch(w.first * S::kTok);
    for (int tile = w.first; tile < last; ++tile) {
        const int t0 = tile * S::kTok;
#pragma unroll
        for (int k = 0; k < S::kUnits; ++k) {
            const Quad d = step_of(nd[k].values(), bias, a.softplus, t0 + w.token(k) < w.len);
            delta[w.unit(k)] = unquad(d);
            drive[w.unit(k)] = unquad(mul4(d, quad(nx[k].values())));
            rx[k] = nx[k];
        }
        w.store_row(bs, nb);
        w.store_row(cs, nc);
        __syncthreads();
        if (kGate) w.load(rz, z, a.z_l, t0);         // (used behind the tokens)
        if (tile + 1 < last) fetch(t0 + S::kTok);
        if (t0 % kPeriod == 0) {
            put_right(h, a2, passed);
            passed.clear();
        }
        if (a.saved && t0 % kTile == 0) w.store_states(h, a.saved + w.state(a, (int64_t)w.b * a.ntiles + t0 / kTile));
#pragma unroll 4
        for (int t = 0; t < S::kTok; ++t) {
            const float4 d = delta[t * S::kGroups + mine], u = drive[t * S::kGroups + mine];
            const Quad B = quad(bs[t * S::P + p]), C = quad(cs[t * S::P + p]);
            const Quad v[4] = {mul4(both(u.x), B), mul4(both(u.y), B), mul4(both(u.z), B), mul4(both(u.w), B)};
            advance(h, a2, d, v, passed);
            share[t][threadIdx.x + mine] = make_float4(dot4(C, h[0]), dot4(C, h[1]), dot4(C, h[2]), dot4(C, h[3]));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < S::kUnits; ++k) {
            const int t = w.token(k);
            if (!w.on_u || t0 + t >= a.L) continue;
            const float4 *q = &share[t][threadIdx.x % S::kGroups * (S::P + 1)];
            Quad o = quad(q[0]);
#pragma unroll
            for (int i = 1; i < S::P; ++i) {
                const Quad v = quad(q[i]);
                o = {add2(o.lo, v.lo), add2(o.hi, v.hi)};
            }
            o = fma4(skip, quad(rx[k].values()), o);
            if (kGate) {
                const float4 g = rz[k].values();
                o = mul4(o, mul4(quad(g), quad(make_float4(sigma(g.x), sigma(g.y), sigma(g.z), sigma(g.w)))));
            }
            if (t0 + t >= w.len) o = {0, 0};
            Four<T>::store(y + (int64_t)(t0 + t) * a.y_l, unquad(o));
        }
    }
    for (int tile = max(w.first, last); tile < w.last; ++tile)         // padding
#pragma unroll
        for (int k = 0; k < S::kUnits; ++k) {
            const int to = tile * S::kTok + w.token(k);
            if (w.on_u && to < a.L) Four<T>::store(y + (int64_t)to * a.y_l, make_float4(0.f, 0.f, 0.f, 0.f));
        }
    put_right(h, a2, passed);
    if (a.state_out && w.seg == a.nseg - 1) w.store_states(h, a.state_out + w.state(a, w.b));
}

// One token, P lanes a channel.
constexpr int kStepThreads = 128;
template <typename T, int N>
__global__ void __launch_bounds__(kStepThreads) k_step(Args<T> a, int64_t rows, float *state) {
    constexpr int P = N / 4;
    wait_for_previous();
    const int64_t i = (int64_t)blockIdx.x * kStepThreads + threadIdx.x, r = i / P;
    const int p = (int)(i % P);
    const bool on = r < rows;
    float o = 0.f, xv = 0.f;
    int64_t b = 0;
    int c = 0;
    if (on) {
        b = r / a.D;
        c = (int)(r - b * a.D);
        float4 *s = reinterpret_cast<float4 *>(state + r * N + 4 * p);
        const Quad h = quad(*s), a2 = mul4(both(kLog2e), quad(*reinterpret_cast<const float4 *>(a.A + (int64_t)c * N + 4 * p)));
        Four<T> B, C;
        B.load(a.b + b * a.b_b + 4 * p);
        C.load(a.c + b * a.c_b + 4 * p);
        xv = (float)a.x[b * a.x_b + c];
        const float v = (float)a.dt[b * a.dt_b + c] + (a.bias ? a.bias[c] : 0.f), d = a.softplus ? unpack(softplus(both(v))).x : v;
        const Quad u = mul4(both(d * xv), quad(B.values()));
        const Quad next = {fma2(decay_alone(both(d), a2.lo), h.lo, u.lo), fma2(decay_alone(both(d), a2.hi), h.hi, u.hi)};
        *s = unquad(next);
        o = dot4(quad(C.values()), next);
    }
#pragma unroll
    for (int m = 1; m < P; m <<= 1) o += __shfl_xor_sync(~0u, o, m);
    if (!on || p != 0) return;
    if (a.skip) o = fmaf(a.skip[c], xv, o);
    if (a.z) {
        const float g = (float)a.z[b * a.z_b + c];
        o *= g * sigma(g);
    }
    st_elem(a.y + b * a.y_b + c, o);
}

template <typename T, int N>
cudaError_t forward(Args<T> &a, int64_t B, cudaStream_t st) {
    const dim3 grid((unsigned)Block<N>::blocks_of(B, a.D, a.nseg));
    if (a.nseg > 1) {
        const cudaError_t e = launch_dependent(k_ends<T, N>, grid, kThreads, 0, st, 1, a);
        if (e != cudaSuccess) return e;
    }
    return launch_dependent(a.z ? k_forward<T, N, true> : k_forward<T, N, false>, grid, kThreads, 0, st, 1, a);
}

template <typename T>
Args<T> arguments(const rlm_strided &x, const rlm_strided &dt, const rlm_strided &b, const rlm_strided &c, const rlm_strided *z,
                  const rlm_strided &y, const rlm_ssm_params &p) {
    Args<T> a = {};
    auto field = [](const rlm_strided &f, const T *&q, int64_t &sb, int64_t &sl) { q = static_cast<const T *>(f.ptr), sb = f.stride_b, sl = f.stride_l; };
    field(x, a.x, a.x_b, a.x_l);
    field(dt, a.dt, a.dt_b, a.dt_l);
    field(b, a.b, a.b_b, a.b_l);
    field(c, a.c, a.c_b, a.c_l);
    if (z) field(*z, a.z, a.z_b, a.z_l);
    a.y = static_cast<T *>(y.ptr), a.y_b = y.stride_b, a.y_l = y.stride_l;
    a.A = p.A, a.skip = p.skip, a.bias = p.dt_bias, a.softplus = p.softplus;
    a.L = (int)x.L, a.D = p.D;
    return a;
}

template <typename T>
cudaError_t run_forward(Args<T> a, int64_t B, int N, cudaStream_t st) {
    return N == 8 ? forward<T, 8>(a, B, st) : N == 16 ? forward<T, 16>(a, B, st) : forward<T, 32>(a, B, st);
}
template <typename T>
cudaError_t run_step(Args<T> a, int64_t B, int N, float *state, cudaStream_t st) {
    const int64_t rows = B * a.D;
    const dim3 grid((unsigned)((rows * (N / 4) + kStepThreads - 1) / kStepThreads));
    return launch_dependent(N == 8 ? k_step<T, 8> : N == 16 ? k_step<T, 16> : k_step<T, 32>, grid, kStepThreads, 0, st, 1, a, rows, state);
}

struct Plan {
    int ntiles, nseg, per;
    size_t end_delta, bytes;
};
Plan plan(int64_t B, int64_t L, int D, int N) {
    Plan p;
    p.ntiles = (int)((L + kTile - 1) / kTile);
    const int width = 1024 / N;     // channels of a block of two warps
    const int want = segments(B * ((D + width - 1) / width), p.ntiles, 6, 1.6);
    p.per = (p.ntiles + want - 1) / want;
    p.nseg = (p.ntiles + p.per - 1) / p.per;
    const size_t rows = p.nseg > 1 ? (size_t)B * p.nseg * D : 0;
    p.end_delta = rows * N * sizeof(float);
    p.bytes = p.end_delta + rows * sizeof(float);
    return p;
}

}  // namespace
}  // namespace ssm

size_t ssm_ws_bytes(int64_t B, int64_t L, int D, int N) { return ssm::plan(B, L, D, N).bytes; }

cudaError_t ssm_forward(const rlm_strided &x, const rlm_strided &dt, const rlm_strided &b, const rlm_strided &c, const rlm_strided *z,
                        const rlm_ssm_params &p, const float *state_in, const rlm_strided &y, float *state_out, float *saved,
                        const int *lengths, void *ws, cudaStream_t st) {
    const ssm::Plan q = ssm::plan(x.B, x.L, p.D, p.N);
    auto call = [&](auto a) {
        a.state_in = state_in, a.state_out = state_out, a.saved = saved, a.lengths = lengths;
        a.ntiles = q.ntiles, a.nseg = q.nseg, a.per = q.per;
        a.end_state = static_cast<float *>(ws);
        a.end_delta = reinterpret_cast<float *>(static_cast<char *>(ws) + q.end_delta);
        return ssm::run_forward(a, x.B, p.N, st);
    };
    return x.dtype == RLM_BF16 ? call(ssm::arguments<__nv_bfloat16>(x, dt, b, c, z, y, p)) : call(ssm::arguments<float>(x, dt, b, c, z, y, p));
}

cudaError_t ssm_step(const rlm_strided &x, const rlm_strided &dt, const rlm_strided &b, const rlm_strided &c, const rlm_strided *z,
                     const rlm_ssm_params &p, float *state, const rlm_strided &y, cudaStream_t st) {
    return x.dtype == RLM_BF16 ? ssm::run_step(ssm::arguments<__nv_bfloat16>(x, dt, b, c, z, y, p), x.B, p.N, state, st)
                               : ssm::run_step(ssm::arguments<float>(x, dt, b, c, z, y, p), x.B, p.N, state, st);
}

}  // namespace rlm
