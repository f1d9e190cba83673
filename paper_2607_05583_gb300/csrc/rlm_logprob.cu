// rlm_logprob.cu -- log probabilities of given tokens under rows of logits, the rows' entropy and
// top alternatives, and the gradient of the logits.
//
//   m = max_j z_j,  S = sum_j e^(z_j - m),  log p_j = (z_j - m) - log S
//   H = log S - (1 / S) sum_j e^(z_j - m) (z_j - m)
//   dz_j = g ([j = target] - p_j) - e p_j (log p_j + H)
//
// m and log S are kept apart: their sum would lose log S's bits where logits are large.
//
// One pass.  A thread keeps (m, S, W) of the values it has met, W = sum e^(z - m) (z - m); a larger
// maximum scales both by f = e^(m - m') (W first gains (m - m') S), and two such triples join the
// same way.  z - m is held at -200 and above, where e^(z - m) is 0 in fp32: an infinitely negative
// logit (a token that is ruled out) then adds nothing, and 0 times infinity does not arise.  NaN
// passes through the maximum.  Short rows stay in a warp's registers, or go through them in tiles; longer
// ones go by a block, and where there are few rows by a cluster of up to 8 blocks, each with a
// range of the row, whose first block joins the others' results out of its own shared memory.
//
// Top alternatives.  Logits are ordered by a 64-bit key, the value's bits made monotonic above the
// index's complement: no two keys are equal, so ties go to the lowest index, and NaN (above all
// numbers) is shown rather than hidden.  The pass over a long row only notes the maximum of every chunk, the 32
// vectors that a warp loads at once.  The k chunks with the largest maxima (of equal ones the first) hold the k
// largest values, since each has one no smaller than any value outside them; they are read again (a few KB, out of
// L2), and what reaches the k-th chunk's maximum, of what equals it the first k of a chunk, is ranked.  A row in
// which more values do than the buffer holds (sorted logits) is searched k times instead.  (Keeping the best k while
// the row goes by took 236 us for 20 of 4096 x 32000 bf16 logits where the pass alone takes 48.)  A warp that has a row for itself
// bounds its candidates by the k-th largest of its lanes' maxima of even and of odd values, 64 groups, which about
// 64 ln(64 / (64 - k)) values of a row in no order reach, and ranks them by counting.
//
// Rows go to warps where there are enough of them, since a block's two barriers and its last loads' latency come
// with every row (us, fp32, without alternatives / with 20; a block a row, a warp a row):
//   1216 rows of 2000       5.0 / 15.1    3.6 / 10.1        19456 rows of 1100   58.6 / 208.5    18.4 / 54.4
//   1216 rows of 8000       6.6 / 20.1    8.7 / 25.1         2432 rows of 8000   12.0 / 38.0     14.6 / 28.1
//   4864 rows of 4000      17.2 / 66.8   14.5 / 35.9        19456 rows of 8000    108 / 297       103 / 167
// so up to 4096 logits from 8 rows an SM on, up to 8192 from 16 rows on, and always up to 1024.  (The rule does not ask for
// alternatives: 2432 rows of 8000 without any would be faster by blocks.)  In registers, without tiles, a
// row of up to 500 goes faster (19456 of 300: 7.9 / 31 us, in tiles 9.6 / 36; of 520 15.1 / 68 and 12.3 / 41).
// A single alternative is the first value equal to the maximum (67108 rows of 1000: 79 us -> 66; the branch
// costs those with 32 alternatives 190 -> 198).
//
// Bound by memory: the logits are read once, by the gradient once more.  Registers are bounded for the blocks of an SM; three
// instances spill 4 to 16 bytes for it (bf16: the block form with alternatives, 64 registers, the gradient with
// entropy, 80).
#include <algorithm>
#include <type_traits>

#include "rlm_device.cuh"
#include "rlm_internal.h"

namespace rlm {

namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 4;                // 16-byte vectors of a thread's tile
constexpr int kMaxTop = RLM_MAX_TOP;
constexpr int kWarpRow = 500;           // longest row of the warp form
constexpr int kMaxCluster = 8;
constexpr float kLow = -200.f;          // e^kLow is 0 in fp32
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float exp_of(float d) {      // e^d for d <= 0
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d * kLog2e));
    return e;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

template <typename T>
struct Vec;     // 16 bytes of logits
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ float at(const uint4 &v, int i) {
        const uint32_t r = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return __uint_as_float(i & 1 ? r & 0xffff0000u : r << 16);
    }
    static __device__ __forceinline__ uint32_t bits(const __nv_bfloat16 *p) {
        return *reinterpret_cast<const volatile unsigned short *>(p);
    }
    static __device__ __forceinline__ uint4 absent() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
    static __device__ __forceinline__ void set(uint4 &v, int i, uint32_t b) {
        uint32_t &r = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        r = i & 1 ? (r & 0xffffu) | b << 16 : (r & 0xffff0000u) | b;
    }
    static __device__ __forceinline__ float value(const __nv_bfloat16 *p) { return __uint_as_float(bits(p) << 16); }
};
template <>
struct Vec<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ float at(const uint4 &v, int i) {
        return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
    }
    static __device__ __forceinline__ uint32_t bits(const float *p) { return *reinterpret_cast<const volatile uint32_t *>(p); }
    static __device__ __forceinline__ uint4 absent() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    static __device__ __forceinline__ void set(uint4 &v, int i, uint32_t b) {
        (i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w) = b;
    }
    static __device__ __forceinline__ float value(const float *p) { return __uint_as_float(bits(p)); }
};

// A row as 16-byte vectors of the buffer that it lies in: vector i holds columns
// i N - phase + 0 .. N - 1.  Vectors that reach over an end of the row are read by elements,
// and their columns outside it are -inf.
template <typename T>
struct Row {
    static constexpr int kN = Vec<T>::kN;
    const T *p;
    int V, phase, vecs;
    __device__ __forceinline__ Row(const T *z, int64_t row, int64_t ld, int V_) : p(z + row * ld), V(V_) {
        phase = (int)((row * ld) & (kN - 1));
        vecs = (V + phase + kN - 1) / kN;
    }
    __device__ __forceinline__ int column(int vec) const { return vec * kN - phase; }
    __device__ __forceinline__ uint4 load(int vec, int end) const {
        if (vec >= end) return Vec<T>::absent();
        const int j = column(vec);
        if (j >= 0 && j + kN <= V) return load_once(p + j);
        uint4 v = Vec<T>::absent();
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (j + i >= 0 && j + i < V) Vec<T>::set(v, i, Vec<T>::bits(p + j + i));
        return v;
    }
};

// Monotonic in the value: NaN above all, -0 as +0; 0 is below every value's key.
__device__ __forceinline__ uint32_t order(float v) {
    if (v != v) return 0xffffffffu;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key == 0xffffffffu ? 0x7fffffffu : key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
using Key = unsigned long long;
__device__ __forceinline__ Key key_of(float v, int index) { return (Key)order(v) << 32 | (uint32_t)~index; }

// (m, S, W) of some values; none: m = -inf, S = W = 0.
struct Sum {
    float m, S, W;
};
// Brings t to a reference m of its own or larger.
__device__ __forceinline__ void refer(Sum &t, float m) {
    const float d = fmaxf(t.m - m, kLow), f = t.m == kNegInf ? 0.f : exp_of(d);
    t.W = f * fmaf(d, t.S, t.W);
    t.S *= f;
    t.m = m;
}
template <bool kEntropy>
__device__ __forceinline__ Sum join_lanes(Sum t) {
    refer(t, warp_max(t.m));
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        t.S += __shfl_xor_sync(~0u, t.S, o);
        if constexpr (kEntropy) t.W += __shfl_xor_sync(~0u, t.W, o);
    }
    return t;
}

// Adds kCount values whose maximum is top.
template <bool kEntropy, int kCount, typename Value>
__device__ __forceinline__ void add_values(Sum &t, float top, Value value) {
    if (!(top <= t.m)) refer(t, max_nan(top, t.m));
    if (t.m == kNegInf) return;
    const f32x2 minus_m = pack(make_float2(-t.m, -t.m)), log2e = pack(make_float2(kLog2e, kLog2e));
    f32x2 S = pack(make_float2(t.S, 0.f)), W = pack(make_float2(t.W, 0.f));
#pragma unroll
    for (int i = 0; i < kCount; i += 2) {
        f32x2 d = add2(pack(make_float2(value(i), value(i + 1))), minus_m);
        if constexpr (kEntropy) {
            const float2 u = unpack(d);
            d = pack(make_float2(fmaxf(u.x, kLow), fmaxf(u.y, kLow)));
        }
        const float2 x = unpack(mul2(d, log2e));
        float2 e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(x.x));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(x.y));
        S = add2(S, pack(e));
        if constexpr (kEntropy) W = fma2(pack(e), d, W);
    }
    const float2 s = unpack(S), w = unpack(W);
    t.S = s.x + s.y;
    if constexpr (kEntropy) t.W = w.x + w.y;
}

template <typename T>
struct LogprobArgs {
    const T *z;
    int64_t ld, R;
    const void *targets;        // nullable
    bool wide;                  // 64-bit targets
    float *logprob, *entropy, *stats;       // [R], [R], [R][2]; nullable
    int *top_id;                // [R][k]
    float *top_logprob;         // [R][k]
    int V, k;
};

__device__ __forceinline__ int target_of(const void *p, bool wide, int64_t r, int V) {
    if (!p) return -1;
    const int64_t t = wide ? static_cast<const int64_t *>(p)[r] : (int64_t)static_cast<const int32_t *>(p)[r];
    return t >= 0 && t < V ? (int)t : -1;
}

// A row with NaN or +inf has no probabilities (NaN); one of -inf alone has log probabilities -inf and entropy 0.
__device__ __forceinline__ float log_probability(float z, float m, float log_s) {
    if (!(m < -kNegInf)) return m - m;
    return z == kNegInf ? z : z - m - log_s;
}

template <typename T>
__device__ __forceinline__ void row_results(const LogprobArgs<T> &a, int64_t r, Sum t, float log_s) {
    if (a.stats) reinterpret_cast<float2 *>(a.stats)[r] = make_float2(t.m, log_s);
    if (a.logprob) {
        const int tok = target_of(a.targets, a.wide, r, a.V);
        a.logprob[r] = tok < 0 ? 0.f : log_probability(Vec<T>::value(a.z + r * a.ld + tok), t.m, log_s);
    }
    if (a.entropy) a.entropy[r] = t.m == kNegInf ? 0.f : log_s - t.W / t.S + (t.m - t.m);      // (NaN where m is +inf or NaN)
}

template <typename T>
__device__ __forceinline__ void write_top(const LogprobArgs<T> &a, int64_t r, int n, Key x, float m, float log_s) {
    if (a.top_id) a.top_id[r * a.k + n] = (int)~(uint32_t)x;
    if (a.top_logprob) a.top_logprob[r * a.k + n] = log_probability(value_of((uint32_t)(x >> 32)), m, log_s);
}

// ------------------------------------------------------------ a warp's alternatives
constexpr int kWarpCand = 128;
constexpr int kFewTop = 16;             // up to so many alternatives the bound is found maximum after maximum

// A warp's candidates; before there are any, the 64 maxima that give the bound.
struct __align__(16) WarpTop {       // (the maxima are read as vectors of 16 bytes)
    union {
        Key cand[kWarpCand];
        uint32_t maxima[64];
    };
    int count;
};

// The k-th largest of the maxima of the lanes' even and odd values: at least k values of the row reach it, and hardly more than
// the buffer holds.  (Where there is no column the value is -inf: as a bound it lets every column pass.)
__device__ __forceinline__ uint32_t kth_maximum(WarpTop &s, const float (&tops)[2], int k) {
    const int lane = threadIdx.x & 31;
    uint32_t a = order(tops[0]), b = order(tops[1]);
    if (k <= kFewTop) {
        uint32_t bound = 0;
        for (int n = 0; n < k; ++n) {
            const uint32_t best = max(a, b);
            bound = __reduce_max_sync(~0u, best);
            if (lane == __ffs(__ballot_sync(~0u, best == bound)) - 1) (a == bound ? a : b) = 0;
        }
        return bound;
    }
    s.maxima[lane] = a, s.maxima[lane + 32] = b;
    __syncwarp();
    int above_a = 0, above_b = 0;
#pragma unroll
    for (int j = 0; j < 64; j += 4) {
        const uint4 q = *reinterpret_cast<const uint4 *>(s.maxima + j);
        above_a += (q.x > a) + (q.y > a) + (q.z > a) + (q.w > a);
        above_b += (q.x > b) + (q.y > b) + (q.z > b) + (q.w > b);
    }
    __syncwarp();
    return __reduce_min_sync(~0u, min(above_a < k ? a : ~0u, above_b < k ? b : ~0u));
}

// The k largest of s.cand[0 .. n), n <= kMine * 32, as the row's alternatives.
template <int kMine, typename T>
__device__ __forceinline__ void rank_warp(const LogprobArgs<T> &a, int64_t r, const WarpTop &s, int n, float m, float log_s) {
    const int lane = threadIdx.x & 31;
    Key mine[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) mine[i] = lane + 32 * i < n ? s.cand[lane + 32 * i] : 0;
    int rank[kMine] = {};
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
        const Key x = s.cand[j];
#pragma unroll
        for (int i = 0; i < kMine; ++i) rank[i] += x > mine[i];
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (lane + 32 * i < n && rank[i] < a.k) write_top(a, r, rank[i], mine[i], m, log_s);
}
template <typename T>
__device__ __forceinline__ void rank_warp(const LogprobArgs<T> &a, int64_t r, const WarpTop &s, int n, float m, float log_s) {
    if (n <= 32) {
        rank_warp<1>(a, r, s, n, m, log_s);
    } else if (n <= 64) {
        rank_warp<2>(a, r, s, n, m, log_s);
    } else {
        rank_warp<4>(a, r, s, n, m, log_s);
    }
}

// Sums of the lanes before this one.
__device__ __forceinline__ int sum_before(int n) {
    int at = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(~0u, at, o);
        if ((threadIdx.x & 31) >= o) at += u;
    }
    return at - n;
}

// The candidates among kVec vectors a lane, vector i of them at column0 + i * 32 * kN: those that reach the bound and lie in
// the row; with `first_ties`, of those equal to it only the row's first k (`ties` have been met; the vectors come in order).
// Counts on when the buffer is full.
template <int kVec, typename T>
__device__ __forceinline__ void collect(WarpTop &s, const Row<T> &row, int column0, float least, int k, bool first_ties, int &ties,
                                        const uint4 (&v)[kVec]) {
    constexpr int kN = Vec<T>::kN, kWords = (kVec * kN + 31) / 32;
    auto value = [&](int i) { return Vec<T>::at(v[i / kN], i % kN); };
    uint32_t pass[kWords] = {};
#pragma unroll
    for (int i = 0; i < kVec * kN; ++i) pass[i / 32] |= (uint32_t)!(value(i) < least) << i % 32;
    if (!(least > kNegInf)) {
#pragma unroll
        for (int i = 0; i < kVec * kN; ++i) {
            const int j = column0 + i / kN * 32 * kN + i % kN;
            if (j < 0 || j >= row.V) pass[i / 32] &= ~(1u << i % 32);
        }
    }
    if (first_ties) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            uint32_t same = 0;
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (value(i * kN + e) == least) same |= 1u << (i * kN + e) % 32;
            uint32_t &mine = pass[i * kN / 32];
            same &= mine;
            int before = ties + sum_before(__popc(same));
            ties = __shfl_sync(~0u, before + __popc(same), 31);
            for (; same; same &= same - 1)
                if (before++ >= k) mine &= ~(same & -same);
        }
    }
    int n = 0;
#pragma unroll
    for (uint32_t m : pass) n += __popc(m);
    if (n == 0) return;
    int at = atomicAdd(&s.count, n);
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        for (uint32_t m = pass[w]; m; m &= m - 1, ++at) {
            const int i = w * 32 + __ffs(m) - 1, j = column0 + i / kN * 32 * kN + i % kN;
            uint4 u = v[0];         // (registers have no index)
#pragma unroll
            for (int q = 1; q < kVec; ++q)
                if (i / kN == q) u = v[q];
            float x = Vec<T>::at(u, 0);
#pragma unroll
            for (int e = 1; e < kN; ++e)
                if (i % kN == e) x = Vec<T>::at(u, e);
            if (at < kWarpCand) s.cand[at] = key_of(x, j);
        }
    }
}

// The first column whose value is m, the row's largest (neither NaN nor -inf), among kVec vectors a lane as above; the warp's.
template <int kVec, typename T>
__device__ __forceinline__ int first_of(int column0, float m, const uint4 (&v)[kVec]) {
    constexpr int kN = Vec<T>::kN;
    uint32_t first = ~0u;
#pragma unroll
    for (int i = kVec * kN - 1; i >= 0; --i)
        if (Vec<T>::at(v[i / kN], i % kN) == m) first = i / kN * 32 * kN + i % kN;
    return (int)__reduce_min_sync(~0u, first == ~0u ? first : column0 + first);
}

// ------------------------------------------------------- short rows, a warp each
template <typename T, int kV, bool kEntropy, bool kTop>
__global__ void __launch_bounds__(kThreads, kTop && kV > 2 ? 3 : 4) k_logprob_warp(LogprobArgs<T> a) {
    constexpr int kN = Vec<T>::kN;
    __shared__ typename std::conditional<kTop, WarpTop, char>::type tops_of[kThreads / 32];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t stride = (int64_t)gridDim.x * (kThreads / 32);
    uint4 v[kV], next[kV];
    int64_t r = (int64_t)blockIdx.x * (kThreads / 32) + warp;
    if (r >= a.R) return;
    {
        const Row<T> row(a.z, r, a.ld, a.V);
#pragma unroll
        for (int i = 0; i < kV; ++i) next[i] = row.load(i * 32 + lane, row.vecs);
    }
    for (; r < a.R; r += stride) {
        const Row<T> row(a.z, r, a.ld, a.V);
#pragma unroll
        for (int i = 0; i < kV; ++i) v[i] = next[i];
        if (r + stride < a.R) {
            const Row<T> then(a.z, r + stride, a.ld, a.V);
#pragma unroll
            for (int i = 0; i < kV; ++i) next[i] = then.load(i * 32 + lane, then.vecs);
        }
        auto value = [&](int i) { return Vec<T>::at(v[i / kN], i % kN); };
        float tops[2] = {kNegInf, kNegInf};
#pragma unroll
        for (int i = 0; i < kV * kN; ++i) tops[i & 1] = max_nan(tops[i & 1], value(i));
        Sum t{warp_max(max_nan(tops[0], tops[1])), 0, 0};
        add_values<kEntropy, kV * kN>(t, t.m, value);
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            t.S += __shfl_xor_sync(~0u, t.S, o);
            if constexpr (kEntropy) t.W += __shfl_xor_sync(~0u, t.W, o);
        }
        const float log_s = t.m == kNegInf ? 0.f : logf(t.S);
        if (lane == 0) row_results(a, r, t, log_s);
        if constexpr (kTop) {
            WarpTop &s = tops_of[warp];
            if (a.k == 1 && t.m > kNegInf) {        // (the general way: 131072 x 256 bf16 65 us, so 37)
                const int j = first_of<kV, T>(row.column(lane), t.m, v);
                if (lane == 0) write_top(a, r, 0, key_of(t.m, j), t.m, log_s);
                continue;
            }
            const float least = value_of(kth_maximum(s, tops, a.k));
            int n = 0;
            for (int first_ties = 0; first_ties < 2; ++first_ties) {
                int ties = 0;
                if (lane == 0) s.count = 0;
                __syncwarp();
                collect<kV>(s, row, row.column(lane), least, a.k, first_ties, ties, v);
                __syncwarp();
                n = s.count;
                __syncwarp();
                if (n <= kWarpCand) break;
            }
            if (n <= kWarpCand) {
                rank_warp(a, r, s, n, t.m, log_s);
            } else {        // the largest key not above `last`, k times: a lane's own best is found again when it was taken
                Key last = ~0ull, best = 0, x = 0;
                bool stale = true;
                for (int n = 0; n < a.k; ++n) {
                    if (stale) {
                        best = 0;
#pragma unroll
                        for (int i = 0; i < kV * kN; ++i) {
                            const int j = row.column(i / kN * 32 + lane) + i % kN;
                            const Key key = key_of(value(i), j);
                            if (j >= 0 && j < a.V && key <= last && key > best) best = key;
                        }
                    }
                    const uint32_t hi = __reduce_max_sync(~0u, (uint32_t)(best >> 32));
                    const uint32_t lo = __reduce_max_sync(~0u, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
                    stale = best == ((Key)hi << 32 | lo);
                    if (stale) last = best - 1;
                    if (lane == n) x = (Key)hi << 32 | lo;
                }
                if (lane < a.k) write_top(a, r, lane, x, t.m, log_s);
            }
            __syncwarp();
        }
    }
}

// ------------------------------------------- many rows of some thousand logits, a warp each
// As the short rows, but tile by tile, the next one's loads (at a row's end the next row's) in flight.
constexpr int kStreamRow = 8192, kLoneRow = 1024;
constexpr int kStreamVecs = 4;
template <typename T, bool kEntropy, bool kTop>
__global__ void __launch_bounds__(kThreads, 3) k_logprob_stream(LogprobArgs<T> a) {
    constexpr int kN = Vec<T>::kN, kTile = kStreamVecs * 32, kChunks = (kStreamRow + 2 * kN - 2) / kN / 32 + 1;
    __shared__ typename std::conditional<kTop, WarpTop, char>::type tops_of[kThreads / 32];
    __shared__ float chunk_max[kTop ? kThreads / 32 : 1][kTop ? kChunks : 1];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t stride = (int64_t)gridDim.x * (kThreads / 32);
    int64_t r = (int64_t)blockIdx.x * (kThreads / 32) + warp;
    if (r >= a.R) return;
    uint4 v[kStreamVecs], next[kStreamVecs];
    auto fetch = [&](const Row<T> &row, int vec0) {
#pragma unroll
        for (int i = 0; i < kStreamVecs; ++i) next[i] = row.load(vec0 + i * 32 + lane, row.vecs);
    };
    fetch(Row<T>(a.z, r, a.ld, a.V), 0);
    for (; r < a.R; r += stride) {
        const Row<T> row(a.z, r, a.ld, a.V);
        Sum t{kNegInf, 0, 0};
        float tops[2] = {kNegInf, kNegInf};
        for (int vec0 = 0; vec0 < row.vecs; vec0 += kTile) {
#pragma unroll
            for (int i = 0; i < kStreamVecs; ++i) v[i] = next[i];
            if (vec0 + kTile < row.vecs) {
                fetch(row, vec0 + kTile);
            } else if (r + stride < a.R) {
                fetch(Row<T>(a.z, r + stride, a.ld, a.V), 0);
            }
            float top = kNegInf;
#pragma unroll
            for (int i = 0; i < kStreamVecs; ++i) {
                float m[2] = {kNegInf, kNegInf};
#pragma unroll
                for (int j = 0; j < kN; ++j) m[j & 1] = max_nan(m[j & 1], Vec<T>::at(v[i], j));
                top = max_nan(top, max_nan(m[0], m[1]));
                if constexpr (kTop) {
                    tops[0] = max_nan(tops[0], m[0]), tops[1] = max_nan(tops[1], m[1]);
                    const float most = warp_max(max_nan(m[0], m[1]));
                    if (lane == 0 && vec0 + i * 32 < row.vecs) chunk_max[warp][vec0 / 32 + i] = most;
                }
            }
            add_values<kEntropy, kStreamVecs * kN>(t, top, [&](int i) { return Vec<T>::at(v[i / kN], i % kN); });
        }
        t = join_lanes<kEntropy>(t);
        const float log_s = t.m == kNegInf ? 0.f : logf(t.S);
        if (lane == 0) row_results(a, r, t, log_s);
        if constexpr (kTop) {
            WarpTop &s = tops_of[warp];
            __syncwarp();
            if (a.k == 1 && t.m > kNegInf) {        // in the first chunk with that maximum
                const int chunks = (row.vecs + 31) / 32;
                uint32_t have = 0;
                int c = -32;
                while (!have && c + 32 < chunks) {
                    c += 32;
                    have = __ballot_sync(~0u, c + lane < chunks && chunk_max[warp][min(c + lane, chunks - 1)] == t.m);
                }
                c += __ffs(have) - 1;
                const uint4 u[1] = {row.load(c * 32 + lane, row.vecs)};
                const int j = first_of<1, T>(row.column(c * 32 + lane), t.m, u);
                if (lane == 0) write_top(a, r, 0, key_of(t.m, j), t.m, log_s);
                __syncwarp();
                continue;
            }
            const float least = value_of(kth_maximum(s, tops, a.k));
            // fn(vector, its values) for the chunks that hold a candidate, four chunks' loads at a time
            const int chunks = (row.vecs + 31) / 32;
            auto each = [&](auto fn) {
                for (int c0 = 0; c0 < chunks; c0 += 32) {
                    uint32_t have = __ballot_sync(~0u, c0 + lane < chunks && !(chunk_max[warp][min(c0 + lane, chunks - 1)] < least));
                    while (have) {
                        constexpr int kAtOnce = 4;
                        int c[kAtOnce];
                        uint4 u[kAtOnce][1];
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i) {
                            c[i] = have ? c0 + __ffs(have) - 1 : chunks;
                            have &= have - 1;
                            u[i][0] = row.load(c[i] * 32 + lane, row.vecs);
                        }
#pragma unroll
                        for (int i = 0; i < kAtOnce; ++i)
                            if (c[i] < chunks) fn(c[i] * 32 + lane, u[i]);
                    }
                }
            };
            int n = 0;
            for (int first_ties = 0; first_ties < 2; ++first_ties) {
                int ties = 0;
                if (lane == 0) s.count = 0;
                __syncwarp();
                each([&](int vec, const uint4 (&u)[1]) {
                    collect<1>(s, row, row.column(vec), least, a.k, first_ties, ties, u);
                    __syncwarp();
                });
                n = s.count;
                __syncwarp();
                if (n <= kWarpCand) break;
            }
            if (n <= kWarpCand) {
                rank_warp(a, r, s, n, t.m, log_s);
            } else {
                Key last = ~0ull;
                for (int i = 0; i < a.k; ++i) {
                    Key best = 0;
                    each([&](int vec, const uint4 (&u)[1]) {
#pragma unroll
                        for (int e = 0; e < kN; ++e) {
                            const int j = row.column(vec) + e;
                            const Key x = key_of(Vec<T>::at(u[0], e), j);
                            if (vec < row.vecs && j >= 0 && j < a.V && x <= last && x > best) best = x;
                        }
                    });
                    const uint32_t hi = __reduce_max_sync(~0u, (uint32_t)(best >> 32));
                    const uint32_t lo = __reduce_max_sync(~0u, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
                    best = (Key)hi << 32 | lo;
                    if (lane == 0) write_top(a, r, i, best, t.m, log_s);
                    last = best - 1;
                }
            }
            __syncwarp();
        }
    }
}

// ------------------------------------------------- longer rows, a block or a cluster each
constexpr int kCand = kMaxTop * kMaxTop + 1024;     // ties of the chosen chunks, and what lies above them
struct TopState {
    Key best[kMaxTop];
    Key cand[kCand];
    Key warp_best[kThreads / 32];
    uint32_t chosen[kMaxTop], bound;
    int count;
};
struct RowState {
    Sum part[kThreads / 32];
    Sum joined[kMaxCluster];        // of the cluster's blocks (in its first block)
    Key best[kMaxCluster * kMaxTop];
};

// cand[0 .. n), all different -> best[0 .. k), descending; what lies behind the last stays.
__device__ __forceinline__ void rank_candidates(const Key *cand, int n, Key *best, int k) {
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const Key x = cand[i];
        if (x == 0) continue;
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += cand[j] > x;
        if (rank < k) best[rank] = x;
    }
}

// The k largest of count maxima, of equal ones the first, into s.chosen, and the k-th (0 where there are fewer): one warp.
__device__ __forceinline__ void choose(TopState &s, uint32_t *maxima, int count, int k) {
    constexpr int kHeld = 8;                // of a lane's maxima in registers; any more are looked through in shared memory
    const int lane = threadIdx.x & 31, n = min(k, count);
    uint32_t held[kHeld], rest = 0, rest_at = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = lane + 32 * i < count ? maxima[lane + 32 * i] : 0;
    auto look = [&] {
        rest = 0;
        for (int i = lane + 32 * kHeld; i < count; i += 32)
            if (maxima[i] > rest) rest = maxima[i], rest_at = i;
    };
    look();
    for (int i = 0; i < n; ++i) {
        uint32_t best = rest, at = rest_at;
#pragma unroll
        for (int j = kHeld - 1; j >= 0; --j)
            if (held[j] >= best) best = held[j], at = lane + 32 * j;
        all = __reduce_max_sync(~0u, best);
        const uint32_t first = __reduce_min_sync(~0u, best == all ? at : ~0u);
        if (lane == 0) s.chosen[i] = first;
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
            if (first == lane + 32 * j) held[j] = 0;
        if (first >= 32 * kHeld && first % 32 == lane) {
            maxima[first] = 0;
            look();
        }
    }
    if (lane == 0) s.bound = n < k ? 0 : all;
}

// The same by counting, with all threads: few maxima at less latency (where rows fill the GPU, the other one).
constexpr int kFewMaxima = 128;
__device__ __forceinline__ void choose_by_rank(TopState &s, const uint32_t *maxima, int count, int k) {
    const int i = threadIdx.x;
    if (i < count) {
        const uint32_t x = maxima[i];
        int rank = 0;
#pragma unroll 16
        for (int j = 0; j < count; ++j) {
            const uint32_t y = maxima[j];
            rank += y > x || (y == x && j < i);
        }
        if (rank < k) s.chosen[rank] = i;
        if (rank == k - 1) s.bound = x;
    }
    if (i == 0 && count < k) s.bound = 0;
}

// The block's k largest keys into s.best; called by all threads, the chunks' maxima being in maxima (not where there are
// fewer than k of them).
template <typename T>
__device__ __forceinline__ void find_top(TopState &s, uint32_t *maxima, int k, const Row<T> &row, int begin, int end, float top,
                                         bool hasty) {
    constexpr int kN = Vec<T>::kN;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int count = (end - begin + 31) / 32;
    if (k == 1) {           // the first value of the first chunk with the largest maximum; read behind the caller's next barrier
        __syncthreads();
        if (warp != 0) return;
        choose(s, maxima, count, 1);
        __syncwarp();
        const uint32_t bound = s.bound;
        const int vec = begin + (count ? (int)s.chosen[0] : 0) * 32 + lane, j0 = row.column(vec);
        const uint4 v = row.load(vec, end);
        uint32_t first = ~0u;
#pragma unroll
        for (int i = kN - 1; i >= 0; --i) {
            const int j = j0 + i;
            if (vec < end && j >= 0 && j < row.V && order(Vec<T>::at(v, i)) == bound) first = j;
        }
        first = __reduce_min_sync(~0u, first);
        if (lane == 0) s.best[0] = count ? (Key)bound << 32 | (uint32_t)~first : 0;
        return;
    }
    // A block with fewer chunks than k (of one tile) takes its bound from the threads' maxima, and looks at every chunk.
    const bool few = count < k;
    if (few) maxima[tid] = begin + tid < end ? order(top) : 0;
    __syncthreads();
    if (hasty && !few && count <= kFewMaxima) {
        choose_by_rank(s, maxima, count, k);
    } else if (warp == 0) {
        choose(s, maxima, few ? kThreads : count, k);
    }
    if (tid < kMaxTop) s.best[tid] = 0;
    if (tid == 0) s.count = 0;
    __syncthreads();
    const uint32_t bound = s.bound;
    const int chosen = few ? count : k;
    auto chunk = [&](int c) { return few ? c : (int)s.chosen[c]; };
    constexpr int kLoads = kMaxTop / (kThreads / 32);
    uint4 loaded[kLoads];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
        const int c = warp + l * (kThreads / 32);
        loaded[l] = c < chosen ? row.load(begin + chunk(c) * 32 + lane, end) : Vec<T>::absent();
    }
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
        const int c = warp + l * (kThreads / 32);
        if (c >= chosen) break;
        const int vec = begin + chunk(c) * 32 + lane, j0 = row.column(vec);
        const uint4 v = loaded[l];
        uint32_t key[kN];
        int ties = 0;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int j = j0 + i;
            key[i] = vec < end && j >= 0 && j < row.V ? order(Vec<T>::at(v, i)) : 0u;
            ties += key[i] != 0 && key[i] == bound;
        }
        int before = ties;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(~0u, before, o);
            if (lane >= o) before += u;
        }
        before -= ties;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            if (key[i] == 0 || key[i] < bound) continue;
            if (key[i] == bound && before++ >= k) continue;
            const int at = atomicAdd(&s.count, 1);
            if (at < kCand) s.cand[at] = (Key)key[i] << 32 | (uint32_t)~(j0 + i);
        }
    }
    __syncthreads();
    const int n = s.count;
    if (n <= kCand) {
        rank_candidates(s.cand, n, s.best, k);
    } else {
        Key last = ~0ull;
        for (int i = 0; i < k; ++i) {
            Key best = 0;
            for (int c = warp; c < chosen; c += kThreads / 32) {
                const int vec = begin + chunk(c) * 32 + lane, j0 = row.column(vec);
                const uint4 v = row.load(vec, end);
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    const int j = j0 + e;
                    const Key x = key_of(Vec<T>::at(v, e), j);
                    if (vec < end && j >= 0 && j < row.V && x <= last && x > best) best = x;
                }
            }
            const uint32_t hi = __reduce_max_sync(~0u, (uint32_t)(best >> 32));
            const uint32_t lo = __reduce_max_sync(~0u, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
            if (lane == 0) s.warp_best[warp] = (Key)hi << 32 | lo;
            __syncthreads();
            best = 0;
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) best = s.warp_best[w] > best ? s.warp_best[w] : best;
            if (tid == 0) s.best[i] = best;
            last = best - 1;
            __syncthreads();
            if (best == 0) break;
        }
    }
    __syncthreads();
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_first_block(const void *p) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)));
    return r;
}

template <typename T, bool kEntropy, bool kTop>
__global__ void __launch_bounds__(kThreads, 4) k_logprob_block(LogprobArgs<T> a, int cluster) {
    constexpr int kN = Vec<T>::kN;
    extern __shared__ uint32_t maxima[];        // with kTop: the maxima of the block's chunks, as order() of them
    __shared__ RowState row_state;
    __shared__ typename std::conditional<kTop, TopState, char>::type top_state;
    wait_for_previous();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int part = blockIdx.x % cluster;
    const int64_t r = blockIdx.x / cluster;
    const Row<T> row(a.z, r, a.ld, a.V);
    const int per = (row.vecs + cluster - 1) / cluster, begin = min(part * per, row.vecs), end = min(begin + per, row.vecs);
    uint4 v[kVecs], next[kVecs];
    auto fetch = [&](int vec0) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) next[i] = row.load(vec0 + tid + i * kThreads, end);
    };
    fetch(begin);
    const bool noted = (end - begin + 31) / 32 >= a.k;      // (else find_top writes to maxima at once)
    Sum t{kNegInf, 0, 0};
    float top = kNegInf;
    for (int vec0 = begin; vec0 < end; vec0 += kVecs * kThreads) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = next[i];
        if (vec0 + kVecs * kThreads < end) fetch(vec0 + kVecs * kThreads);
        top = kNegInf;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            float m = kNegInf;
#pragma unroll
            for (int j = 0; j < kN; ++j) m = max_nan(m, Vec<T>::at(v[i], j));
            top = max_nan(top, m);
            if constexpr (kTop) {
                if (noted) {
                    m = warp_max(m);
                    const int first = vec0 + i * kThreads + warp * 32;
                    if (lane == 0 && first < end) maxima[(first - begin) / 32] = order(m);
                }
            }
        }
        add_values<kEntropy, kVecs * kN>(t, top, [&](int i) { return Vec<T>::at(v[i / kN], i % kN); });
    }
    if constexpr (kTop) find_top<T>(top_state, maxima, a.k, row, begin, end, top, cluster > 1);
    t = join_lanes<kEntropy>(t);
    if (lane == 0) row_state.part[warp] = t;
    __syncthreads();
    if (warp == 0) {
        t = lane < kThreads / 32 ? row_state.part[lane] : Sum{kNegInf, 0, 0};
        t = join_lanes<kEntropy>(t);
    }
    const Key *best = nullptr;
    if constexpr (kTop) best = top_state.best;
    if (cluster > 1) {
        cluster_sync();         // the first block runs, and its part of the row is behind it
        if (tid == 0) {
            const uint32_t to = in_first_block(&row_state.joined[part]);
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(t.m) : "memory");
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4), "f"(t.S) : "memory");
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 8), "f"(t.W) : "memory");
        }
        if constexpr (kTop) {
            if (tid < a.k)
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(in_first_block(&row_state.best[part * a.k + tid])),
                             "l"(top_state.best[tid])
                             : "memory");
        }
        cluster_sync();
        if (part != 0) return;
        if (warp == 0) t = join_lanes<kEntropy>(lane < cluster ? row_state.joined[lane] : Sum{kNegInf, 0, 0});
        if constexpr (kTop) {
            rank_candidates(row_state.best, cluster * a.k, top_state.cand, a.k);
            best = top_state.cand;
        }
        __syncthreads();
    }
    if (warp == 0) {
        const float log_s = t.m == kNegInf ? 0.f : logf(t.S);
        if (lane == 0) row_results(a, r, t, log_s);
        if constexpr (kTop)
            if (lane < a.k) write_top(a, r, lane, best[lane], t.m, log_s);
    }
}

// ------------------------------------------------------------------ gradient
template <typename TI, typename TO>
struct GradArgs {
    const TI *z;
    TO *dz;
    int64_t ld, dz_ld, R;
    const void *targets;
    bool wide;
    const float *stats, *d_logprob, *entropy, *d_entropy;   // entropy and d_entropy nullable together
    int V, lanes, chunks;       // lanes: threads that share a row; chunks: pieces of columns
    int64_t pieces;             // at most 2^31
};

// kN logits as loaded.
template <typename T, int kN>
struct In {
    uint32_t w[kN * sizeof(T) / 4];
    __device__ __forceinline__ void load(const T *p) {          // aligned to their size
#pragma unroll
        for (int i = 0; i < kN * (int)sizeof(T) / 4; i += 4) {
            if constexpr (kN * sizeof(T) >= 16) {
                const uint4 v = load_once(reinterpret_cast<const char *>(p) + 4 * i);
                w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
            } else {
                const uint2 v = load_once8(p);
                w[0] = v.x, w[1] = v.y;
            }
        }
    }
    __device__ __forceinline__ void set(int i, uint32_t b) {
        if constexpr (sizeof(T) == 4) {
            w[i] = b;
        } else {
            w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | b << 16 : (w[i / 2] & 0xffff0000u) | b;
        }
    }
    __device__ __forceinline__ float2 pair(int i) const {       // i even
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[i]), __uint_as_float(w[i + 1]));
        return make_float2(__uint_as_float(w[i / 2] << 16), __uint_as_float(w[i / 2] & 0xffff0000u));
    }
};
__device__ __forceinline__ void store_values(float *p, const float (&f)[4]) {
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void store_values(__nv_bfloat16 *p, const float (&f)[8]) {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 o = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        r[i] = *reinterpret_cast<const uint32_t *>(&o);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}

// What a row's gradient takes beside its logits.
struct Factors {
    int tok;
    float m, log_s, g, e, H;
    bool zero;
};

// Vectors are those of the output's rows; the logits are read the same way where they lie the same way.  A block
// takes pieces of 256 / lanes rows by lanes x kVecs vectors.  kAhead (bf16 on either side): every gridDim.x-th piece, the
// next one's logits in flight while this one is formed, and the factors of the one after it, which say whether its
// logits are read (8192 x 50257 bf16: 275 us, 6.0 TB/s; with a piece a block and the loads' latency in the
// open 408).  fp32 on both sides has half the arithmetic a byte: a piece of 8 vectors a thread a block, four blocks on an
// SM (2047 x 32000: 80 us, 6.5 TB/s; 87 and more ahead).
template <typename TI, typename TO, bool kEntropy, int kVecs, int kResident, bool kAhead>
__global__ void __launch_bounds__(kThreads, kResident) k_logprob_grad(GradArgs<TI, TO> a) {
    constexpr int kN = Vec<TO>::kN;
    wait_for_previous();
    const int64_t rows = kThreads / a.lanes;
    const int vec_in_piece = threadIdx.x % a.lanes, row_in_piece = threadIdx.x / a.lanes;
    auto row_of = [&](int64_t piece) { return (int64_t)((uint32_t)piece / (uint32_t)a.chunks) * rows + row_in_piece; };
    auto factors = [&](int64_t piece) {
        Factors f = {-1, kNegInf, 0.f, 0.f, 0.f, 0.f, true};
        const int64_t r = row_of(piece);
        if (piece >= a.pieces || r >= a.R) return f;
        f.tok = target_of(a.targets, a.wide, r, a.V);
        const float2 st = reinterpret_cast<const float2 *>(a.stats)[r];
        f.m = st.x, f.log_s = st.y;
        f.g = f.tok >= 0 ? a.d_logprob[r] : 0.f;
        if constexpr (kEntropy) f.e = a.d_entropy[r], f.H = a.entropy[r];
        f.zero = f.m == kNegInf || (f.g == 0.f && (!kEntropy || f.e == 0.f));
        return f;
    };
    In<TI, kN> next[kVecs], v[kVecs];
    auto fetch = [&](int64_t piece, const Factors &f) {
        const int64_t r = row_of(piece);
        if (f.zero || piece >= a.pieces || r >= a.R) return;
        const Row<TO> out(a.dz, r, a.dz_ld, a.V);
        const bool alike = ((r * a.ld) & (kN - 1)) == out.phase;
        const TI *z = a.z + r * a.ld;
        const int vec0 = (int)((uint32_t)piece % (uint32_t)a.chunks) * a.lanes * kVecs + vec_in_piece;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int vec = vec0 + i * a.lanes, j = out.column(vec);
            if (vec >= out.vecs) break;
            if (alike && j >= 0 && j + kN <= a.V) {
                next[i].load(z + j);
            } else {
#pragma unroll
                for (int c = 0; c < kN; ++c) next[i].set(c, j + c >= 0 && j + c < a.V ? Vec<TI>::bits(z + j + c) : 0u);
            }
        }
    };
    const int64_t step = gridDim.x;
    Factors f, f1 = factors(blockIdx.x), f2 = f1;
    if constexpr (kAhead) f2 = factors(blockIdx.x + step);
    fetch(blockIdx.x, f1);
    for (int64_t piece = blockIdx.x; piece < a.pieces; piece += step) {
        f = f1, f1 = f2;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = next[i];
        if constexpr (kAhead) {
            fetch(piece + step, f1);
            f2 = factors(piece + 2 * step);
        }
        const int64_t r = row_of(piece);
        if (r >= a.R) continue;
        const Row<TO> out(a.dz, r, a.dz_ld, a.V);
        TO *dz = a.dz + r * a.dz_ld;
        const int vec0 = (int)((uint32_t)piece % (uint32_t)a.chunks) * a.lanes * kVecs + vec_in_piece;
        const f32x2 log2e = pack(make_float2(kLog2e, kLog2e)), minus_m = pack(make_float2(-f.m, -f.m));
        const f32x2 minus_s = pack(make_float2(-f.log_s, -f.log_s)), minus_g = pack(make_float2(-f.g, -f.g));
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int vec = vec0 + i * a.lanes, j = out.column(vec);
            if (vec >= out.vecs) break;
            float o[kN];
#pragma unroll
            for (int c = 0; c < kN; c += 2) {
                const f32x2 lp = add2(add2(pack(v[i].pair(c)), minus_m), minus_s);
                float2 p = unpack(mul2(lp, log2e));
                asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.x));
                asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(p.y));
                f32x2 w = mul2(minus_g, pack(p));
                if constexpr (kEntropy) {
                    float2 l = unpack(lp);
                    l = make_float2(fmaxf(l.x, kLow) + f.H, fmaxf(l.y, kLow) + f.H);
                    w = fma2(mul2(pack(make_float2(-f.e, -f.e)), pack(p)), pack(l), w);
                }
                const float2 q = unpack(w);
                o[c] = f.zero ? 0.f : q.x, o[c + 1] = f.zero ? 0.f : q.y;
            }
            if ((unsigned)(f.tok - j) < (unsigned)kN && !f.zero) {      // the target's own term
#pragma unroll
                for (int c = 0; c < kN; ++c)
                    if (j + c == f.tok) o[c] += f.g;
            }
            if (j >= 0 && j + kN <= a.V) {
                store_values(dz + j, o);
            } else {
#pragma unroll
                for (int c = 0; c < kN; ++c)
                    if (j + c >= 0 && j + c < a.V) st_elem(dz + j + c, o[c]);
            }
        }
    }
}

template <typename T>
LogprobArgs<T> arguments(const rlm_matrix &z, const rlm_tokens *targets, float *logprob, float *entropy, int k, int *top_id,
                         float *top_logprob, float *stats) {
    return {static_cast<const T *>(z.ptr), z.ld, z.rows, targets ? targets->ptr : nullptr, targets && targets->bits == 64, logprob,
            entropy, stats, top_id, top_logprob, (int)z.cols, k};
}

template <typename T, int kV, bool kEntropy>
cudaError_t forward_warp(const LogprobArgs<T> &a, cudaStream_t st) {
    // A warp a row; with many rows 8 blocks an SM, whose warps have the next row's loads in flight.
    const int64_t rows = kThreads / 32, blocks = std::min((a.R + rows - 1) / rows, (int64_t)8 * sm_count());
    return launch_dependent(a.k ? k_logprob_warp<T, kV, kEntropy, true> : k_logprob_warp<T, kV, kEntropy, false>, dim3((unsigned)blocks),
                            kThreads, 0, st, 1, a);
}

template <typename T, bool kEntropy>
cudaError_t forward_e(const LogprobArgs<T> &a, cudaStream_t st) {
    constexpr int kN = Vec<T>::kN;
    if (a.V <= kWarpRow) {
        const int vecs = (a.V + (a.ld % kN ? 2 : 1) * (kN - 1)) / kN;       // (at any phase, where rows have several)
        if (vecs <= 32) return forward_warp<T, 1, kEntropy>(a, st);
        if (vecs <= 64) return forward_warp<T, 2, kEntropy>(a, st);
        return forward_warp<T, kWarpRow / 32 / kN + 1, kEntropy>(a, st);
    }
    if (a.V <= kLoneRow || (a.V <= kStreamRow && a.R >= (int64_t)(a.V <= kStreamRow / 2 ? 8 : 16) * sm_count())) {
        const int64_t rows = kThreads / 32, blocks = std::min((a.R + rows - 1) / rows, (int64_t)3 * sm_count());
        return launch_dependent(a.k ? k_logprob_stream<T, kEntropy, true> : k_logprob_stream<T, kEntropy, false>, dim3((unsigned)blocks),
                                kThreads, 0, st, 1, a);
    }
    // Clusters while that leaves every block half a tile and gives no SM more than two blocks (100 x 32000 fp32 with 20
    // alternatives: pairs 10.6 us, clusters of 4 11.6; 200 x 32000 bf16: single blocks 12.4, pairs 13.9).
    int cluster = 1;
    while (cluster < kMaxCluster && a.R * cluster <= sm_count() && a.V / (2 * cluster) >= kThreads * kVecs * kN / 2) cluster *= 2;
    const dim3 grid((unsigned)(a.R * cluster));
    if (!a.k) return launch_dependent(k_logprob_block<T, kEntropy, false>, grid, kThreads, 0, st, cluster, a, cluster);
    const int vecs = (a.V + 2 * kN - 2) / kN;
    const size_t bytes = std::max((vecs / cluster + 63) / 32, kThreads) * sizeof(uint32_t);       // (at most 32 KB, with 19 KB of its own)
    auto *fn = k_logprob_block<T, kEntropy, true>;
    if (bytes > 24 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, 40 * 1024);
        if (e != cudaSuccess) return e;
    }
    return launch_dependent(fn, grid, kThreads, bytes, st, cluster, a, cluster);
}
template <typename T>
cudaError_t forward(const LogprobArgs<T> &a, cudaStream_t st) {
    return a.entropy ? forward_e<T, true>(a, st) : forward_e<T, false>(a, st);
}

template <typename TI, typename TO>
cudaError_t backward(const rlm_matrix &z, const rlm_tokens &targets, const float *stats, const float *d_logprob,
                     const float *entropy, const float *d_entropy, const rlm_matrix &dz, cudaStream_t st) {
    constexpr int kN = Vec<TO>::kN;
    constexpr bool wide = sizeof(TI) == 4 && sizeof(TO) == 4;
    constexpr int kV = wide ? 8 : 4, kResident = wide ? 4 : sizeof(TI) == 2 ? 3 : 2;
    constexpr bool kAhead = !wide;
    GradArgs<TI, TO> a{static_cast<const TI *>(z.ptr), static_cast<TO *>(dz.ptr), z.ld, dz.ld, z.rows, targets.ptr, targets.bits == 64,
                       stats, d_logprob, entropy, d_entropy, (int)z.cols, 8, 1, 0};
    const int vecs = (a.V + 2 * kN - 2) / kN;
    while (a.lanes < kThreads && a.lanes * kV < vecs) a.lanes *= 2;
    a.chunks = (vecs + a.lanes * kV - 1) / (a.lanes * kV);
    const int64_t rows = kThreads / a.lanes;
    a.pieces = (a.R + rows - 1) / rows * a.chunks;
    const dim3 grid((unsigned)(kAhead ? std::min<int64_t>(a.pieces, kResident * sm_count()) : a.pieces));
    return launch_dependent(d_entropy ? k_logprob_grad<TI, TO, true, kV, kResident, kAhead> : k_logprob_grad<TI, TO, false, kV, kResident, kAhead>,
                            grid, kThreads, 0, st, 1, a);
}

}  // namespace

cudaError_t logprob_forward(const rlm_matrix &z, const rlm_tokens *targets, float *logprob, float *entropy, int k, int *top_id,
                            float *top_logprob, float *stats, cudaStream_t st) {
    if (z.dtype == RLM_BF16)
        return forward(arguments<__nv_bfloat16>(z, targets, logprob, entropy, k, top_id, top_logprob, stats), st);
    return forward(arguments<float>(z, targets, logprob, entropy, k, top_id, top_logprob, stats), st);
}

cudaError_t logprob_backward(const rlm_matrix &z, const rlm_tokens &targets, const float *stats, const float *d_logprob,
                             const float *entropy, const float *d_entropy, const rlm_matrix &dz, cudaStream_t st) {
    if (z.dtype == RLM_BF16)
        return dz.dtype == RLM_BF16
                   ? backward<__nv_bfloat16, __nv_bfloat16>(z, targets, stats, d_logprob, entropy, d_entropy, dz, st)
                   : backward<__nv_bfloat16, float>(z, targets, stats, d_logprob, entropy, d_entropy, dz, st);
    return dz.dtype == RLM_BF16 ? backward<float, __nv_bfloat16>(z, targets, stats, d_logprob, entropy, d_entropy, dz, st)
                                : backward<float, float>(z, targets, stats, d_logprob, entropy, d_entropy, dz, st);
}

}  // namespace rlm
