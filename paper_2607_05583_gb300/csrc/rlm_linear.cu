// rlm_linear.cu -- matrix products with fused epilogues: a linear layer and its gradients.
//
//   forward   z = x w^T + bias, y = act(z) + residual         x [R][K], w [N][K]
//   backward  dz = dy act'(z);  dx = dz w;  dw = dz^T x;  dbias = sum over rows of dz
//
// The three products are one kernel, C[M][N] = sum_k A[m][k] B[n][k], whose operands lie
// either with the contraction index contiguous (K-major) or with the row index contiguous
// (MN-major): x w^T is K, K; dz w is K, MN; dz^T x is MN, MN.  TMA brings either form into
// 128-byte swizzled shared memory and tcgen05.mma reads either, so nothing is transposed.
//
// k_gemm.  Persistent, one CTA per SM, contraction steps of 64; tiles of 256 x 256 or 256 x
// 128 by pairs of CTAs (cta_group::2), or 128 x 128 by single ones where pairs would be
// few.  Warp 16 feeds a ring of operand stages, warp 17 issues the MMAs into one of two TMEM
// accumulators, warps 0-15 empty the other: warp w owns TMEM lanes 32 (w mod 4) .. + 31 and
// quarter w / 4 of the columns, 64 bytes of output at a time, from registers through its own
// 2 KB of shared memory to 64-byte row pieces.  (TMA stores share the copy engine with the
// operands, a row a request: 48 against 36 us at 131072 x 256 x 512.)  Long contractions are
// bound by the tensor pipe (91 % busy at 8192 x 2048 x 4096; 8192 x 4096 x 8192 takes 271 to
// 285 us by the machine, 1930 to 2030 TFLOP/s), short ones by memory and this path's latency:
// sixteen warps where eight would do, 35 us at 131072 x 256 x 512 (5.7 TB/s).  A pair halves
// what a CTA reads of B: the same kernel with single 128 x 256 tiles took 319 us.  The MMA and
// copy warps run warp-uniform code and elect a lane at the instruction itself; issued from a
// divergent thread an MMA took 130 cycles, whatever its width.  Where the last round of 256 x
// 256 tiles would leave half the pairs idle its tiles are cut into halves (4096 x 4096 x 4096
// with gelu, bias and residual 80 -> 74 us, gradients of 8192 x 2048 x 8192 387 -> 366).  A
// product of few tiles is cut along the contraction (splits): partial sums go to the
// workspace in fp32 and k_finish adds them in order and applies the epilogue.  Accumulation is
// fp32 throughout; results repeat bit for bit.
//
// dz is rounded to bf16 once, the operand type of the two products that read it; dbias is
// summed from the fp32 values.
#include <algorithm>
#include <atomic>
#include <mutex>
#include <type_traits>

#include "rlm_device.cuh"
#include "rlm_internal.h"
#include "rlm_umma.cuh"

namespace rlm {

__device__ int g_linear_status = 0;
static std::atomic<bool> g_linear_waits{false};      // whether a kernel that may set it was launched

namespace {

using namespace umma;
using bf16 = __nv_bfloat16;

// ------------------------------------------------------------- activations
__device__ __forceinline__ float sigmoidf(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
constexpr float kBend1 = 1.5957691216f, kBend3 = 0.0713548163f;     // 2 sqrt(2 / pi), and times 0.044715

template <int kAct>
__device__ __forceinline__ float act(float z) {
    if (kAct == RLM_ACT_SILU) return z * sigmoidf(z);
    if (kAct == RLM_ACT_SIGMOID) return sigmoidf(z);
    if (kAct == RLM_ACT_GELU) return z * sigmoidf(z * fmaf(kBend3 * z, z, kBend1));
    return z;
}
__device__ __forceinline__ float act_of(int kind, float z) {
    switch (kind) {
        case RLM_ACT_SILU: return act<RLM_ACT_SILU>(z);
        case RLM_ACT_SIGMOID: return act<RLM_ACT_SIGMOID>(z);
        case RLM_ACT_GELU: return act<RLM_ACT_GELU>(z);
        default: return z;
    }
}
// The same on two values.  sigma's exponential and reciprocal are the approximate instructions
// (2^-22 each); e^-u past fp32's range gives 1 / inf = 0.
__device__ __forceinline__ f32x2 sigmoid2(f32x2 minus_u_log2e) {
    float2 e = unpack(minus_u_log2e);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    e = unpack(add2(pack(e), 0x3f8000003f800000ull));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    return pack(e);
}
__device__ __forceinline__ f32x2 twice(float v) { return pack(make_float2(v, v)); }
template <int kAct>
__device__ __forceinline__ f32x2 act2(f32x2 z) {
    constexpr float l2e = 1.44269504f;
    if (kAct == RLM_ACT_SILU) return mul2(z, sigmoid2(mul2(z, twice(-l2e))));
    if (kAct == RLM_ACT_SIGMOID) return sigmoid2(mul2(z, twice(-l2e)));
    if (kAct == RLM_ACT_GELU)
        return mul2(z, sigmoid2(mul2(z, fma2(mul2(z, z), twice(-l2e * kBend3), twice(-l2e * kBend1)))));
    return z;
}
// act'(z) of two values.  1 - sigma(u) is e^-u sigma(u): the difference would lose it for large
// u.  z is held where |u| < 85.2, so that e^-u, its inverse and z's powers stay within fp32 (the
// slope is 0 or 1 to 2^-110 from there on); min and max of NaN are NaN.
__device__ __forceinline__ float held(float z, float most) {
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(z) : "f"(most));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(z) : "f"(-most));
    return z;
}
template <int kAct>
__device__ __forceinline__ f32x2 act_grad2(float z0, float z1) {
    constexpr float l2e = 1.44269504f, most = kAct == RLM_ACT_GELU ? 9.9f : 85.f;
    const f32x2 one = 0x3f8000003f800000ull, z = pack(make_float2(held(z0, most), held(z1, most))), zz = mul2(z, z);
    float2 f = unpack(mul2(kAct == RLM_ACT_GELU ? mul2(z, fma2(zz, twice(kBend3), twice(kBend1))) : z, twice(-l2e)));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(f.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(f.y));
    const f32x2 e = pack(f);
    f = unpack(add2(e, one));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(f.x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(f.y));
    const f32x2 s = pack(f), rest = mul2(e, s);
    if (kAct == RLM_ACT_SIGMOID) return mul2(s, rest);
    const f32x2 slope = kAct == RLM_ACT_GELU ? mul2(z, fma2(zz, twice(3.0f * kBend3), twice(kBend1))) : z;
    return mul2(s, fma2(slope, rest, one));
}

// -------------------------------------------------------------------- gemm
constexpr int kBM = 128, kBK = 64;
constexpr int kEpiWarps = 16;
constexpr int kGemmThreads = (kEpiWarps + 2) * 32;
constexpr int kStageOut = 2048;                 // one epilogue warp's staging: 32 rows of 64 bytes

// kPair: two CTAs share a 256-row tile (cta_group::2): each holds its 128 rows of A and half of
// B's rows, so B is loaded once and read once for both.
template <bool kPair, int kBN>
struct GemmCfg {
    static constexpr int kRowsB = kPair ? kBN / 2 : kBN;        // rows of B in this CTA's shared memory
    static constexpr int kTileM = kPair ? 2 * kBM : kBM;
    static constexpr int kA = kBM * kBK * 2, kB = kRowsB * kBK * 2, kStage = kA + kB;
    static constexpr int kStages = (229376 - kEpiWarps * kStageOut) / kStage;
    static constexpr int kOffOut = kStages * kStage;
    static constexpr int kOffBar = kOffOut + kEpiWarps * kStageOut;
    static constexpr int kBars = 2 * kStages + 4;
    static constexpr int kOffMisc = kOffBar + kBars * 8;
    static constexpr int kSmem = kOffMisc + 16 + 1024;          // and room to align the ring
    static_assert(kSmem <= 232448, "shared memory budget");
};

struct GemmArgs {
    int M, N;                   // output rows and columns
    int tiles_m, tiles_n, splits, steps_per_split, steps;
    int whole, units;           // units that are whole tiles (of a split), and all (see unit_of())
    const float *bias;          // nullable [N]
    const bf16 *residual;       // nullable [M][ld]
    int64_t residual_ld;
    int act;
    void *out;                  // bf16, or fp32 [splits][M][ld]
    bf16 *pre;
    int64_t out_ld, pre_ld;
};

// Order of the tiles: columns of kGroup row tiles, so that the CTAs at work share operands in L2.
constexpr int kGroup = 16;
__device__ __forceinline__ void tile_of(int t, const GemmArgs &g, int &tm, int &tn) {
    const int per = kGroup * g.tiles_n, grp = t / per, first = grp * kGroup;
    const int rows = min(kGroup, g.tiles_m - first), in = t - grp * per;
    tn = in / rows;
    tm = first + in - tn * rows;
}

// Unit u of the work: a tile, or a split's share of one; of 256 columns also half a tile, where
// the last round of tiles would leave more than half the pairs idle (launch_gemm()).
struct Unit {
    int tm, split, col, half;   // row tile, split, first column, whether 128 columns in place of 256
};
template <int kBN>
__device__ __forceinline__ Unit unit_of(int u, const GemmArgs &g) {
    Unit r;
    const int past = u - g.whole;
    r.half = kBN == 256 && past >= 0;
    const int t = r.half ? g.whole + (past >> 1) : u;
    r.split = t % g.splits;
    int tn;
    tile_of(t / g.splits, g, r.tm, tn);
    r.col = tn * kBN + (r.half && (past & 1) ? 128 : 0);
    return r;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float lo16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

__device__ __forceinline__ void st_shared16(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
// Byte offset of 16-byte piece p of row r in a staging buffer: neither eight lanes of a row
// each nor those of two rows meet in a bank.
__device__ __forceinline__ uint32_t piece(int r, int p) { return r * 64 + ((p ^ ((r >> 1) & 3)) << 4); }

// What a product writes: the epilogue act(sum + bias) + residual as bf16; the raw sums as fp32
// (partial sums, or a gradient kept in fp32); or the epilogue and sum + bias, both bf16.
enum : int { kOutBf16 = 0, kOutF32 = 1, kOutPre = 2 };
template <bool kPair, bool kAMn, bool kBMn, int kBN, int kOut, int kAct>
__global__ void __launch_bounds__(kGemmThreads, 1)
    k_gemm(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
           const GemmArgs g) {
    using Cfg = GemmCfg<kPair, kBN>;
    constexpr int ST = Cfg::kStages;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const uint32_t bars = base + Cfg::kOffBar;
    const uint32_t full = bars, empty = bars + ST * 8, acc_full = bars + 2 * ST * 8, acc_empty = acc_full + 16;
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + Cfg::kOffMisc);
    uint32_t *tmem_at = reinterpret_cast<uint32_t *>(smem + Cfg::kOffMisc + 8);
    // A pair: rank 0 issues the MMAs and holds the barriers that count both CTAs' copies (full)
    // and both CTAs' readers (acc_empty); empty and acc_full are signalled in both.
    const int rank = kPair ? (int)(blockIdx.x & 1) : 0;
    const int unit0 = kPair ? blockIdx.x >> 1 : blockIdx.x, unit_step = kPair ? gridDim.x >> 1 : gridDim.x;

    if (tid == 0) {
        for (int i = 0; i < ST; ++i) {
            bar_init(full + i * 8, 1);
            bar_init(empty + i * 8, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(acc_full + i * 8, 1);
            bar_init(acc_empty + i * 8, (kPair ? 2 : 1) * kEpiWarps);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kEpiWarps) {
        tmem_alloc<kPair>(smem_u32(tmem_at), 2 * kBN);
        if (lane == 0) {
            prefetch_map(&map_a);
            prefetch_map(&map_b);
        }
    }
    fence_before();
    __syncthreads();
    if (kPair) cluster_sync();
    fence_after();
    wait_for_previous();
    const uint32_t tmem = *tmem_at;
    const int units = g.units;

    if (warp == kEpiWarps) {
        int it = 0;
        bool ok = true;
        for (int u = unit0; ok && u < units; u += unit_step) {
            const Unit unit = unit_of<kBN>(u, g);
            const int s0 = unit.split * g.steps_per_split, s1 = min(g.steps, s0 + g.steps_per_split);
            const int boxes = Cfg::kRowsB / 64 >> unit.half;            // of 64 rows of B each
            const int ra = unit.tm * Cfg::kTileM + rank * kBM, rb = unit.col + rank * boxes * 64;
            const uint32_t bytes = (kPair ? 2 : 1) * (Cfg::kA + boxes * 8192);
            for (int s = s0; s < s1; ++s, ++it) {
                const int st = it % ST;
                if (it >= ST && !(ok = wait_bar(empty + st * 8, (it / ST - 1) & 1, abort_flag, &g_linear_status))) break;
                const uint32_t a = base + st * Cfg::kStage, b = a + Cfg::kA;
                const uint32_t bar = kPair ? map_rank(full + st * 8, 0) : full + st * 8;
                if (elect()) {
                    if (rank == 0) bar_expect_tx(full + st * 8, bytes);
                    auto load = [&](uint32_t to, const CUtensorMap *map, int c0, int c1) {
                        if constexpr (kPair) tma_load_2d_pair(to, map, c0, c1, bar);
                        else tma_load_2d(to, map, c0, c1, bar);
                    };
                    if (kAMn) {
#pragma unroll
                        for (int j = 0; j < kBM / 64; ++j) load(a + j * 8192, &map_a, ra + j * 64, s * kBK);
                    } else {
                        load(a, &map_a, s * kBK, ra);
                    }
#pragma unroll
                    for (int j = 0; j < Cfg::kRowsB / 64; ++j) {
                        if (j >= boxes) break;
                        if (kBMn) load(b + j * 8192, &map_b, rb + j * 64, s * kBK);
                        else load(b + j * 8192, &map_b, s * kBK, rb + j * 64);
                    }
                }
                __syncwarp();
            }
        }
        // Copies in flight land before the CTA may end (after a timeout; otherwise they have).
        if (*abort_flag && rank == 0)
            for (int i = max(0, it - ST); i < it; ++i)
                for (int n = 0; n < 1 << 22 && !bar_try(full + (i % ST) * 8, (i / ST) & 1); ++n) {}
    } else if (warp == kEpiWarps + 1) {
        if (rank == 0) {
            constexpr uint32_t a_k = (kAMn ? 2048 : 32) >> 4, b_k = (kBMn ? 2048 : 32) >> 4;       // 16 contraction indexes on
            const uint64_t da0 = desc(base, kAMn ? 8192 : 16, 1024), db0 = desc(base + Cfg::kA, kBMn ? 8192 : 16, 1024);
            int it = 0, n = 0;
            bool ok = true;
            for (int u = unit0; ok && u < units; u += unit_step, ++n) {
                const Unit unit = unit_of<kBN>(u, g);
                const int s0 = unit.split * g.steps_per_split, s1 = min(g.steps, s0 + g.steps_per_split);
                const uint32_t id = unit.half ? idesc(Cfg::kTileM, 128, kAMn, kBMn) : idesc(Cfg::kTileM, kBN, kAMn, kBMn);
                const int buf = n & 1;
                const uint32_t d = tmem + buf * kBN;
                if (n >= 2 && !(ok = wait_bar(acc_empty + buf * 8, (n / 2 - 1) & 1, abort_flag, &g_linear_status))) break;
                fence_after();
                for (int s = s0; s < s1; ++s, ++it) {
                    const int st = it % ST;
                    if (!(ok = wait_bar(full + st * 8, (it / ST) & 1, abort_flag, &g_linear_status))) break;
                    fence_after();
                    const uint64_t da = da0 + st * (Cfg::kStage >> 4), db = db0 + st * (Cfg::kStage >> 4);
                    if (elect()) {
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k)
                            mma<kPair>(d, da + k * a_k, db + k * b_k, id, (uint32_t)(s > s0 || k > 0));
                        commit<kPair>(empty + st * 8);
                    }
                    __syncwarp();
                }
                if (elect()) commit<kPair>(acc_full + buf * 8);
                __syncwarp();
            }
        }
    } else {
        constexpr bool kF32 = kOut == kOutF32;
        constexpr int kCols = kF32 ? 16 : 32;               // output columns handled at a time, 64 bytes
        constexpr int kWarpCols = kBN / (kEpiWarps / 4);    // a warp's columns of a tile (of half a tile 32)
        const uint32_t staging = base + Cfg::kOffOut + warp * kStageOut;
        int n = 0;
        // The staged rows to memory, eight rows of 64 bytes a request; to: (row0, col), `cols` columns there.
        auto send = [&](char *to, int64_t pitch, int row0, int cols) {
            __syncwarp();
            const int p = lane & 3, r0 = lane >> 2;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + i * 8;
                const uint4 v = ld_shared16(staging + piece(r, p));
                if (row0 + r < g.M && p * (kF32 ? 4 : 8) < cols) *reinterpret_cast<uint4 *>(to + r * pitch + p * 16) = v;
            }
            __syncwarp();
        };
        auto send_bf16 = [&](const f32x2 (&z)[16], bf16 *to, int64_t ld, int row0, int cols) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack(z[4 * p + i]);
                    w[i] = pack2(f.x, f.y);
                }
                st_shared16(staging + piece(lane, p), make_uint4(w[0], w[1], w[2], w[3]));
            }
            send(reinterpret_cast<char *>(to), ld * 2, row0, cols);
        };
        for (int u = unit0; u < units; u += unit_step, ++n) {
            const Unit unit = unit_of<kBN>(u, g);
            const int cols = kWarpCols >> unit.half;
            const int row0 = unit.tm * Cfg::kTileM + rank * kBM + (warp & 3) * 32, col0 = unit.col + (warp >> 2) * cols;
            const int buf = n & 1;
            // The residual's chunk and a lane's bias, asked for ahead of the accumulator; both are handed
            // to the lanes that need them through the staging buffer.
            uint4 res[4];
            auto ask = [&](int col) {
                if constexpr (!kF32) {
                    if (!g.residual) return;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = row0 + i * 8 + (lane >> 2), cc = col + (lane & 3) * 8;
                        res[i] = r < g.M && cc < g.N
                                     ? *reinterpret_cast<const uint4 *>(g.residual + (int64_t)r * g.residual_ld + cc)
                                     : make_uint4(0, 0, 0, 0);
                    }
                }
            };
            ask(col0);
            // The next tile's into L2, a row a lane, where the products leave no time for its latency (72 ->
            // 63 us at 131072 x 256 x 512).
            if (!kF32 && g.residual && g.steps <= 16 && u + unit_step < units) {
                const Unit next = unit_of<kBN>(u + unit_step, g);
                const int r = next.tm * Cfg::kTileM + rank * kBM + (warp & 3) * 32 + lane;
                const int c = next.col + (warp >> 2) * (kWarpCols >> next.half);
                if (r < g.M && c < g.N) {
                    const bf16 *p = g.residual + (int64_t)r * g.residual_ld + c;
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
                    if (kWarpCols == 64 && c + 56 < g.N) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + 56));
                }
            }
            float bias0 = 0.f, bias1 = 0.f;
            if (!kF32 && g.bias) {
                if (col0 + lane < g.N) bias0 = g.bias[col0 + lane];
                if (kWarpCols == 64 && col0 + 32 + lane < g.N) bias1 = g.bias[col0 + 32 + lane];
            }
            if (!wait_bar(acc_full + buf * 8, (n / 2) & 1, abort_flag, &g_linear_status)) break;
            fence_after();
            const uint32_t acc = tmem + buf * kBN + (warp >> 2) * cols + ((uint32_t)(warp & 3) << 21);
#pragma unroll 1
            for (int c = 0; c < cols; c += kCols) {
                const int col = col0 + c;
                uint32_t v[kCols];
#pragma unroll
                for (int i = 0; i < kCols; i += 16) tmem_ld16(acc + c + i, v + i);
                tmem_wait_ld();
                if (c + kCols >= cols) {                    // the last read of this accumulator
                    fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (kPair) bar_arrive_cluster(map_rank(acc_empty + buf * 8, 0));
                        else bar_arrive(acc_empty + buf * 8);
                    }
                }
                if (row0 >= g.M || col >= g.N) continue;
                if constexpr (kF32) {
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        st_shared16(staging + piece(lane, p), make_uint4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]));
                    send(reinterpret_cast<char *>(static_cast<float *>(g.out) + ((int64_t)unit.split * g.M + row0) * g.out_ld + col),
                         g.out_ld * 4, row0, g.N - col);
                } else {
                    f32x2 z[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = pack(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])));
                    if (g.bias) {
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(staging + lane * 4), "f"(c == 0 ? bias0 : bias1) : "memory");
                        __syncwarp();
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const uint4 b = ld_shared16(staging + q * 16);
                            z[2 * q] = add2(z[2 * q], pack(make_float2(__uint_as_float(b.x), __uint_as_float(b.y))));
                            z[2 * q + 1] = add2(z[2 * q + 1], pack(make_float2(__uint_as_float(b.z), __uint_as_float(b.w))));
                        }
                        __syncwarp();
                    }
                    if constexpr (kOut == kOutPre) send_bf16(z, g.pre + (int64_t)row0 * g.pre_ld + col, g.pre_ld, row0, g.N - col);
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = act2<kAct>(z[i]);
                    if (g.residual) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) st_shared16(staging + piece(i * 8 + (lane >> 2), lane & 3), res[i]);
                        __syncwarp();
                        if (c + kCols < cols) ask(col + kCols);
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            const uint4 r = ld_shared16(staging + piece(lane, p));
                            z[4 * p] = add2(z[4 * p], pack(make_float2(lo16(r.x), hi16(r.x))));
                            z[4 * p + 1] = add2(z[4 * p + 1], pack(make_float2(lo16(r.y), hi16(r.y))));
                            z[4 * p + 2] = add2(z[4 * p + 2], pack(make_float2(lo16(r.z), hi16(r.z))));
                            z[4 * p + 3] = add2(z[4 * p + 3], pack(make_float2(lo16(r.w), hi16(r.w))));
                        }
                        __syncwarp();
                    }
                    send_bf16(z, static_cast<bf16 *>(g.out) + (int64_t)row0 * g.out_ld + col, g.out_ld, row0, g.N - col);
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    if (kPair) cluster_sync();                      // neither CTA leaves while the other may still signal it
    if (warp == kEpiWarps) tmem_free<kPair>(tmem, 2 * kBN);
}

// ---------------------------------------------------------------- few rows
// R <= 8 kTok rows (serving): bound by reading w once.  A 128-row tile would do 128 / R
// times the work on too few CTAs, so here 16 rows of w are a CTA's: w is the 16-row
// operand of mma.sync (m16n8k16), tokens its 8 columns.  The warps share the contraction
// in 32-long blocks.  The order of the products within a block is free as long as both
// operands agree, so a lane takes 8 consecutive k of its rows by one 16-byte load from
// global memory, straight into the fragments: no shared memory, no shuffles.  The warps'
// sums are added in order in shared memory.
struct FewArgs {
    const bf16 *x, *w, *residual;
    const float *bias;
    bf16 *y, *pre;
    int64_t x_ld, w_ld, residual_ld, y_ld, pre_ld;
    int R, N, K, act;
};
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int kTok, int kWarps>
__global__ void __launch_bounds__(kWarps * 32) k_few(const FewArgs a) {
    __shared__ float part[kWarps][16][8 * kTok + 1];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int n0 = blockIdx.x * 16;
    const bf16 *w0 = a.w + (int64_t)min(n0 + g, a.N - 1) * a.w_ld + q * 8;
    const bf16 *w8 = a.w + (int64_t)min(n0 + 8 + g, a.N - 1) * a.w_ld + q * 8;
    const bf16 *xp[kTok];
#pragma unroll
    for (int i = 0; i < kTok; ++i) xp[i] = a.x + (int64_t)min(i * 8 + g, a.R - 1) * a.x_ld + q * 8;
    float d[kTok][4] = {};
    constexpr int kDeep = kTok > 2 ? 2 : 4;         // blocks in flight
    // They follow one another in w's rows where that leaves no warp without a share (from HBM, us,
    // kWarps blocks apart / one after the other: 8 rows, K = N = 4096 8.0 / 7.5, 4096 x 11008 17.0 /
    // 16.4; 16 rows, 4096 x 4096 10.4 / 9.1; but 8 rows, 1024 x 1024 2.4 / 3.0).
    const int apart = a.K >= kDeep * kWarps * 32 ? 32 : kWarps * 32;
    auto blocks = [&](int k, auto whole) {
        uint4 w[kDeep][2], x[kDeep][kTok];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const int at = k + u * apart;
            const bool ok = decltype(whole)::value || at + q * 8 < a.K;
            w[u][0] = ok ? load_once(w0 + at) : make_uint4(0, 0, 0, 0);
            w[u][1] = ok ? load_once(w8 + at) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < kTok; ++i)
                x[u][i] = ok ? *reinterpret_cast<const uint4 *>(xp[i] + at) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                mma16816(d[t], w[u][0].x, w[u][1].x, w[u][0].y, w[u][1].y, x[u][t].x, x[u][t].y);
                mma16816(d[t], w[u][0].z, w[u][1].z, w[u][0].w, w[u][1].w, x[u][t].z, x[u][t].w);
            }
    };
    int k = warp * (apart == 32 ? kDeep * 32 : 32);
    for (; k + (kDeep - 1) * apart + 32 <= a.K; k += kDeep * kWarps * 32) blocks(k, std::true_type{});
    if (k < a.K) blocks(k, std::false_type{});
#pragma unroll
    for (int t = 0; t < kTok; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[warp][(i >> 1) * 8 + g][t * 8 + q * 2 + (i & 1)] = d[t][i];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * 8 * kTok; i += kWarps * 32) {
        const int n = i % 16, t = i / 16, col = n0 + n;
        if (t >= a.R || col >= a.N) continue;
        float z = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) z += part[w][n][t];
        if (a.bias) z += a.bias[col];
        if (a.pre) a.pre[t * a.pre_ld + col] = __float2bfloat16_rn(z);
        z = act_of(a.act, z);
        if (a.residual) z += __bfloat162float(a.residual[t * a.residual_ld + col]);
        a.y[t * a.y_ld + col] = __float2bfloat16_rn(z);
    }
}

// ------------------------------------------------- sums of split products
// part [splits][M][N] fp32, added in order, then the epilogue; a thread per 4 columns.
struct FinishArgs {
    const float *part;
    int64_t M;
    int N, splits, act, out_f32;
    const float *bias;
    const bf16 *residual;
    int64_t residual_ld, out_ld, pre_ld;
    void *out;
    bf16 *pre;
};
__global__ void __launch_bounds__(256) k_finish(const FinishArgs f) {
    wait_for_previous();
    const int64_t q = f.N / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= f.M * q) return;
    const int64_t row = i / q;
    const int col = (int)(i - row * q) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < f.splits; ++k) {
        const float4 v = *reinterpret_cast<const float4 *>(f.part + ((int64_t)k * f.M + row) * f.N + col);
        s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    if (f.out_f32) {
        *reinterpret_cast<float4 *>(static_cast<float *>(f.out) + row * f.out_ld + col) = s;
        return;
    }
    if (f.bias) {
        const float4 b = *reinterpret_cast<const float4 *>(f.bias + col);
        s.x += b.x, s.y += b.y, s.z += b.z, s.w += b.w;
    }
    if (f.pre) *reinterpret_cast<uint2 *>(f.pre + row * f.pre_ld + col) = make_uint2(pack2(s.x, s.y), pack2(s.z, s.w));
    s.x = act_of(f.act, s.x), s.y = act_of(f.act, s.y), s.z = act_of(f.act, s.z), s.w = act_of(f.act, s.w);
    if (f.residual) {
        const uint2 r = *reinterpret_cast<const uint2 *>(f.residual + row * f.residual_ld + col);
        s.x += lo16(r.x), s.y += hi16(r.x), s.z += lo16(r.y), s.w += hi16(r.y);
    }
    *reinterpret_cast<uint2 *>(static_cast<bf16 *>(f.out) + row * f.out_ld + col) = make_uint2(pack2(s.x, s.y), pack2(s.z, s.w));
}

// --------------------------------------------- dz = dy act'(z), and dbias
// Blocks of 128 rows (fewer where that leaves SMs idle) by 256 columns (fewer where N is
// less, and more rows at a time), a thread per 8 columns.  Bound by its 6 bytes an element (2
// without an activation).  The block's column sums go to
// `part` [row blocks][N], which k_column_sum adds in order.
struct DzArgs {
    const bf16 *dy, *pre;
    bf16 *dz;               // (unused without an activation: dy serves)
    float *part;            // nullable (no dbias)
    int64_t R, dy_ld, pre_ld;
    int N, rows, log2_groups;       // rows of a block; column groups of 8 in a block, at most 32
};
template <int kAct>
__global__ void __launch_bounds__(256) k_dz(const DzArgs a) {
    __shared__ float sums[256 * 8];             // [rows at a time][columns]
    wait_for_previous();
    const int groups = 1 << a.log2_groups, cg = threadIdx.x & (groups - 1), rl = threadIdx.x >> a.log2_groups;
    const int at_once = 256 >> a.log2_groups, cols = groups * 8;
    const int col = blockIdx.y * 256 + cg * 8;
    const int64_t r0 = (int64_t)blockIdx.x * a.rows, r1 = min(a.R, r0 + a.rows);
    f32x2 s[4] = {0, 0, 0, 0};
    if (col < a.N) {
        // Eight rows' loads ahead of their stores, which the compiler may not reorder (dz of 16387 x
        // 2048 with its column sums 42 -> 34 us); without stores, a row at a time and more blocks per
        // SM (131072 x 512: 25.5 us against 32.6 with four).
        constexpr int kDeep = kAct == RLM_ACT_NONE ? 1 : 8;
        for (int64_t r = r0 + rl; r < r1; r += kDeep * at_once) {
            uint4 d[kDeep], p[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const int64_t row = min(r + u * at_once, r1 - 1);
                d[u] = load_once(a.dy + row * a.dy_ld + col);
                if constexpr (kAct != RLM_ACT_NONE) p[u] = load_once(a.pre + row * a.pre_ld + col);
            }
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const int64_t row = r + u * at_once;
                if (row >= r1) break;
                const uint32_t dw[4] = {d[u].x, d[u].y, d[u].z, d[u].w};
                f32x2 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = pack(make_float2(lo16(dw[i]), hi16(dw[i])));
                if constexpr (kAct != RLM_ACT_NONE) {
                    const uint32_t pw[4] = {p[u].x, p[u].y, p[u].z, p[u].w};
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] = mul2(v[i], act_grad2<kAct>(lo16(pw[i]), hi16(pw[i])));
                        const float2 f = unpack(v[i]);
                        w[i] = pack2(f.x, f.y);
                    }
                    *reinterpret_cast<uint4 *>(a.dz + row * a.N + col) = make_uint4(w[0], w[1], w[2], w[3]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = add2(s[i], v[i]);
            }
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float2 *>(&sums[rl * cols + cg * 8 + 2 * i]) = unpack(s[i]);
    __syncthreads();
    const int c = blockIdx.y * 256 + threadIdx.x;
    if ((int)threadIdx.x < cols && c < a.N) {
        float t = 0.f;
        for (int w = 0; w < at_once; ++w) t += sums[w * cols + threadIdx.x];
        a.part[(int64_t)blockIdx.x * a.N + c] = t;
    }
}
// Column sums of part [n][N]: 32 columns a block, 32 row strides, then a fixed-order sum.
__global__ void __launch_bounds__(1024) k_column_sum(const float *part, int64_t n, int N, float *out) {
    __shared__ float sums[32][33];
    wait_for_previous();
    const int c = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    float s = 0.f;
    if (col < N) {
#pragma unroll 8
        for (int64_t r = w; r < n; r += 32) s += part[r * N + col];
    }
    sums[w][c] = s;
    __syncthreads();
    if (w == 0 && col < N) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sums[i][c];
        out[col] = t;
    }
}

// ---------------------------------------------------------------- host side
using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
    static EncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeFn>(p);
    });
    return fn;
}

// An operand: rows of `inner` contiguous bf16, `outer` of them, ld apart; boxes of 64 x box_rows.
bool operand_map(CUtensorMap *map, const void *ptr, int64_t inner, int64_t outer, int64_t ld, int box_rows) {
    EncodeFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
    cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    cuuint32_t one[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(ptr), dims, strides, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
struct GemmPlan {
    bool pair;
    int bn, splits, steps_per_split, steps, tiles_m, tiles_n;
};

// Tile and splits, by time in microseconds: a launch, then rounds of units, each its steps or
// (for short contractions) its epilogue, which the next unit's steps overlap; no less than the
// operands' bytes take; for splits a second launch and the partial sums' bytes through L2.  Measured
// on 512 to 131072 rows, K and N of 64 to 8192; the choices it makes are within 10 % of the best.
struct TileKind {
    bool pair;
    int bn;
    double launch, step, epilogue;
};
constexpr TileKind kTiles[] = {{true, 256, 5.7, 0.285, 1.9}, {true, 128, 5.1, 0.17, 1.2}, {false, 128, 4.0, 0.19, 1.0}};

// Tiles of 256 x 256 whose halves are units of their own: those of the last round, where their
// halves fit into one.  (4096 x 4096 x 4096: 256 tiles on 76 pairs, three rounds and a half in
// place of four.)
int64_t halved(int64_t tiles, int64_t slots) {
    const int64_t last = tiles % slots;
    return tiles > slots && 2 * last <= slots ? last : 0;
}

GemmPlan find_plan(int64_t M, int64_t N, int64_t K) {
    GemmPlan best = {};
    double best_cost = 0;
    const int sms = sm_count();
    for (const TileKind &t : kTiles) {
        const int64_t tm = (M + (t.pair ? 255 : 127)) / (t.pair ? 256 : 128), tn = (N + t.bn - 1) / t.bn;
        const int64_t slots = t.pair ? sms / 2 : sms;
        const int steps = (int)((K + kBK - 1) / kBK);
        for (int splits = 1; splits <= 64 && splits <= steps; ++splits) {
            const int per = (steps + splits - 1) / splits;
            if ((steps + per - 1) / per != splits) continue;
            if (splits > 1 && tm * tn * splits > slots) break;      // more work units than SMs: nothing to fill
            const bool halves = t.bn == 256 && splits == 1 && halved(tm * tn, slots) > 0;
            const int64_t rounds = (tm * tn * splits + slots - 1) / slots - halves;
            // Bytes from memory, and from L2: every unit's operands, at 20 TB/s beside the output.
            const double out = 2.0 * M * N, bytes = 2.0 * ((double)M * K + (double)N * K) + out;
            const double l2 = (double)(tm * tn) * steps * kBK * 2.0 * ((t.pair ? 256 : 128) + t.bn);
            double work = (double)rounds * std::max(per * t.step, t.epilogue);
            if (halves) work += std::max(per * kTiles[1].step, kTiles[1].epilogue);
            double cost = t.launch + std::max({work, bytes / 6.0e6, l2 / 20.0e6 + out / 8.0e6});
            if (splits > 1) cost += 3.0 + 8.0 * splits * (double)M * N / 8.0e6;
            if (best_cost == 0 || cost < best_cost) {
                best_cost = cost;
                best = {t.pair, t.bn, splits, per, steps, (int)tm, (int)tn};
            }
        }
    }
    return best;
}

// A program's few shapes come again and again: their plans are kept (they depend on the shape and
// the device's SM count alone).
GemmPlan gemm_plan(int64_t M, int64_t N, int64_t K) {
    struct Kept {
        int64_t M, N, K;
        int sms;
        GemmPlan plan;
    };
    static thread_local Kept kept[32] = {};
    const int sms = sm_count();
    Kept &k = kept[(unsigned)(M * 31 + N * 17 + K / 8 * 5 + M / 64) % 32];
    if (k.M != M || k.N != N || k.K != K || k.sms != sms) k = {M, N, K, sms, find_plan(M, N, K)};
    return k.plan;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t gemm_ws(const GemmPlan &p, int64_t M, int64_t N) {
    return p.splits > 1 ? round256((size_t)p.splits * M * N * sizeof(float)) : 0;
}

struct Operand {
    const void *ptr;
    int64_t ld;
};
struct Epilogue {
    const float *bias = nullptr;
    const bf16 *residual = nullptr;
    int64_t residual_ld = 0;
    int act = RLM_ACT_NONE;
    void *out = nullptr;
    int64_t out_ld = 0;
    bool out_f32 = false;
    void *pre = nullptr;
    int64_t pre_ld = 0;
};

template <bool kPair, bool kAMn, bool kBMn, int kBN, int kOut, int kAct>
cudaError_t launch_gemm(const CUtensorMap &ma, const CUtensorMap &mb, GemmArgs g, cudaStream_t st) {
    using Cfg = GemmCfg<kPair, kBN>;
    auto *fn = k_gemm<kPair, kAMn, kBMn, kBN, kOut, kAct>;
    static std::atomic<int> ctas[64];               // per device: CTAs that fit, once the kernel is set up
    int dev = 0;
    cudaGetDevice(&dev);
    int room = ctas[dev & 63].load(std::memory_order_relaxed);
    if (room == 0) {
        cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
        if (e != cudaSuccess) return e;
        room = sm_count();
        if (kPair) {
            // Pairs sit in one GPC: an odd SM of a GPC stays out.
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(2);
            cfg.blockDim = dim3(kGemmThreads);
            cfg.dynamicSmemBytes = Cfg::kSmem;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = 2;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            int n = 0;
            if ((e = cudaOccupancyMaxActiveClusters(&n, fn, &cfg)) != cudaSuccess) return e;
            room = 2 * std::max(n, 1);
        }
        ctas[dev & 63].store(room, std::memory_order_relaxed);
    }
    g_linear_waits.store(true, std::memory_order_relaxed);
    constexpr int kCtas = kPair ? 2 : 1;
    g.whole = g.units = g.tiles_m * g.tiles_n * g.splits;
    if (kBN == 256 && g.splits == 1) {
        const int last = halved(g.units, room / kCtas);
        g.whole -= last;
        g.units += last;
    }
    return launch_dependent(fn, dim3((unsigned)std::min<int64_t>((int64_t)g.units * kCtas, room)), kGemmThreads, Cfg::kSmem, st,
                            kCtas, ma, mb, g);
}

template <bool kPair, bool kAMn, bool kBMn, int kBN>
cudaError_t pick_gemm(const CUtensorMap &ma, const CUtensorMap &mb, const GemmArgs &g, int out, cudaStream_t st) {
    if (out == kOutF32) return launch_gemm<kPair, kAMn, kBMn, kBN, kOutF32, RLM_ACT_NONE>(ma, mb, g, st);
    if constexpr (!kAMn && !kBMn) {         // only the forward product has an activation, or keeps z
        switch (g.act * 2 + (out == kOutPre)) {
            case RLM_ACT_NONE * 2 + 1: return launch_gemm<kPair, kAMn, kBMn, kBN, kOutPre, RLM_ACT_NONE>(ma, mb, g, st);
            case RLM_ACT_SILU * 2: return launch_gemm<kPair, kAMn, kBMn, kBN, kOutBf16, RLM_ACT_SILU>(ma, mb, g, st);
            case RLM_ACT_SILU * 2 + 1: return launch_gemm<kPair, kAMn, kBMn, kBN, kOutPre, RLM_ACT_SILU>(ma, mb, g, st);
            case RLM_ACT_GELU * 2: return launch_gemm<kPair, kAMn, kBMn, kBN, kOutBf16, RLM_ACT_GELU>(ma, mb, g, st);
            case RLM_ACT_GELU * 2 + 1: return launch_gemm<kPair, kAMn, kBMn, kBN, kOutPre, RLM_ACT_GELU>(ma, mb, g, st);
            case RLM_ACT_SIGMOID * 2:
                return launch_gemm<kPair, kAMn, kBMn, kBN, kOutBf16, RLM_ACT_SIGMOID>(ma, mb, g, st);
            case RLM_ACT_SIGMOID * 2 + 1:
                return launch_gemm<kPair, kAMn, kBMn, kBN, kOutPre, RLM_ACT_SIGMOID>(ma, mb, g, st);
            default: break;
        }
    }
    return launch_gemm<kPair, kAMn, kBMn, kBN, kOutBf16, RLM_ACT_NONE>(ma, mb, g, st);
}

template <bool kAMn, bool kBMn>
cudaError_t gemm(Operand a, Operand b, int64_t M, int64_t N, int64_t K, const Epilogue &ep, float *part, cudaStream_t st) {
    const GemmPlan p = gemm_plan(M, N, K);
    CUtensorMap ma, mb;
    if (!(kAMn ? operand_map(&ma, a.ptr, M, K, a.ld, 64) : operand_map(&ma, a.ptr, K, M, a.ld, kBM)) ||
        !(kBMn ? operand_map(&mb, b.ptr, N, K, b.ld, 64) : operand_map(&mb, b.ptr, K, N, b.ld, 64)))
        return cudaErrorInvalidValue;
    const bool split = p.splits > 1;
    const int out = split || ep.out_f32 ? kOutF32 : ep.pre ? kOutPre : kOutBf16;
    GemmArgs g = {};
    g.M = (int)M, g.N = (int)N;
    g.tiles_m = p.tiles_m, g.tiles_n = p.tiles_n;
    g.splits = p.splits, g.steps_per_split = p.steps_per_split, g.steps = p.steps;
    g.out = split ? part : ep.out;
    g.out_ld = split ? N : ep.out_ld;
    if (!split) {
        g.pre = static_cast<bf16 *>(ep.pre);
        g.pre_ld = ep.pre_ld;
        g.bias = ep.bias;
        g.residual = ep.residual;
        g.residual_ld = ep.residual_ld;
        g.act = ep.act;
    }
    const cudaError_t e = !p.pair        ? pick_gemm<false, kAMn, kBMn, 128>(ma, mb, g, out, st)
                          : p.bn == 256 ? pick_gemm<true, kAMn, kBMn, 256>(ma, mb, g, out, st)
                                        : pick_gemm<true, kAMn, kBMn, 128>(ma, mb, g, out, st);
    if (e != cudaSuccess || !split) return e;
    FinishArgs f = {};
    f.part = part;
    f.M = M;
    f.N = (int)N;
    f.splits = p.splits;
    f.act = ep.act;
    f.out_f32 = ep.out_f32;
    f.bias = ep.bias;
    f.residual = ep.residual;
    f.residual_ld = ep.residual_ld;
    f.out = ep.out;
    f.out_ld = ep.out_ld;
    f.pre = static_cast<bf16 *>(ep.pre);
    f.pre_ld = ep.pre_ld;
    return launch_dependent(k_finish, dim3((unsigned)((M * (N / 4) + 255) / 256)), 256, 0, st, 1, f);
}

}  // namespace

// Whether k_few serves a product: always up to 8 rows; from there its reads of x grow with the
// rows while the tiles' cost does not (us, from HBM, k_few / tiles): 16 rows, K x N = 4096 x 4096
// 8.8 / 10.8, 8192 x 1024 10.1 / 8.8, 4096 x 11008 22 / 19; 32 rows, 1024 x 1024 3.4 / 5.4,
// 2048 x 2048 5.2 / 6.7, 2048 x 4096 9.1 / 8.7, 512 x 16384 10.0 / 6.3.
bool few_rows(int64_t R, int64_t K, int64_t N) {
    if (R <= 8) return true;
    if (R <= 16) return K <= 4096 && K * N <= 24 << 20;
    return R <= 32 && K <= 2048 && K * N <= 4 << 20;
}

template <int kTok>
cudaError_t launch_few(const FewArgs &a, cudaStream_t st) {
    // Sixteen warps share the contraction, eight where there are three CTAs and more for each SM:
    // 7.5 against 10.0 us (K = N = 4096, 8 rows), 18.6 against 17.0 us (K = 4096, N = 11008).
    const unsigned ctas = (unsigned)((a.N + 15) / 16);
    if (ctas >= 3u * (unsigned)sm_count())
        return launch_dependent(k_few<kTok, 8>, dim3(ctas), 8 * 32, 0, st, 1, a);
    return launch_dependent(k_few<kTok, 16>, dim3(ctas), 16 * 32, 0, st, 1, a);
}

size_t linear_ws_bytes(int64_t R, int64_t K, int64_t N) {
    return few_rows(R, K, N) ? 0 : gemm_ws(gemm_plan(R, N, K), R, N);
}

namespace {
int dz_rows(int64_t R, int64_t N) {
    int rows = 128;
    if (R <= 64) return rows;               // one block of rows: its sums are dbias, without a second kernel
    while (rows > 16 && ((R + rows - 1) / rows) * ((N + 255) / 256) < 8 * sm_count()) rows /= 2;
    return rows;
}
}  // namespace

size_t linear_backward_ws_bytes(int64_t R, int64_t K, int64_t N, int act) {
    const size_t dz = act == RLM_ACT_NONE ? 0 : round256((size_t)R * N * 2);
    const int rows = dz_rows(R, N);
    const size_t sums = round256((size_t)((R + rows - 1) / rows) * N * sizeof(float));
    return dz + sums + std::max(gemm_ws(gemm_plan(R, K, N), R, K), gemm_ws(gemm_plan(N, K, R), N, K));
}

cudaError_t linear_forward(const rlm_matrix &x, const rlm_matrix &w, const float *bias, int act_kind,
                           const rlm_matrix *residual, const rlm_matrix *pre, const rlm_matrix &y, void *ws,
                           cudaStream_t st) {
    if (few_rows(x.rows, x.cols, w.rows)) {
        FewArgs a = {};
        a.x = static_cast<const bf16 *>(x.ptr), a.x_ld = x.ld;
        a.w = static_cast<const bf16 *>(w.ptr), a.w_ld = w.ld;
        a.y = static_cast<bf16 *>(y.ptr), a.y_ld = y.ld;
        if (residual) a.residual = static_cast<const bf16 *>(residual->ptr), a.residual_ld = residual->ld;
        if (pre) a.pre = static_cast<bf16 *>(pre->ptr), a.pre_ld = pre->ld;
        a.bias = bias;
        a.R = (int)x.rows, a.N = (int)w.rows, a.K = (int)x.cols;
        a.act = act_kind;
        return a.R <= 8 ? launch_few<1>(a, st) : a.R <= 16 ? launch_few<2>(a, st) : launch_few<4>(a, st);
    }
    Epilogue ep;
    ep.bias = bias;
    ep.act = act_kind;
    if (residual) {
        ep.residual = static_cast<const bf16 *>(residual->ptr);
        ep.residual_ld = residual->ld;
    }
    if (pre) {
        ep.pre = pre->ptr;
        ep.pre_ld = pre->ld;
    }
    ep.out = y.ptr;
    ep.out_ld = y.ld;
    return gemm<false, false>({x.ptr, x.ld}, {w.ptr, w.ld}, x.rows, w.rows, x.cols, ep, static_cast<float *>(ws), st);
}

cudaError_t linear_backward(const rlm_matrix &dy, const rlm_matrix &x, const rlm_matrix &w, const rlm_matrix *pre,
                            int act_kind, const rlm_matrix *dx, const rlm_matrix *dw, float *dbias, void *ws,
                            cudaStream_t st) {
    const int64_t R = x.rows, K = x.cols, N = w.rows;
    char *at = static_cast<char *>(ws);
    Operand dz = {dy.ptr, dy.ld};
    const int rows = dz_rows(R, N);
    const int64_t blocks = (R + rows - 1) / rows;
    const float *sums = nullptr;
    if (act_kind != RLM_ACT_NONE || dbias) {
        DzArgs a = {};
        a.dy = static_cast<const bf16 *>(dy.ptr);
        a.dy_ld = dy.ld;
        a.R = R;
        a.N = (int)N;
        a.rows = rows;
        while (a.log2_groups < 5 && (8 << a.log2_groups) < N) ++a.log2_groups;
        if (act_kind != RLM_ACT_NONE) {
            a.pre = static_cast<const bf16 *>(pre->ptr);
            a.pre_ld = pre->ld;
            a.dz = reinterpret_cast<bf16 *>(at);
            at += round256((size_t)R * N * 2);
            dz = {a.dz, N};
        }
        if (dbias) sums = a.part = blocks > 1 ? reinterpret_cast<float *>(at) : dbias;
        at += round256((size_t)blocks * N * sizeof(float));
        auto *fn = act_kind == RLM_ACT_SILU      ? k_dz<RLM_ACT_SILU>
                   : act_kind == RLM_ACT_GELU    ? k_dz<RLM_ACT_GELU>
                   : act_kind == RLM_ACT_SIGMOID ? k_dz<RLM_ACT_SIGMOID>
                                                 : k_dz<RLM_ACT_NONE>;
        const cudaError_t e = launch_dependent(fn, dim3((unsigned)blocks, (unsigned)((N + 255) / 256)), 256, 0, st, 1, a);
        if (e != cudaSuccess) return e;
    }
    float *part = reinterpret_cast<float *>(at);
    if (dx) {
        Epilogue ep;
        ep.out = dx->ptr;
        ep.out_ld = dx->ld;
        const cudaError_t e = gemm<false, true>(dz, {w.ptr, w.ld}, R, K, N, ep, part, st);
        if (e != cudaSuccess) return e;
    }
    if (dw) {
        Epilogue ep;
        ep.out = dw->ptr;
        ep.out_ld = dw->ld;
        ep.out_f32 = dw->dtype == RLM_F32;
        const cudaError_t e = gemm<true, true>(dz, {x.ptr, x.ld}, N, K, R, ep, part, st);
        if (e != cudaSuccess) return e;
    }
    // Last: ahead of the products its few large blocks would hold up the first of them.
    if (dbias && blocks > 1)
        return launch_dependent(k_column_sum, dim3((unsigned)((N + 31) / 32)), 1024, 0, st, 1, sums, blocks, (int)N,
                                dbias);
    return cudaSuccess;
}

cudaError_t read_and_clear_linear_status(int *status, cudaStream_t st) {
    *status = RLM_OK;
    if (!g_linear_waits.load(std::memory_order_relaxed)) return cudaSuccess;
    cudaError_t e = cudaMemcpyFromSymbolAsync(status, g_linear_status, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
    if (e != cudaSuccess) return e;
    if ((e = cudaStreamSynchronize(st)) != cudaSuccess) return e;
    if (*status == RLM_OK) return cudaSuccess;
    const int zero = 0;
    if ((e = cudaMemcpyToSymbolAsync(g_linear_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, st)) != cudaSuccess)
        return e;
    return cudaStreamSynchronize(st);
}

}  // namespace rlm
