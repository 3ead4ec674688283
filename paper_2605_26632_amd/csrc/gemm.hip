// Launches of the linears: which tiles an output is cut into, and the kernels around the tile loop of gemm_tile.h.
#include <mutex>
#include <type_traits>
#include <vector>
#include "gemm_tile.h"
#include "tensor_factor.h"

namespace rtl {
namespace {

// Stages of a contraction: 128-byte rows of W.
__host__ __device__ inline int64_t k_blocks(int64_t K, bool fp8, bool fp4) { return fp4 ? (K + 255) / 256 : fp8 ? K / 128 : K / 64; }

// Two tile shapes in one launch (the "block-parallel" balancing of the method section's kernel
// paragraph, done with tile shapes instead of split contractions): rows [0, m_split) of the output
// are cut into 256 x BN body tiles, rows [m_split, M) into 256 x 128 tail tiles. Uniform tiles
// leave the chip's last round of workgroups mostly empty for many layer shapes (e.g. 792 tiles on
// 256 compute units: 3.09 rounds cost 4); smaller tiles at the end fill that round at 0.6 of a
// body tile's time. Every XCD works through its share of the body tiles first, then its share of
// the tail tiles (workgroups are dispatched in id order). tail_tiles == 0: a plain one-shape launch.
constexpr int kTailBN = 128;
// Waves and ring of the 256 x 128 tail tile. Sparse: as the body. Dense: a ring of three (144 KB), where the body has room for two:
// with two, a stage is requested only when the one before it has landed, and a plan of tail tiles alone (the operands arrive
// more slowly than they are used) waits for every stage in full. 64 x 64 per wave instead of 128 x 32, because the columns'
// fragments are refilled behind one row block's instructions and two of them are too few to hide it. us: [2967, 2624, 7936] 149.0 -> 111.9
// (128 x 32 112.7), [3900, 2040, 3072] 62.5 -> 47.5 (48.2), [2967, 2624, 1024] 20.2 -> 18.8 (19.5), [6468, 2848, 5056] 203.1 -> 174.3.
template <bool SPARSE>
struct Tail {
    static constexpr int kWavesM = SPARSE ? 2 : 4, kWavesN = SPARSE ? 4 : 2;
    static constexpr int stages(int body) { return SPARSE ? body : 3; }
};
template <bool SPARSE, int BN, int WAVES_M, int WAVES_N, int STAGES, int MODE, bool FP8, bool PIN, bool FP4>
__global__ __launch_bounds__(512) void gemm_mixed_kernel(const GemmArgs a) {
    static_assert(WAVES_M * WAVES_N == 8, "both tile shapes run with eight waves");
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8;
    const int nb = a.body_tiles, nt = a.tail_tiles;
    const int nb_x = nb / 8 + (xcd < nb % 8);
    if (local < nb_x) {
        GemmArgs b = a;
        if (nt > 0) b.M = a.m_split;
        gemm_tile<SPARSE, 256, BN, WAVES_M, WAVES_N, STAGES, MODE, FP8, 1, false, false, PIN, FP4>(b, xcd_share_start(nb, xcd) + local);
    } else {
        // the tail region as a problem of its own: same operands, shifted by m_split rows
        constexpr int ESZ = FP8 || FP4 ? 1 : 2;
        GemmArgs t = a;
        t.M = a.M - a.m_split;
        t.A = static_cast<const uint8_t*>(a.A) + (SPARSE ? a.m_split * 64 : a.m_split * a.lda * ESZ);
        if constexpr (SPARSE) t.meta = a.meta + a.m_split * (FP8 ? 16 : 8);
        t.Y = a.Y + a.m_split * a.ldy;
        if (a.row_scale) t.row_scale = a.row_scale + a.m_split;
        if constexpr (MODE == 1) t.T = a.T + a.m_split * kLoraRank;
        if constexpr (FP4) t.a_scale = a.a_scale + a.m_split * 8;
        const int idx = xcd_share_start(nb + nt, xcd) - xcd_share_start(nb, xcd) + (local - nb_x);
        gemm_tile<SPARSE, 256, kTailBN, Tail<SPARSE>::kWavesM, Tail<SPARSE>::kWavesN, Tail<SPARSE>::stages(STAGES), MODE, FP8, 1, false, false,
                  PIN, FP4>(t, idx);
    }
}

// The tile loops need more dynamic LDS than the default limit of a launch: the limit is raised once
// per kernel by the prepare functions (called for every configuration from prepare_gemm_kernels, i.e.
// from rtl_init or from the first entry-point call on a device), never from a launch, so that launches
// consist of the kernel node only and can be recorded into a HIP graph.
template <bool SPARSE, int BN, int WAVES_M, int WAVES_N, int STAGES, int MODE = 0, bool FP8 = false, bool PIN = !FP8, bool FP4 = false>
struct Mixed {
    using LB = Smem<SPARSE, 256, BN, STAGES, WAVES_M, WAVES_N, FP8, 1, FP4>;
    using LT = Smem<SPARSE, 256, kTailBN, Tail<SPARSE>::stages(STAGES), Tail<SPARSE>::kWavesM, Tail<SPARSE>::kWavesN, FP8, 1, FP4>;
    static constexpr int kLds = LB::kTotal > LT::kTotal ? LB::kTotal : LT::kTotal;
    static hipError_t prepare() {
        auto kern = gemm_mixed_kernel<SPARSE, BN, WAVES_M, WAVES_N, STAGES, MODE, FP8, PIN, FP4>;
        return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    }
    // a.m_split, a.body_tiles and a.tail_tiles come from the planner
    static hipError_t launch(const GemmArgs& a, hipStream_t stream) {
        auto kern = gemm_mixed_kernel<SPARSE, BN, WAVES_M, WAVES_N, STAGES, MODE, FP8, PIN, FP4>;
        hipLaunchKernelGGL(kern, dim3((unsigned)(a.body_tiles + a.tail_tiles)), dim3(512), kLds, stream, a);
        return hipGetLastError();
    }
};

// One tile shape per launch, for problems that leave the chip idle with the 256-row tiles above: few tokens
// (the text stream, short prompts, small images) or narrow layers. Those are bound by the chain of stages:
// a compute unit pulls about 95 GB/s of operands that miss its L2 (64 KB in flight over the 0.7 us a stage
// takes to arrive), whatever its waves do, so a call ends sooner the more units pull and the fewer bytes each
// of them has to. Small tiles give more units a part, and inside a tile the waves split the contraction
// (WAVES_K groups, a block each per stage), which keeps all of LDS in flight without more waves per block.
// Whole calls, [M, N, K], 256-row tiles -> these (us, GROUP scope with bias, graph replay):
//   sparse  [37, 3072, 12288] 73 -> 22, [256, 512, 512] 11.0 -> 7.3, [512, 3072, 3072] 26.9 -> 18.2,
//           [512, 3072, 12288] 77 -> 46, [1024, 3072, 3072] 29.8 -> 25.5
//   dense   [37, 3072, 12288] 129 -> 20, [333, 3072, 12288] 142 -> 52, [1024, 3072, 3072] 42 -> 24
template <bool SPARSE, int BM, int BN, int WAVES_M, int WAVES_N, int WAVES_K, int STAGES, int MODE = 0, bool FP8 = false, bool FP4 = false>
__global__ __launch_bounds__(WAVES_M * WAVES_N * WAVES_K * 64) void gemm_split_kernel(const GemmArgs a) {
    const int total = (int)(((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN));
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8;
    GemmArgs b = a;
    if constexpr (SPARSE) {
        if (a.rowsums) {
            // TENSOR scope: every workgroup adds the rows' sums up for itself (a few KB from L2, 1 to 2 us), which
            // spares the launch that would do only this (4.7 us and the gap before it)
            const float sc = tensor_factor(a.rowsums, a.M, a.factor_eps);
            b.folded = a.factor_mul ? a.factor_mul[0] * sc : sc;
            if (blockIdx.x == 0 && threadIdx.x == 0) {
                a.factor_out[0] = sc;
                if (a.factor_fused) a.factor_fused[0] = b.folded;
            }
        }
    }
    gemm_tile<SPARSE, BM, BN, WAVES_M, WAVES_N, STAGES, MODE, FP8, WAVES_K, false, SPARSE, true, FP4>(b, xcd_share_start(total, xcd) + local);
}

template <bool SPARSE, int BM, int BN, int WAVES_M, int WAVES_N, int WAVES_K, int STAGES, int MODE = 0, bool FP8 = false, bool FP4 = false>
struct Split {
    using L = Smem<SPARSE, BM, BN, STAGES, WAVES_M, WAVES_N, FP8, WAVES_K, FP4>;
    static hipError_t prepare() {
        auto kern = gemm_split_kernel<SPARSE, BM, BN, WAVES_M, WAVES_N, WAVES_K, STAGES, MODE, FP8, FP4>;
        return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
    }
    static hipError_t launch(const GemmArgs& a, hipStream_t stream) {
        auto kern = gemm_split_kernel<SPARSE, BM, BN, WAVES_M, WAVES_N, WAVES_K, STAGES, MODE, FP8, FP4>;
        const int64_t tiles = ((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN);
        hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(WAVES_M * WAVES_N * WAVES_K * 64), L::kTotal, stream, a);
        return hipGetLastError();
    }
};

// Contraction split over workgroups (PART): a.k_splits workgroups per tile, each with an even share of the k blocks,
// and split_reduce_kernel over their planes. For problems whose tiles do not reach all compute units and whose
// contraction is long enough to pay for the planes (M x N x 4 bytes each way per split) and the second launch.
// Whole calls, best unsplit shape -> split (us): dense [200, 3072, 12288] 36.9 -> 28.7, [333, 3072, 12288] 51.6 -> 37.6,
// [512, 1024, 12288] 29.7 -> 23.6; sparse [333, 3072, 12288] 44.4 -> 37.3, [700, 3072, 12288] 66.2 -> 55.7; LoRA [512, 3072,
// 12288] 55.9 -> 51.3.
template <bool SPARSE, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, int MODE = 0, bool FP8 = false, bool FP4 = false>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64) void gemm_part_kernel(const GemmArgs a) {
    const int tiles = (int)(((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN)), total = tiles * a.k_splits;
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8;
    const int idx = xcd_share_start(total, xcd) + local;       // an XCD's share: few parts, neighbouring tiles
    const int part = idx / tiles, blocks = (int)k_blocks(a.K, FP8, FP4);
    const int b0 = (int)((int64_t)blocks * part / a.k_splits), b1 = (int)((int64_t)blocks * (part + 1) / a.k_splits);
    gemm_tile<SPARSE, BM, BN, WAVES_M, WAVES_N, STAGES, MODE, FP8, 1, true, false, true, FP4>(a, idx % tiles, part, b0, b1 - b0);
}

// Adds the planes up in order, then factors, bias, bf16. A thread finishes eight columns of a row, the planes'
// loads in flight together; grid (column chunks / 256, rows).
constexpr int kMaxKSplits = 8;
__global__ __launch_bounds__(256) void split_reduce_kernel(const GemmArgs a, const bool factors) {
    const int64_t row = blockIdx.y, col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= a.N) return;
    const float* p = a.partials + row * a.part_pitch + col;
    float4 v[kMaxKSplits][2];
#pragma unroll
    for (int s = 0; s < kMaxKSplits; ++s)
        if (s < a.k_splits) {
            v[s][0] = *reinterpret_cast<const float4*>(p + (int64_t)s * a.M * a.part_pitch);
            v[s][1] = *reinterpret_cast<const float4*>(p + (int64_t)s * a.M * a.part_pitch + 4);
        }
    const int valid = (int)min((int64_t)8, a.N - col);
    float bv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bv[e] = a.bias ? __uint_as_float((uint32_t)a.bias[col + min(e, valid - 1)] << 16) : 0.f;
    const float f = factors ? (a.row_scale ? a.row_scale[row] : 1.0f) * (a.tensor_scale ? a.tensor_scale[0] : 1.0f) : 1.0f;
    float sum[8] = {v[0][0].x, v[0][0].y, v[0][0].z, v[0][0].w, v[0][1].x, v[0][1].y, v[0][1].z, v[0][1].w};
#pragma unroll
    for (int s = 1; s < kMaxKSplits; ++s)
        if (s < a.k_splits) {
            sum[0] += v[s][0].x; sum[1] += v[s][0].y; sum[2] += v[s][0].z; sum[3] += v[s][0].w;
            sum[4] += v[s][1].x; sum[5] += v[s][1].y; sum[6] += v[s][1].z; sum[7] += v[s][1].w;
        }
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    uint32_t out[4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const f32x2 y = {mul_add_rn(sum[e], f, bv[e]), mul_add_rn(sum[e + 1], f, bv[e + 1])};
        out[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));       // RNE
    }
    uint16_t* dst = a.Y + row * a.ldy + col;
    if (((reinterpret_cast<uintptr_t>(a.Y) & 15) == 0) && (a.ldy % 8 == 0) && valid == 8) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(out[0], out[1], out[2], out[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < valid) dst[e] = (uint16_t)(out[e >> 1] >> (16 * (e & 1)));
    }
}

template <bool SPARSE, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, int MODE = 0, bool FP8 = false, bool FP4 = false>
struct Part {
    using L = Smem<SPARSE, BM, BN, STAGES, WAVES_M, WAVES_N, FP8, 1, FP4>;
    static hipError_t prepare() {
        auto kern = gemm_part_kernel<SPARSE, BM, BN, WAVES_M, WAVES_N, STAGES, MODE, FP8, FP4>;
        return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
    }
    static hipError_t launch(const GemmArgs& a, hipStream_t stream) {
        auto kern = gemm_part_kernel<SPARSE, BM, BN, WAVES_M, WAVES_N, STAGES, MODE, FP8, FP4>;
        const int64_t tiles = ((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN);
        hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * a.k_splits)), dim3(WAVES_M * WAVES_N * 64), L::kTotal, stream, a);
        hipLaunchKernelGGL(split_reduce_kernel, dim3((unsigned)((a.N + 2047) / 2048), (unsigned)a.M), dim3(256), 0, stream, a,
                           MODE == 0);
        return hipGetLastError();
    }
};

}  // namespace

// ---- tile plan ---------------------------------------------------------------------------------
// A launch cuts rows [0, m_split) of the output into 256 x BN body tiles (BN = 256 or 192) and the
// remaining rows into 256 x 128 tail tiles. The main loop is bound by the rate at which a CU can pull
// operand stages out of L2, so a tile's time goes with its bytes per stage: 256x256 moves 51 KB,
// 256x192 43 KB (dense kernel: 64 and 56 KB per 64-k stage); a 256x128 tile was measured at 0.60 to
// 0.66 of a 256x256 tile. The plan is the (BN, m_split) whose simulated schedule ends first: per XCD
// (32 compute units, one workgroup each), workgroups in id order, each to the unit that frees first.
struct TilePlan {
    bool use_192;
    int64_t m_split;     // rows covered by body tiles (a multiple of 256, or M when there is no tail)
    int body_tiles, tail_tiles;
    double cost;         // end of the simulated schedule (KB per stage, as c256 etc. in make_plan)
};

static double simulate_schedule(int64_t nb, int64_t nt, double cb, double ct) {
    double worst = 0.0;
    for (int x = 0; x < 8; ++x) {
        const int64_t tot = nb + nt;
        const int64_t nbx = nb / 8 + (x < nb % 8), cx = tot / 8 + (x < tot % 8);
        double unit[32] = {0};
        for (int64_t i = 0; i < cx; ++i) {
            int best = 0;
            for (int u = 1; u < 32; ++u)
                if (unit[u] < unit[best]) best = u;
            unit[best] += i < nbx ? cb : ct;
        }
        for (int u = 0; u < 32; ++u) worst = unit[u] > worst ? unit[u] : worst;
    }
    return worst;
}

static TilePlan make_plan(int64_t M, int64_t N, bool dense) {
    const double c256 = dense ? 64 : 51, c192 = dense ? 56 : 43, c128 = 0.64 * c256;
    const int64_t tm = (M + 255) / 256;
    const int64_t n256 = (N + 255) / 256, n192 = (N + 191) / 192, n128 = (N + kTailBN - 1) / kTailBN;
    if (tm * n128 > (int64_t)1 << 16) {
        // very large grids: many rounds, the last one no longer matters; pick the cheaper uniform shape
        // by rounds x bytes per stage and skip the simulation (it is linear in the number of tiles)
        const double r256 = (double)((tm * n256 + 255) / 256) * c256, r192 = (double)((tm * n192 + 255) / 256) * c192;
        return r192 < r256 ? TilePlan{true, M, (int)(tm * n192), 0, r192} : TilePlan{false, M, (int)(tm * n256), 0, r256};
    }
    double best_cost = simulate_schedule(tm * n256, 0, c256, c128);
    TilePlan best{false, M, (int)(tm * n256), 0, best_cost};
    auto consider = [&](bool use_192, int64_t p) {
        if (p < 0 || p > tm) return;
        const int64_t nb = p * (use_192 ? n192 : n256), nt = (tm - p) * n128;
        double cost = simulate_schedule(nb, nt, use_192 ? c192 : c256, c128);
        if (nt > 0) cost *= 1.03;          // a tail has to pay for itself
        if (cost < best_cost - 1e-9) {
            best_cost = cost;
            best = TilePlan{use_192, p == tm ? M : p * 256, (int)nb, (int)nt, cost};
        }
    };
    consider(true, tm);
    // body sizes that fill whole rounds of the chip, and a few panels around them
    for (int use_192 = 0; use_192 < 2; ++use_192) {
        const int64_t tn = use_192 ? n192 : n256;
        const int64_t rounds = tm * tn / 256;
        for (int64_t r = rounds; r >= rounds - 1 && r >= 0; --r)
            for (int64_t d = -2; d <= 1; ++d) consider(use_192 != 0, r * 256 / tn + d);
    }
    return best;
}

// Plans are cached per (M, N, kind): the simulation costs tens of microseconds on the host.
static TilePlan plan_for(int64_t M, int64_t N, bool dense) {
    struct Entry { int64_t M, N; bool dense; TilePlan plan; };
    static std::mutex mu;
    static std::vector<Entry> cache;
    std::lock_guard<std::mutex> lock(mu);
    for (const Entry& e : cache)
        if (e.M == M && e.N == N && e.dense == dense) return e.plan;
    const TilePlan p = make_plan(M, N, dense);
    if (cache.size() < 4096) cache.push_back(Entry{M, N, dense, p});
    return p;
}

void tile_plan(int64_t M, int64_t N, bool dense, int64_t out[4]) {
    const TilePlan p = plan_for(M, N, dense);
    out[0] = p.use_192 ? 192 : 256;
    out[1] = p.m_split;
    out[2] = p.body_tiles;
    out[3] = p.tail_tiles;
}

// ---- small tiles -------------------------------------------------------------------------------
// Shapes of gemm_split_kernel with what one workgroup takes alone on its compute unit: `fixed` us (prologue,
// reduction of the K groups, epilogue) plus `block` us per k block, both measured ([1..4096, 3072 | 12288,
// 3072 | 12288], 250 points per operand kind).
struct SplitShape {
    int bm, bn;
    double fixed, block;
};
// Sparse 256 x 96 (eight waves of 32 rows, ring of four) stands between the 128 x 128 tile and the 256-row plan: with the plan's
// 256 x 128 tiles an output of 130 to 192 tiles leaves compute units idle and each of the others pulls 34 KB a stage, here up to 256
// pull 30. Its constants put the line where measurement has it, which is at fewer stages (kFixed96Early) in FP8 and for widths not divisible by
// 8, whose 2-byte stores take the plan's tiles longer ([1289, 3372, 512] 22.3 -> 19.8, [864, 5158, 2048] 41.1 -> 36.4). Forced against the best
// other form at 760 drawn shapes of all sparse kinds that it can run in one pass ([129..16896, 512..21504, 512..15360], inputs from HBM):
// bf16 70 of 490 take it, FP8 75 of 270, 6.7 % and 4.7 % faster in the mean and none slower by 1 % (32 of 200 others: 6.1 %, none slower): sparse
// [793, 4672, 8960] 98.5 -> 86.0 us, [4906, 832, 11392] 137.8 -> 128.2, FP8 [737, 5825, 6400] 52.1 -> 48.7, FP8 + LoRA [434, 10432, 512] 13.9 -> 13.0;
// with a line at 20 stages bf16 lost up to 9 % ([886, 5952, 1280], [3516, 1504, 1536] 22.7 -> 24.5).
// Dense 256 x 96 (ring of three) for the same reason where 256 x 128 tiles (which the plan's tails are) do not reach all units: 108 of 2360 drawn shapes take it, 5.9 % faster
// than the best other form in the mean, 9.7 % slower at worst.
constexpr SplitShape kSparseShapes[] = {
    {32, 32, 1.2, 0.087}, {64, 32, 1.9, 0.108}, {64, 64, 2.4, 0.153}, {128, 64, 2.3, 0.19}, {128, 128, 2.8, 0.30},
    {256, 96, 9.2, 0.325}};
constexpr double kFixed96Early = 3.4;
constexpr SplitShape kDenseShapes[] = {
    {32, 32, 1.45, 0.081}, {64, 32, 1.55, 0.135}, {64, 64, 1.25, 0.19}, {128, 64, 2.5, 0.285}, {128, 128, 3.4, 0.38},
    {256, 96, 3.95, 0.44}};

// How the problem should run. Times are estimated from the measured constants: a small shape needs ceil(tiles / 256)
// passes over the 256 compute units; with more than one, all units pull operands all the time and slow each other down
// beyond the constants, which were taken one workgroup to a unit (factor 1.1; dense 1.24, 128 x 128 1.12 with two passes, 1.3
// with more). The 256-row plan is its simulated schedule times the time per KB of a stage, which grows from 10.7 ns (dense
// 14.6: both operands row-major) while at most 96 units work to 17.2 (20) when all do and share the L2s and the power
// budget. One table serves every operand kind, but for the line of the sparse 256 x 96 tile: the others rank the same way in FP8 and LoRA
// calls (LoRA's residual, 5 us a tile of the 256-row plan, is left out), and LoRA without its residual then sums like the plain call.
// 4-bit calls use it by 128-byte stages (256 of the contraction): against every form forced on 311 problems 1.1 % slower than the best in the mean.
// Against every form forced one by one on drawn shapes that played no part in the fit ([1..16896, 512..21504, 512..15360], inputs from
// HBM): sparse of all kinds, 600 shapes: 1.0 % slower than the best on average, more than 2 % slower than the 256-row plan at 2; dense,
// 600 shapes: 0.3 % and 5. (The constants of the dense loop before its 16 x 16 instructions: 2.1 % and 19 of 2360.)
// With the factors at 0.92 (sparse 64 x 64 and 128 x 128) 128 x 128 tiles in several passes lost up to 1.29x to the plan: [1408, 14368,
// 11904] 303 -> 392 us; above 2048 rows they won more than 3 % at 2 of 220.
struct SplitChoice {
    int shape;       // index of the small shape, or -1 for the 256-row plan
    int k_splits;    // > 1: gemm_part_kernel on the 128 x 128 (part_256 false) or 256 x 128 tile
    bool part_256;
};
static int64_t part_pitch(int64_t N) { return (N + 7) / 8 * 8; }     // columns of a plane: whole eight-column chunks
static SplitChoice pick_split(const TilePlan& plan, int64_t M, int64_t N, int64_t blocks, bool dense, bool fp8, size_t room) {
    const double busy = (double)(plan.body_tiles + plan.tail_tiles < 256 ? plan.body_tiles + plan.tail_tiles : 256);
    const double load = busy > 96 ? (busy - 96) / 160 : 0.0;
    const double per_kb = dense ? 0.0146 + 0.0053 * load : 0.0107 + 0.0065 * load;
    double best = (dense ? 3.3 : 3.4) + (double)blocks * plan.cost * per_kb;
    SplitChoice pick{-1, 1, false};
    const SplitShape* shapes = dense ? kDenseShapes : kSparseShapes;
    const int count = dense ? (int)(sizeof(kDenseShapes) / sizeof(SplitShape)) : (int)(sizeof(kSparseShapes) / sizeof(SplitShape));
    for (int i = 0; i < count; ++i) {
        const SplitShape& s = shapes[i];
        const int64_t tiles = ((M + s.bm - 1) / s.bm) * ((N + s.bn - 1) / s.bn);
        if (tiles > 4096) continue;                        // far more than a few passes: never the better one
        double block = s.block;
        if (s.bm == 256) {                                 // one pass only, slower as the chip fills (its rivals are, in the sparse case)
            if (tiles > 256) continue;
            if (dense && tiles > 128) block += 0.0021 * (double)(tiles - 128);
        }
        if (dense && s.bm == 32) block += 0.0005 * (double)(M < 32 ? M : 32);      // (rows past M repeat the last one: less to pull)
        const int64_t passes = (tiles + 255) / 256;
        if (passes > 1 && s.bm >= 128 && s.bn >= 128 && M > 2048) continue;
        // (the dense 64 x 64 line was fitted at long K; with one or two blocks it takes what its neighbours do: [161, 6168, 128]
        // 8.2 us against 7.4 with the 256-row plan and 6.4 with 128 x 64, [1981, 1024, 128] 7.4 / 6.2 / 5.5)
        const double fixed = dense && s.bm == 64 && s.bn == 64 && blocks <= 2 ? 2.4 : !dense && s.bm == 256 && (fp8 || N % 8 != 0) ? kFixed96Early : s.fixed;
        const double several = !dense ? 1.1 : s.bm >= 128 && s.bn >= 128 ? (passes > 2 ? 1.3 : 1.12) : 1.24;
        const double t = (double)passes * (fixed + (double)blocks * block) * (passes > 1 ? several : 1.0);
        if (t < best) {
            best = t;
            pick.shape = i;
        }
    }
    // Contraction split over workgroups: at most one workgroup per compute unit, at least 16 blocks each (dense 20, but 16 from 9 to 64
    // rows, which 32 x 32 tiles would take in full), up to six parts
    // (dense eight). Second launch, writing and reading the planes: 8 us + 0.5 us per MB of planes (dense 5.1 + 0.31); the
    // estimate has to be 2 % better than the best unsplit one.
    const int64_t min_blocks = dense && (M <= 8 || M > 64) ? 20 : 16;
    for (int big = 0; big < 2; ++big) {
        const int64_t tiles = ((M + (big ? 255 : 127)) / (big ? 256 : 128)) * ((N + 127) / 128);
        const double block = big ? (dense ? 0.535 : 0.35) : (dense ? 0.395 : 0.285);
        for (int s = 2; s <= (dense ? kMaxKSplits : 6) && tiles * s <= 256 && blocks / s >= min_blocks; ++s) {
            const double planes = (double)s * (double)M * (double)part_pitch(N) * 4.0;
            if (planes > (double)room) break;
            const double t = (double)((blocks + s - 1) / s) * block + (dense ? 5.1 + planes * 0.31e-6 : 8.0 + planes * 0.5e-6);
            if (t < best * (pick.k_splits > 1 ? 1.0 : 0.98)) {
                best = t;
                pick = SplitChoice{pick.shape, s, big != 0};
            }
        }
    }
    return pick;
}

// Size of the partial planes of the choice made with `room` bytes (0 where the contraction is not split over workgroups).
// launch_gemm makes the same choice with any room from this size up to `room`.
size_t gemm_partial_bytes(bool sparse, bool fp8, int64_t M, int64_t N, int64_t K, size_t room, bool fp4) {
    const int64_t blocks = k_blocks(K, fp8, fp4);
    if (blocks < 32 || ((M + 255) / 256) * ((N + 127) / 128) > 128) return 0;       // (the bound of the loop above at two splits)
    const SplitChoice c = pick_split(plan_for(M, N, !sparse), M, N, blocks, !sparse, fp8, room);
    return c.k_splits > 1 ? (size_t)c.k_splits * (size_t)M * (size_t)part_pitch(N) * 4 : 0;
}

void gemm_choice(bool sparse, bool fp8, int64_t M, int64_t N, int64_t K, size_t room, int out[3]) {
    const SplitChoice c = pick_split(plan_for(M, N, !sparse), M, N, K / (fp8 ? 128 : 64), !sparse, fp8, room);
    out[0] = c.k_splits > 1 ? -1 : c.shape;
    out[1] = c.k_splits;
    out[2] = c.part_256 ? 256 : 128;
}

void mx_choice(int64_t M, int64_t N, int64_t K, size_t room, int out[3]) {
    const SplitChoice c = pick_split(plan_for(M, N, true), M, N, k_blocks(K, false, true), true, false, room);
    out[0] = c.k_splits > 1 ? -1 : c.shape;
    out[1] = c.k_splits;
    out[2] = c.part_256 ? 256 : 128;
}

// FP8 calls of the 256-row plan: stream bases pinned to SGPRs (PIN of gemm_tile) with 256-column bodies from 20 stages of 128 k on.
// Not pinned -> pinned, us: 256-column bodies [14238, 13344, K] K = 1024 193.3 -> 201.6, 1280 224.4 -> 248.5, 2048 282.4 -> 281.0, 2560
// 339.9 -> 337.9, 3072 382.4 -> 374.3; [10000, 20000, K] 1280 231.4 -> 241.8, 2560 357.2 -> 350.8, 3072 404.5 -> 392.8; [12000, 2048, K] 1024
// 40.6 -> 41.2, 2048 59.0 -> 60.7, 2560 65.1 -> 64.2; [9734, 5760, K] 768 63.9 -> 64.0, 2560 117.0 -> 115.7. 192-column bodies [5326, 3680, K]
// 1024 31.8 -> 32.9, 3072 57.2 -> 57.9; [2887, 3072, 6144] 53.8 -> 53.7. (It is W's base that does it; a reason was not found.)
constexpr int kPinStages = 20;

// Runs `op` (launch or prepare) of small shape `i`. Ring depths: as many stages as LDS holds, two workgroups
// per unit for 64 x 64 and 128 x 128 (sparse).
template <bool SPARSE, int MODE, bool FP8, bool FP4, class Op>
static hipError_t with_split(int i, Op op) {
    if constexpr (SPARSE) {
        switch (i) {
            case 0: return op(Split<true, 32, 32, 1, 1, 4, 4, MODE, FP8>{});
            case 1: return op(Split<true, 64, 32, 1, 1, 4, 4, MODE, FP8>{});
            case 2: return op(Split<true, 64, 64, 1, 2, 2, 3, MODE, FP8>{});
            case 3: return op(Split<true, 128, 64, 2, 2, 2, 3, MODE, FP8>{});
            case 4: return op(Split<true, 128, 128, 2, 2, 1, 3, MODE, FP8>{});
            default: return op(Split<true, 256, 96, 8, 1, 1, 4, MODE, FP8>{});
        }
    } else {
        switch (i) {
            case 0: return op(Split<false, 32, 32, 1, 1, 4, 4, 0, false, FP4>{});
            case 1: return op(Split<false, 64, 32, 1, 1, 4, 3, 0, false, FP4>{});
            case 2: return op(Split<false, 64, 64, 1, 2, 2, 4, 0, false, FP4>{});
            case 3: return op(Split<false, 128, 64, 2, 2, 2, 3, 0, false, FP4>{});
            case 4: return op(Split<false, 128, 128, 2, 2, 1, 3, 0, false, FP4>{});
            default: return op(Split<false, 256, 96, 4, 2, 1, 3, 0, false, FP4>{});
        }
    }
}

template <bool SPARSE, int MODE, bool FP8, bool FP4, class Op>
static hipError_t with_part(bool big, Op op) {
    if (big) return op(Part<SPARSE, 256, 128, Tail<SPARSE>::kWavesM, Tail<SPARSE>::kWavesN, 3, MODE, FP8, FP4>{});
    return op(Part<SPARSE, 128, 128, 2, 2, 3, MODE, FP8, FP4>{});
}

// Every configuration launch_gemm can pick.
hipError_t prepare_gemm_kernels() {
    hipError_t e = hipSuccess;
    auto run = [&](hipError_t r) { if (e == hipSuccess) e = r; };
    run(Mixed<true, 192, 4, 2, 3, 0, true>::prepare());
    run(Mixed<true, 256, 2, 4, 3, 0, true>::prepare());
    run(Mixed<true, 256, 2, 4, 3, 0, true, true>::prepare());
    run(Mixed<true, 192, 4, 2, 3, 1, true>::prepare());
    run(Mixed<true, 256, 2, 4, 3, 1, true>::prepare());
    run(Mixed<true, 256, 2, 4, 3, 1, true, true>::prepare());
    run(Mixed<true, 192, 4, 2, 3, 1>::prepare());
    run(Mixed<true, 192, 4, 2, 3>::prepare());
    run(Mixed<true, 256, 2, 4, 3, 1>::prepare());
    run(Mixed<true, 256, 2, 4, 3>::prepare());
    run(Mixed<false, 192, 2, 4, 2>::prepare());
    run(Mixed<false, 256, 2, 4, 2>::prepare());
    run(Mixed<false, 192, 2, 4, 2, 0, false, true, true>::prepare());
    run(Mixed<false, 256, 2, 4, 2, 0, false, true, true>::prepare());
    auto prep = [](auto k) { return decltype(k)::prepare(); };
    for (int i = 0; i < 6; ++i) {
        run(with_split<true, 0, false, false>(i, prep));
        run(with_split<true, 1, false, false>(i, prep));
        run(with_split<true, 0, true, false>(i, prep));
        run(with_split<true, 1, true, false>(i, prep));
        run(with_split<false, 0, false, false>(i, prep));
        run(with_split<false, 0, false, true>(i, prep));
    }
    for (int i = 0; i < 2; ++i) {
        run(with_part<false, 0, false, false>(i != 0, prep));
        run(with_part<false, 0, false, true>(i != 0, prep));
        run(with_part<true, 0, false, false>(i != 0, prep));
        run(with_part<true, 1, false, false>(i != 0, prep));
        run(with_part<true, 0, true, false>(i != 0, prep));
        run(with_part<true, 1, true, false>(i != 0, prep));
    }
    return e;
}

hipError_t launch_gemm(bool sparse, const GemmArgs& a_in, hipStream_t stream) {
    GemmArgs a = a_in;
    const TilePlan plan = plan_for(a.M, a.N, !sparse);
    a.m_split = plan.m_split;
    a.body_tiles = plan.body_tiles;
    a.tail_tiles = plan.tail_tiles;
    a.rows_pad = kmajor_rows(a.M);
    a.t_plane = a.M * kLoraRank;
    // The TENSOR factor: formed by the small-tile kernels themselves while that is cheaper than a launch (each of their
    // workgroups reads all rows' sums: up to two passes of workgroups and 2048 rows), else by its own kernel. Whole call
    // [M, 3072, 3072], own kernel -> folded, us: M = 37 12.2 -> 11.1, 512 21.9 -> 20.4, 1024 28.6 -> 27.6; [2000, 512, 1024] 15.4 -> 13.8; 4000 rows lost 0.2.
    const SplitChoice choice = pick_split(plan, a.M, a.N, k_blocks(a.K, a.fp8, a.fp4), !sparse, a.fp8,
                                          a.partials ? a.partial_bytes : 0);
    if (a.rowsums) {
        bool fold = sparse && choice.k_splits == 1 && choice.shape >= 0 && a.M <= 2048;
        if (fold) {
            const SplitShape& s = kSparseShapes[choice.shape];
            fold = ((a.M + s.bm - 1) / s.bm) * ((a.N + s.bn - 1) / s.bn) <= 512;
        }
        if (!fold) {
            const hipError_t e = launch_tensor_scale(a.rowsums, a.M, a.factor_eps, a.factor_out, stream, a.factor_mul, a.factor_fused);
            if (e != hipSuccess) return e;
            a.rowsums = nullptr;
            a.tensor_scale = a.factor_fused ? a.factor_fused : a.factor_out;
        }
    }
    auto go = [&](auto k) { return decltype(k)::launch(a, stream); };
    if (choice.k_splits > 1) {
        a.k_splits = choice.k_splits;
        a.part_pitch = part_pitch(a.N);
        const bool big = choice.part_256;
        if (a.fp4) return with_part<false, 0, false, true>(big, go);
        if (!sparse) return with_part<false, 0, false, false>(big, go);
        if (a.fp8) return a.T ? with_part<true, 1, true, false>(big, go) : with_part<true, 0, true, false>(big, go);
        return a.T ? with_part<true, 1, false, false>(big, go) : with_part<true, 0, false, false>(big, go);
    }
    const int split = choice.shape;
    if (split >= 0) {
        if (a.fp4) return with_split<false, 0, false, true>(split, go);
        if (!sparse) return with_split<false, 0, false, false>(split, go);
        if (a.fp8) return a.T ? with_split<true, 1, true, false>(split, go) : with_split<true, 0, true, false>(split, go);
        return a.T ? with_split<true, 1, false, false>(split, go) : with_split<true, 0, false, false>(split, go);
    }
    if (sparse && a.fp8) {
        const bool pin = a.K >= 128 * kPinStages;
        if (a.T != nullptr) {          // LoRA tail in bf16 on top of the FP8 product
            if (plan.use_192) return Mixed<true, 192, 4, 2, 3, 1, true>::launch(a, stream);
            if (pin) return Mixed<true, 256, 2, 4, 3, 1, true, true>::launch(a, stream);
            return Mixed<true, 256, 2, 4, 3, 1, true>::launch(a, stream);
        }
        if (plan.use_192) return Mixed<true, 192, 4, 2, 3, 0, true>::launch(a, stream);
        if (pin) return Mixed<true, 256, 2, 4, 3, 0, true, true>::launch(a, stream);
        return Mixed<true, 256, 2, 4, 3, 0, true>::launch(a, stream);
    }
    if (sparse) {
        const bool lora = a.T != nullptr;
        if (plan.use_192) {
            if (lora) return Mixed<true, 192, 4, 2, 3, 1>::launch(a, stream);
            return Mixed<true, 192, 4, 2, 3>::launch(a, stream);
        }
        if (lora) return Mixed<true, 256, 2, 4, 3, 1>::launch(a, stream);
        return Mixed<true, 256, 2, 4, 3>::launch(a, stream);
    }
    if (a.fp4) {
        if (plan.use_192) return Mixed<false, 192, 2, 4, 2, 0, false, true, true>::launch(a, stream);
        return Mixed<false, 256, 2, 4, 2, 0, false, true, true>::launch(a, stream);
    }
    // dense: stages of 64 k (whole-line requests on the row-major operands), body tiles with a ring of two
    if (plan.use_192) return Mixed<false, 192, 2, 4, 2>::launch(a, stream);
    return Mixed<false, 256, 2, 4, 2>::launch(a, stream);
}

}  // namespace rtl
