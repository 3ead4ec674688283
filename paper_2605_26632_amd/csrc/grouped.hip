// Linears grouped by expert: Y[rows of e] = X[rows of e] W[e]^T (+ b[e]), bf16 or microscaled 4-bit operands, on the dense tile loop.
// An expert's rows are a problem of their own inside the launch: same loop, operands shifted to the expert's first row and weight.
// [8192, 4096, 2048] over eight experts, inputs that change: 124 us with 1024 rows each, 147 with 484 to 1997 (uneven rounds). Into a given
// result one expert takes 108, eight even ones that share a weight 106, with weights of their own 118, the dense linear 107. 4-bit, uneven, the same inputs again: 56.5 us, eight stages a tile; bf16 then 127.9, matrix cores busy 51 % at 2.09 GHz.
#include <cmath>
#include "groups.h"

namespace rtl {
namespace {

// The problem of `rows` rows of an expert.
template <bool FP4>
__device__ __forceinline__ GemmArgs expert_problem(const GemmArgs& a, const GroupArgs& g, int expert, int begin, int rows) {
    constexpr int ESZ = FP4 ? 1 : 2;
    GemmArgs b = a;
    b.M = rows;
    b.A = static_cast<const uint8_t*>(a.A) + begin * a.lda * ESZ;
    b.W = static_cast<const uint8_t*>(a.W) + expert * g.w_stride * ESZ;
    b.Y = a.Y + begin * a.ldy;
    if (a.bias) b.bias = a.bias + expert * a.N;
    if constexpr (FP4) {
        b.a_scale = a.a_scale + (int64_t)begin * 8;
        b.w_scale = a.w_scale + expert * a.N * 8;
    }
    return b;
}

template <bool FP4>
__global__ __launch_bounds__(512) void grouped_mixed_kernel(const GemmArgs a, const GroupArgs g) {
    mixed_tiles(g.offsets, g.experts, (int)a.M, (int)((a.N + 255) / 256), (int)(FP4 ? (a.K + 255) / 256 : a.K / 64), [&](const MixedTile& t) {
        const GemmArgs b = expert_problem<FP4>(a, g, t.expert, t.begin, t.rows);
        if (t.tall) gemm_tile<false, 256, 256, 2, 4, 2, 0, false, 1, false, false, true, FP4, true>(b, t.tile);
        else gemm_tile<false, 128, 256, 2, 4, 3, 0, false, 1, false, false, true, FP4, true>(b, t.tile);
    });
}

template <bool FP4>
struct GroupedMixed {
    using L0 = Smem<false, 256, 256, 2, 2, 4, false, 1, FP4>;
    using L1 = Smem<false, 128, 256, 3, 2, 4, false, 1, FP4>;
    static constexpr int kLds = L0::kTotal > L1::kTotal ? L0::kTotal : L1::kTotal;
    static int64_t grid(int64_t T, int64_t E, int64_t N) { return group_grid(T, E, N, 128, 256); }
    static hipError_t prepare() {
        return hipFuncSetAttribute(reinterpret_cast<const void*>(grouped_mixed_kernel<FP4>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    }
    static hipError_t launch(const GemmArgs& a, const GroupArgs& g, hipStream_t stream) {
        hipLaunchKernelGGL(grouped_mixed_kernel<FP4>, dim3(kUnits), dim3(512), kLds, stream, a, g);
        return hipGetLastError();
    }
};

template <bool FP4, int BM, int BN, int WAVES_M, int WAVES_N, int WAVES_K, int STAGES>
__global__ __launch_bounds__(WAVES_M * WAVES_N * WAVES_K * 64) void grouped_kernel(const GemmArgs a, const GroupArgs g) {
    GroupTile t;
    if (!group_tile(g.offsets, g.experts, (int)a.M, BM, (int)((a.N + BN - 1) / BN), t)) return;
    const GemmArgs b = expert_problem<FP4>(a, g, t.expert, t.begin, t.rows);
    gemm_tile<false, BM, BN, WAVES_M, WAVES_N, STAGES, 0, false, WAVES_K, false, false, true, FP4, true>(b, t.tile);
}

template <bool FP4, int BM, int BN, int WAVES_M, int WAVES_N, int WAVES_K, int STAGES>
struct Grouped {
    using L = Smem<false, BM, BN, STAGES, WAVES_M, WAVES_N, false, WAVES_K, FP4>;
    static int64_t grid(int64_t T, int64_t E, int64_t N) { return group_grid(T, E, N, BM, BN); }
    static hipError_t prepare() {
        auto kern = grouped_kernel<FP4, BM, BN, WAVES_M, WAVES_N, WAVES_K, STAGES>;
        return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
    }
    static hipError_t launch(const GemmArgs& a, const GroupArgs& g, hipStream_t stream) {
        auto kern = grouped_kernel<FP4, BM, BN, WAVES_M, WAVES_N, WAVES_K, STAGES>;
        hipLaunchKernelGGL(kern, dim3((unsigned)grid(a.M, g.experts, a.N)), dim3(WAVES_M * WAVES_N * WAVES_K * 64), L::kTotal, stream,
                           a, g);
        return hipGetLastError();
    }
};

// Zeros into the rows in front of the first expert's and behind the last one's, a thread to eight columns at a time. What it writes is seldom more than a
// few rows, so that it costs its launch, where a fill of the whole result writes all of it twice ([8192, 4096] beside the product into a given result: 13.0 -> 1.6 to 4.2 us).
constexpr int kClearGrid = 1024;
__global__ __launch_bounds__(256) void grouped_clear_kernel(const int* offsets, int E, uint16_t* Y, int64_t T, int64_t cols, int64_t ld) {
    const int64_t first = min((int64_t)max(offsets[0], 0), T), last = min(max((int64_t)offsets[E], first), T);
    const int64_t chunks = (cols + 7) / 8, all = (first + T - last) * chunks;
    for (int64_t n = blockIdx.x * (int64_t)256 + threadIdx.x; n < all; n += (int64_t)gridDim.x * 256) {
        const int64_t i = n / chunks, col = n % chunks * 8;
        uint16_t* p = Y + (i < first ? i : i - first + last) * ld + col;
        if (col + 8 <= cols && reinterpret_cast<uintptr_t>(p) % 16 == 0) *reinterpret_cast<uint4*>(p) = make_uint4(0, 0, 0, 0);
        else
            for (int64_t j = 0; j < 8 && col + j < cols; ++j) p[j] = 0;
    }
}

template <bool FP4, class Op>
auto with_grouped(int shape, Op op) {
    switch (shape) {
        case 0: return op(Grouped<FP4, 32, 32, 1, 1, 4, 4>{});
        case 1: return op(Grouped<FP4, 64, 64, 1, 2, 2, 4>{});
        case 2: return op(Grouped<FP4, 128, 128, 2, 2, 1, 3>{});
        default: return op(GroupedMixed<FP4>{});
    }
}

}  // namespace

int64_t group_grid(int64_t T, int64_t E, int64_t cols, int64_t bm, int64_t bn) {
    return (T / bm + (E < T ? E : T)) * ((cols + bn - 1) / bn);
}

double group_experts(int64_t T, int64_t E) { return E > 1 ? (double)E * (1 - std::pow(1 - 1.0 / (double)E, (double)T)) : 1.0; }

double group_panels(int64_t T, int64_t E, int64_t bm) {
    const double experts = group_experts(T, E), panels = (double)T / experts / (double)bm + 0.5;
    return experts * (panels > 1 ? panels : 1);
}

// Form of a launch: index of with_grouped, or kFew for few_rows.hip, the one with the least estimated time. us of a tile form: `fixed` and `stage` per 128-byte
// stage of the contraction while its tiles find a unit each, more passes in proportion (but only 0.6 of `fixed` again: the next tile starts while another
// ends); measured at 8, 128, 256 and 512 tiles and 8 and 64 stages. No form is faster than what it reads and writes (6.5 TB/s, part of it in the MALL).
// Over 612 problems ([1..64 experts, 1..2000 rows each, 256..4096, 512..6144], uneven experts), bf16 and 4-bit, the choice is 6 and 5 % slower in the mean
// than the best form (the constants were fitted on these problems); by rows per expert alone it could take six times as long.
constexpr int kFew = 4;
int grouped_form(int64_t T, int64_t E, int64_t N, int64_t K, bool fp4) {
    struct Form { int bm, bn; double fixed, stage; };
    static constexpr Form kForms[] = {{32, 32, 3.7, 0.09}, {64, 64, 4.2, 0.185}, {128, 128, 5.0, 0.43}};
    const double stages = (double)(fp4 ? (K + 255) / 256 : K / 64), t = (double)T, n = (double)N, k = (double)K;
    const double stream = 2.5 + (group_experts(T, E) * n * k * (fp4 ? 17.0 / 32 : 2.0) + t * k * (fp4 ? 17.0 / 32 : 2.0) + t * n * 2) / 6.5e6;
    auto floored = [&](double us) { return us > stream ? us : stream; };
    const double halves = group_panels(T, E, 128) * (double)((N + 255) / 256), rounds = halves > 256 ? halves / 256 : 1;
    int pick = 3;
    double best = floored(6.5 + (rounds - 1) * 5 + (0.6 + 0.15 * (halves < 256 ? halves / 256 : 1)) * stages * rounds);
    for (int i = 0; i < 3; ++i) {
        const Form& f = kForms[i];
        const double tiles = group_panels(T, E, f.bm) * (double)((N + f.bn - 1) / f.bn), passes = tiles > 256 ? tiles / 256 : 1;
        const double us = floored(f.fixed * (1 + 0.6 * (passes - 1)) + f.stage * stages * passes);
        if (us < best) {
            best = us;
            pick = i;
        }
    }
    const FewRows few = T <= 8 * E ? few_rows_choice((T + E - 1) / E, T, K, fp4) : FewRows::no;
    if (few != FewRows::no && few_rows_us(T, E, N, K, fp4, stream) - (few == FewRows::quantise ? 2.5 : 0) <= best) pick = kFew;
    return pick;
}

FewRows grouped_few_rows(int64_t T, int64_t E, int64_t N, int64_t K, bool fp4) {
    return grouped_form(T, E, N, K, fp4) == kFew ? few_rows_choice((T + E - 1) / E, T, K, fp4) : FewRows::no;
}

int64_t grouped_grid(int64_t T, int64_t E, int64_t N, int64_t K, bool fp4) {
    const int form = grouped_form(T, E, N, K, fp4);
    if (form == kFew) return few_rows_grid(E, N);
    auto grid = [&](auto k) { return decltype(k)::grid(T, E, N); };
    return fp4 ? with_grouped<true>(form, grid) : with_grouped<false>(form, grid);
}

hipError_t prepare_grouped_kernels() {
    hipError_t e = hipSuccess;
    auto prep = [](auto k) { return decltype(k)::prepare(); };
    for (int i = 0; i < 4 && e == hipSuccess; ++i) {
        e = with_grouped<false>(i, prep);
        if (e == hipSuccess) e = with_grouped<true>(i, prep);
    }
    return e;
}

hipError_t launch_grouped_clear(const int* offsets, int E, uint16_t* Y, int64_t T, int64_t cols, int64_t ld, hipStream_t stream) {
    const int64_t want = (T * ((cols + 7) / 8) + 255) / 256;
    hipLaunchKernelGGL(grouped_clear_kernel, dim3((unsigned)(want < kClearGrid ? want : kClearGrid)), dim3(256), 0, stream, offsets, E, Y, T, cols, ld);
    return hipGetLastError();
}

hipError_t launch_grouped(const GemmArgs& a, const GroupArgs& g, hipStream_t stream) {
    const int form = grouped_form(a.M, g.experts, a.N, a.K, a.fp4);
    if (form == kFew) return launch_grouped_few_rows(a, g, stream);
    auto go = [&](auto k) { return decltype(k)::launch(a, g, stream); };
    return a.fp4 ? with_grouped<true>(form, go) : with_grouped<false>(form, go);
}

}  // namespace rtl
