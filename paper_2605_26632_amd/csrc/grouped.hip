// Linears grouped by expert: Y[rows of e] = X[rows of e] W[e]^T (+ b[e]), bf16 or microscaled 4-bit operands, on the dense tile loop.
// An expert's rows are a problem of their own inside the launch: same loop, operands shifted to the expert's first row and weight.
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
    MixedTile t;
    if (!group_tile_mixed(g.offsets, g.experts, (int)a.M, (int)((a.N + 255) / 256), (int)(FP4 ? (a.K + 255) / 256 : a.K / 64), t)) return;
    const GemmArgs b = expert_problem<FP4>(a, g, t.expert, t.begin, t.rows);
    if (t.height == 256) gemm_tile<false, 256, 256, 2, 4, 2, 0, false, 1, false, false, true, FP4, true>(b, t.tile);
    else if (t.height == 192) gemm_tile<false, 192, 256, 2, 4, 2, 0, false, 1, false, false, true, FP4, true>(b, t.tile);
    else gemm_tile<false, 128, 256, 2, 4, 3, 0, false, 1, false, false, true, FP4, true>(b, t.tile);
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
        hipLaunchKernelGGL(grouped_mixed_kernel<FP4>, dim3((unsigned)grid(a.M, g.experts, a.N)), dim3(512), kLds, stream, a, g);
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

static int grouped_shape(int64_t T, int64_t E) {
    const int64_t rows = T / E;
    return rows <= 24 ? 0 : rows <= 64 ? 1 : rows <= 160 ? 2 : 3;
}

FewRows grouped_few_rows(int64_t T, int64_t E, int64_t K, bool fp4) {
    return T <= 8 * E ? few_rows_choice((T + E - 1) / E, T, K, fp4) : FewRows::no;
}

int64_t grouped_grid(int64_t T, int64_t E, int64_t N, int64_t K, bool fp4) {
    if (grouped_few_rows(T, E, K, fp4) != FewRows::no) return few_rows_grid(E, N);
    auto grid = [&](auto k) { return decltype(k)::grid(T, E, N); };
    return fp4 ? with_grouped<true>(grouped_shape(T, E), grid) : with_grouped<false>(grouped_shape(T, E), grid);
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

hipError_t launch_grouped(const GemmArgs& a, const GroupArgs& g, hipStream_t stream) {
    auto go = [&](auto k) { return decltype(k)::launch(a, g, stream); };
    if (grouped_few_rows(a.M, g.experts, a.K, a.fp4) != FewRows::no) return launch_grouped_few_rows(a, g, stream);
    const int shape = grouped_shape(a.M, g.experts);
    return a.fp4 ? with_grouped<true>(shape, go) : with_grouped<false>(shape, go);
}

}  // namespace rtl
