// Gated linears: H = act(X Wg^T + bg) (X Wu^T + bu) in one kernel, on the dense tile loop (gemm_tile.h, MODE 2), and the elementwise part of their
// backward pass; its products are those of the linears grouped by expert, with one expert.
#include "gemm_tile.h"

namespace rtl {
namespace {

template <int BM, int BN, int WAVES_M, int WAVES_N, int WAVES_K, int STAGES>
__global__ __launch_bounds__(WAVES_M * WAVES_N * WAVES_K * 64) void gated_kernel(const GemmArgs a) {
    const int total = (int)(((a.M + BM - 1) / BM) * ((a.N + BN / 2 - 1) / (BN / 2)));
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8;
    gemm_tile<false, BM, BN, WAVES_M, WAVES_N, STAGES, 2, false, WAVES_K>(a, xcd_share_start(total, xcd) + local);
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int WAVES_K, int STAGES>
struct Gated {
    using L = Smem<false, BM, BN, STAGES, WAVES_M, WAVES_N, false, WAVES_K>;
    static hipError_t prepare() {
        return hipFuncSetAttribute(reinterpret_cast<const void*>(gated_kernel<BM, BN, WAVES_M, WAVES_N, WAVES_K, STAGES>),
                                   hipFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
    }
    static hipError_t launch(const GemmArgs& a, hipStream_t stream) {
        const int64_t tiles = ((a.M + BM - 1) / BM) * ((a.N + BN / 2 - 1) / (BN / 2));
        hipLaunchKernelGGL((gated_kernel<BM, BN, WAVES_M, WAVES_N, WAVES_K, STAGES>), dim3((unsigned)tiles), dim3(WAVES_M * WAVES_N * WAVES_K * 64),
                           L::kTotal, stream, a);
        return hipGetLastError();
    }
};

// dP = [dH U act'(G), dH act(G)] and, with H set, H = act(G) U again. Eight columns to a thread, F a multiple of four, rows of any 8-byte alignment. Bound by
// memory: five or six values of two bytes per element of H. dP is rounded to bf16, the type that the matrix cores take in the products behind it. The
// workspace's two offsets for those products, all rows for the one expert, are written on the way.
constexpr int kGradThreads = 256;
template <bool ERF>
__global__ __launch_bounds__(kGradThreads) void gated_grad_kernel(const GatedGradArgs a) {
    if (a.offsets && blockIdx.x == 0 && threadIdx.x < 2) a.offsets[threadIdx.x] = threadIdx.x ? (int)a.M : 0;
    const int runs = (int)((a.F + 7) / 8);
    const int64_t first = (int64_t)blockIdx.x * kGradThreads, row0 = first / runs;
    const int q = (int)(first - row0 * runs) + (int)threadIdx.x;
    const int64_t row = row0 + q / runs;
    const int col = q % runs * 8;
    if (row >= a.M) return;
    const bool whole = col + 8 <= a.F;
    auto load = [&](const uint16_t* p, float (&f)[8]) {
        uint32_t w[4] = {};
        if (whole) __builtin_memcpy(w, p, 16);
        else __builtin_memcpy(w, p, 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = __uint_as_float(w[e] << 16);
            f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    };
    float g[8], u[8], d[8], dg[8], du[8], h[8];
    load(a.P + row * a.ldp + col, g);
    load(a.P + row * a.ldp + a.F + col, u);
    load(a.dH + row * a.lddh + col, d);
    const GateForm form = gate_form(a.act);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float value, slope;
        gate_both<ERF>(g[e], form, value, slope);
        dg[e] = d[e] * u[e] * slope;
        du[e] = d[e] * value;
        h[e] = value * u[e];
    }
    const int valid = whole ? 8 : 4;
    store_run(a.dP + row * a.lddp + col, dg, valid);
    store_run(a.dP + row * a.lddp + a.F + col, du, valid);
    if (a.H) store_run(a.H + row * a.ldh + col, h, valid);
}

using Gated128 = Gated<128, 128, 2, 2, 1, 3>;

}  // namespace

hipError_t launch_gated(const GemmArgs& a, hipStream_t stream) { return Gated128::launch(a, stream); }

int64_t gated_grad_grid(int64_t M, int64_t F) { return (M * ((F + 7) / 8) + kGradThreads - 1) / kGradThreads; }
hipError_t launch_gated_grad(const GatedGradArgs& a, hipStream_t stream) {
    const int64_t grid = gated_grad_grid(a.M, a.F);
    const dim3 g((unsigned)(grid > 0 ? grid : 1));
    if (a.act == RTL_ACT_GELU) hipLaunchKernelGGL(gated_grad_kernel<true>, g, dim3(kGradThreads), 0, stream, a);
    else hipLaunchKernelGGL(gated_grad_kernel<false>, g, dim3(kGradThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t prepare_gated_kernels() { return Gated128::prepare(); }

}  // namespace rtl
