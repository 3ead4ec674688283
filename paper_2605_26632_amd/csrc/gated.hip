// Gated linears: H = act(X Wg^T + bg) (X Wu^T + bu) in one kernel, on the dense tile loop (gemm_tile.h, MODE 2), and the elementwise part of their
// backward pass; its products are one launch of the weight and input gradient's tiles (grouped_grad.hip).
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

// The 256-row plan: body tiles of 256 x BN rows of W, tail tiles of 256 x 128 over the rows of X behind m_split (gemm.hip has the reasons).
template <int BN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(512) void gated_mixed_kernel(const GemmArgs a) {
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8;
    const int nb = a.body_tiles, nt = a.tail_tiles, nb_x = nb / 8 + (xcd < nb % 8);
    if (local < nb_x) {
        GemmArgs b = a;
        if (nt > 0) b.M = a.m_split;
        gemm_tile<false, 256, BN, WAVES_M, WAVES_N, 2, 2>(b, xcd_share_start(nb, xcd) + local);
    } else {
        GemmArgs t = a;
        t.M = a.M - a.m_split;
        t.A = static_cast<const uint16_t*>(a.A) + a.m_split * a.lda;
        t.Y = a.Y + a.m_split * a.ldy;
        if (a.P) t.P = a.P + a.m_split * a.ldp;
        gemm_tile<false, 256, 128, 4, 2, 3, 2>(t, xcd_share_start(nb + nt, xcd) - xcd_share_start(nb, xcd) + (local - nb_x));
    }
}

template <int BN, int WAVES_M, int WAVES_N>
struct GatedMixed {
    static constexpr int kBody = Smem<false, 256, BN, 2, WAVES_M, WAVES_N, false>::kTotal, kTail = Smem<false, 256, 128, 3, 4, 2, false>::kTotal;
    static constexpr int kLds = kBody > kTail ? kBody : kTail;
    static hipError_t prepare() {
        return hipFuncSetAttribute(reinterpret_cast<const void*>(gated_mixed_kernel<BN, WAVES_M, WAVES_N>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    }
    static hipError_t launch(const GemmArgs& a, hipStream_t stream) {
        hipLaunchKernelGGL((gated_mixed_kernel<BN, WAVES_M, WAVES_N>), dim3((unsigned)(a.body_tiles + a.tail_tiles)), dim3(512), kLds, stream, a);
        return hipGetLastError();
    }
};

// Up to sixteen rows of X: reading W is all there is, and it goes straight from memory into the registers that the matrix instruction takes (few_rows.hip has
// the layout). A workgroup owns COLS columns of H: sixteen, sixteen gate rows of W for one instruction and the sixteen up rows for another; or
// eight, whose gate and up rows are the sixteen of one instruction, where sixteen would leave units idle, each of which pulls at a rate of its own. Its
// waves divide the contraction in lines of 128 bytes, neighbouring waves on neighbouring lines, four lines of a row in flight, and their sums meet in LDS in
// a fixed order. [1, 10240, 3840] 23.9 us one after the other in a graph, 6.6 TB/s.
constexpr int kFewRows = 16, kFewWaves = 4, kFewLines = 4;
template <int COLS>
__global__ __launch_bounds__(kFewWaves * 64, 4) void gated_few_rows_kernel(const GemmArgs a) {
    constexpr int NB = COLS == 16 ? 2 : 1;               // instructions for a line
    __shared__ __align__(16) float sums[kFewWaves][NB][64][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, kb = lane >> 4;
    const int units = (int)(a.K / 64);
    const int64_t n0 = (int64_t)blockIdx.x * COLS;
    const uint16_t* w_row[NB];
#pragma unroll
    for (int f = 0; f < NB; ++f) {
        const int64_t n = min(n0 + li % COLS, a.N - 1) + ((COLS == 16 ? f : li / COLS & 1) ? a.N : 0);
        w_row[f] = static_cast<const uint16_t*>(a.W) + n * a.ldw + kb * 16;
    }
    const uint16_t* const x_row = static_cast<const uint16_t*>(a.A) + min((int64_t)li, a.M - 1) * a.lda + kb * 16;     // (rows behind the last repeat it, never stored)
    f32x4 acc[NB] = {};
    for (int u0 = wave; u0 < units; u0 += kFewWaves * kFewLines) {
        Frag8 w[kFewLines][NB][2], x[kFewLines][2];
#pragma unroll
        for (int u = 0; u < kFewLines; ++u) {
            if (u0 + u * kFewWaves >= units) break;
            const int64_t at = (int64_t)(u0 + u * kFewWaves) * 64;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int f = 0; f < NB; ++f) w[u][f][c].u = *reinterpret_cast<const uint4*>(w_row[f] + at + c * 8);
                x[u][c].u = *reinterpret_cast<const uint4*>(x_row + at + c * 8);
            }
        }
        __builtin_amdgcn_sched_barrier(0);                                                       // all the loads first
#pragma unroll
        for (int u = 0; u < kFewLines; ++u) {
            if (u0 + u * kFewWaves >= units) break;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int f = 0; f < NB; ++f) acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[u][f][c].v, x[u][c].v, acc[f], 0, 0, 0);
        }
    }
    // row li of X, columns 4 kb .. of the sixteen (of fewer, in the first lane groups)
    const int64_t col = n0 + 4 * kb;
    const int valid = 4 * kb >= COLS ? 0 : (int)min((int64_t)4, a.N - col);
    float bias[2][4] = {};
    if (wave == 0 && a.bias && valid > 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t at = col + min(e, valid - 1);
            bias[0][e] = __uint_as_float((uint32_t)a.bias[at] << 16);
            bias[1][e] = __uint_as_float((uint32_t)a.bias[a.N + at] << 16);
        }
#pragma unroll
    for (int f = 0; f < NB; ++f) *reinterpret_cast<f32x4*>(sums[wave][f][lane]) = acc[f];
    __syncthreads();
    if (wave != 0 || li >= a.M || valid <= 0) return;
    const GateForm form = gate_form(a.act);
    uint16_t out[3][4];
    f32x4 s[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        const int from = COLS < 16 && f ? lane + 4 * COLS : lane, block = COLS < 16 ? 0 : f;       // the up rows' sums lie COLS / 4 lane groups further on
        s[f] = *reinterpret_cast<const f32x4*>(sums[0][block][from]);
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) s[f] += *reinterpret_cast<const f32x4*>(sums[w][block][from]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float g = s[0][e] + bias[0][e], u = s[1][e] + bias[1][e];
        out[0][e] = (uint16_t)f32_to_bf16_rne((a.act == RTL_ACT_GELU ? gate_value<true>(g, form) : gate_value<false>(g, form)) * u);
        out[1][e] = (uint16_t)f32_to_bf16_rne(g);
        out[2][e] = (uint16_t)f32_to_bf16_rne(u);
    }
    uint16_t* const to[3] = {a.Y + li * a.ldy + col, a.P + li * a.ldp + col, a.P + li * a.ldp + a.N + col};
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        if (k > 0 && !a.P) break;
        if (valid == 4) {
            __builtin_memcpy(to[k], out[k], 8);                                                  // (at any address)
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < valid) to[k][e] = out[k][e];
        }
    }
}

// dP = [dH U act'(G), dH act(G)] and, with H set, H = act(G) U again. Eight columns to a thread, F a multiple of four, rows of any 8-byte alignment. Bound by
// memory: five or six values of two bytes per element of H. dP is rounded to bf16, the type that the matrix cores take in the products behind it.
constexpr int kGradThreads = 256;
template <bool ERF>
__global__ __launch_bounds__(kGradThreads) void gated_grad_kernel(const GatedGradArgs a) {
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

// Runs `op` (launch or prepare) of small tile `i` of gemm.hip's kGatedShapes.
template <class Op>
hipError_t with_gated(int i, Op op) {
    switch (i) {
        case 0: return op(Gated<32, 32, 1, 1, 4, 4>{});
        case 1: return op(Gated<64, 32, 1, 1, 4, 3>{});
        case 2: return op(Gated<64, 64, 1, 2, 2, 4>{});
        case 3: return op(Gated<128, 64, 2, 2, 2, 3>{});
        case 4: return op(Gated<128, 128, 4, 2, 1, 3>{});
        case 5: return op(Gated<96, 128, 2, 2, 1, 3>{});
        default: return op(Gated<64, 64, 2, 2, 1, 3>{});
    }
}
using Gated256 = GatedMixed<256, 2, 4>;
using Gated192 = GatedMixed<192, 4, 2>;

}  // namespace

hipError_t launch_gated(const GemmArgs& a_in, hipStream_t stream) {
    GemmArgs a = a_in;
    if (a.M <= kFewRows && a.N < (int64_t)1 << 27) {               // (a launch takes fewer than 2^32 threads)
        auto go = [&](auto cols) {
            constexpr int C = decltype(cols)::value;
            hipLaunchKernelGGL(gated_few_rows_kernel<C>, dim3((unsigned)((a.N + C - 1) / C)), dim3(kFewWaves * 64), 0, stream, a);
            return hipGetLastError();
        };
        // Eight columns to a workgroup where sixteen leave units idle, and, with X small beside them, for long rows of W. us, 16 | 8 columns: [16, 700, 4096]
        // 12.8 | 9.5, [1, 1500, 2944] 8.1 | 5.7, [1, 2816, 2048] 6.8 | 7.0, [16, 3000, 1024] 5.3 | 6.1, [1, 10240, 3840] 27.1 | 23.9, [4, 10240, 3840] 28.1 |
        // 26.8, [8, 10240, 3840] 29.2 | 29.8, [2, 8192, 1024] 7.1 | 7.5. (Four columns, and eight or sixteen waves, are not quicker.)
        return a.N <= 2048 || (a.M <= 4 && a.K > 2048) ? go(std::integral_constant<int, 8>{}) : go(std::integral_constant<int, 16>{});
    }
    const GatedForm form = gated_form(a.M, a.N, a.K);
    if (form.shape >= 0) return with_gated(form.shape, [&](auto k) { return decltype(k)::launch(a, stream); });
    a.m_split = form.m_split;
    a.body_tiles = form.body_tiles;
    a.tail_tiles = form.tail_tiles;
    return form.use_192 ? Gated192::launch(a, stream) : Gated256::launch(a, stream);
}

int64_t gated_grad_grid(int64_t M, int64_t F) { return (M * ((F + 7) / 8) + kGradThreads - 1) / kGradThreads; }
hipError_t launch_gated_grad(const GatedGradArgs& a, hipStream_t stream) {
    const int64_t grid = gated_grad_grid(a.M, a.F);
    if (grid == 0) return hipSuccess;
    const dim3 g((unsigned)grid);
    if (a.act == RTL_ACT_GELU) hipLaunchKernelGGL(gated_grad_kernel<true>, g, dim3(kGradThreads), 0, stream, a);
    else hipLaunchKernelGGL(gated_grad_kernel<false>, g, dim3(kGradThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t prepare_gated_kernels() {
    hipError_t e = Gated256::prepare();
    if (e == hipSuccess) e = Gated192::prepare();
    for (int i = 0; i < 7 && e == hipSuccess; ++i) e = with_gated(i, [](auto k) { return decltype(k)::prepare(); });
    return e;
}

}  // namespace rtl
