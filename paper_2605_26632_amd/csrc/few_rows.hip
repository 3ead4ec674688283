// Linears of few rows (single tokens, decoding steps, experts with a row or two): Y = X W^T where reading W is all there is.
//
// No operand passes through LDS on its way to the matrix cores: W is the FIRST matrix operand, and a lane loads its 16-byte chunks straight into
// the registers that the instruction reads (lane l holds row l % 16 of 16 rows of W, chunk l / 16 of four). Up to 16 rows of X are the second one. A workgroup owns
// 16 NB columns of Y; its waves divide the contraction in units of a 128-byte line per row of W, neighbouring waves on neighbouring lines, and each
// has four lines per row in flight. The waves' sums meet in LDS, in a fixed order.
// 4-bit operands: X is quantised by every workgroup for itself into LDS (a few KB that come from L2), which spares the launch that would do only
// this; one launch and no workspace. The arithmetic is that of the tile loop (gemm_tile.h).
#include <initializer_list>
#include "groups.h"
#include "mx_codes.h"

namespace rtl {
namespace {

constexpr int kFewRows = 16;             // rows of X at a time
constexpr int kFewLds = 64 * 1024;       // most LDS of a workgroup

// X as the second operand in LDS (4-bit): rows of K / 2 bytes rounded up to whole units, 16 bytes further apart so that they start in different banks.
__host__ __device__ inline int64_t few_code_pitch(int64_t K) { return (K + 255) / 256 * 128 + 16; }
__host__ __device__ inline int64_t few_scale_pitch(int64_t K) { return (K + 255) / 256 * 8; }

__host__ __device__ inline int64_t few_lds_rows(int64_t M) { return M < kFewRows ? M : kFewRows; }

// rows [0, a.M) of X times columns [n0, n0 + 16 NB) of Y. QUANT: 4-bit product of a bf16 X; without it X is what the product takes (the same sums).
template <bool FP4, bool QUANT, int NB, int WAVES, int U>
__device__ __forceinline__ void few_rows(const GemmArgs& a, const int64_t n0, uint8_t* smem) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, kb = lane >> 4;
    const int units = (int)(FP4 ? (a.K + 255) / 256 : a.K / 64), blocks = (int)(a.K / 32);
    float* const sums = reinterpret_cast<float*>(smem);                                    // [WAVES][NB][64][4]
    uint8_t* const xq = smem + WAVES * NB * 1024;
    uint8_t* const xs = xq + few_lds_rows(a.M) * few_code_pitch(a.K);
    const uint8_t* w_row[NB];
    const uint8_t* ws_row[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int64_t n = min(n0 + b * 16 + li, a.N - 1);
        w_row[b] = static_cast<const uint8_t*>(a.W) + n * a.ldw * (FP4 ? 1 : 2) + kb * 32;
        if constexpr (FP4) ws_row[b] = a.w_scale + n * 8 + kb * 2;
    }
    // the wave's lines of W from unit u0 on, and their scales
    uint4 w[U][NB][2];
    uint32_t sw[U][NB];
    auto load_w = [&](int u0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = min(u0 + u * WAVES, units - 1);                               // (beyond the end: loaded again, not used)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint8_t* p = w_row[b] + (int64_t)unit * 128;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    // a lane's two chunks are neighbours. 4-bit: one behind K is left out
                    if constexpr (FP4) {
                        w[u][b][c] = make_uint4(0, 0, 0, 0);
                        if (unit * 8 + 2 * kb + c < blocks) w[u][b][c] = *reinterpret_cast<const uint4*>(p + c * 16);
                    } else {
                        w[u][b][c] = *reinterpret_cast<const uint4*>(p + c * 16);
                    }
                }
                if constexpr (FP4) sw[u][b] = *reinterpret_cast<const uint16_t*>(ws_row[b] + (int64_t)unit * a.w_scale_rows * 8);
            }
        }
    };
    for (int64_t m0 = 0; m0 < a.M; m0 += kFewRows) {
        const int rows = (int)min((int64_t)kFewRows, a.M - m0);
        load_w(wave);                                                                      // under way while X is quantised
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (QUANT) {
            // eight values per thread, a block of 32 in four neighbouring lanes; zeros up to the end of the last unit
            const int pieces = units * 32;
            for (int q = tid; q < rows * pieces; q += WAVES * 64) {                   // (pieces: whole multiples of four per row)
                const int r = q / pieces, c = q % pieces;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (c * 8 < a.K) v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.A) + (m0 + r) * a.lda + c * 8);
                const uint32_t byte = row_scale_byte(v);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                *reinterpret_cast<uint32_t*>(xq + r * few_code_pitch(a.K) + c * 4) = codes8(w, byte);
                if ((c & 3) == 0) xs[r * few_scale_pitch(a.K) + c / 4] = (uint8_t)byte;
            }
            __syncthreads();
        }
        const int xr = min(li, rows - 1);                                                  // rows behind the last one repeat it, for outputs never stored
        f32x4 acc[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int u0 = wave; u0 < units; u0 += WAVES * U) {
            uint4 x[U][2];
            uint32_t sx[U];
            if (u0 != wave) load_w(u0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int unit = min(u0 + u * WAVES, units - 1);
                if constexpr (!QUANT) {
                    const uint8_t* p = static_cast<const uint8_t*>(a.A) + (m0 + xr) * a.lda * (FP4 ? 1 : 2) + (int64_t)unit * 128 + kb * 32;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (FP4 && unit * 8 + 2 * kb + c >= blocks) x[u][c] = make_uint4(0, 0, 0, 0);
                        else x[u][c] = *reinterpret_cast<const uint4*>(p + c * 16);
                    }
                    if constexpr (FP4) sx[u] = *reinterpret_cast<const uint16_t*>(a.a_scale + ((int64_t)unit * a.a_scale_rows + m0 + xr) * 8 + kb * 2);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u == 0) __builtin_amdgcn_sched_barrier(0);                             // all the loads first
                const int unit = u0 + u * WAVES;
                if (unit >= units) break;
                if constexpr (FP4) {
                    // scale bytes behind K count as zero, whatever the caller's hold: no NaN may come from there
                    const int left = blocks - (unit * 8 + 2 * kb);
                    const uint32_t keep = left >= 2 ? 0xFFFFu : left == 1 ? 0xFFu : 0u;
                    if constexpr (QUANT) {
                        const uint8_t* p = xq + xr * few_code_pitch(a.K) + unit * 128 + kb * 32;
#pragma unroll
                        for (int c = 0; c < 2; ++c) x[u][c] = *reinterpret_cast<const uint4*>(p + c * 16);
                        sx[u] = *reinterpret_cast<const uint16_t*>(xs + xr * few_scale_pitch(a.K) + unit * 8 + kb * 2);
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        acc[b] = fp4_mma<0, 0>(w[u][b][0], x[u][0], acc[b], (int)(sw[u][b] & keep), (int)(sx[u] & keep));
                        acc[b] = fp4_mma<1, 1>(w[u][b][1], x[u][1], acc[b], (int)(sw[u][b] & keep), (int)(sx[u] & keep));
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            Frag8 fw, fx;
                            fw.u = w[u][b][c];
                            fx.u = x[u][c];
                            acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw.v, fx.v, acc[b], 0, 0, 0);
                        }
                }
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(sums + ((wave * NB + b) * 64 + lane) * 4) = acc[b];
        __syncthreads();
        if (tid < NB * 64) {
            // row m = lane % 16 of X, columns 4 (lane / 16) .. of the 16
            f32x4 s = *reinterpret_cast<const f32x4*>(sums + tid * 4);
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += *reinterpret_cast<const f32x4*>(sums + (w * NB * 64 + tid) * 4);
            const int64_t n = n0 + tid / 64 * 16 + 4 * kb;
            const int valid = (int)min((int64_t)4, a.N - n);
            if (li < rows && valid > 0) {
                uint16_t* dst = a.Y + (m0 + li) * a.ldy + n;
                uint32_t out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float y = s[e];
                    if (a.bias) y += __uint_as_float((uint32_t)a.bias[n + min(e, valid - 1)] << 16);
                    out[e] = f32_to_bf16_rne(y);
                }
                const uint2 four = make_uint2(out[0] | out[1] << 16, out[2] | out[3] << 16);
                if (valid == 4) {
                    __builtin_memcpy(dst, &four, 8);                                       // (at any address)
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < valid) dst[e] = (uint16_t)out[e];
                }
            }
        }
        if (m0 + kFewRows < a.M) __syncthreads();                                          // the sums and X's codes are written again
    }
}

extern __shared__ __align__(16) uint8_t few_smem[];

template <bool QUANT, int NB, int WAVES, int U>
__global__ __launch_bounds__(WAVES * 64) void few_rows_kernel(const GemmArgs a) {
    few_rows<true, QUANT, NB, WAVES, U>(a, (int64_t)blockIdx.x * (16 * NB), few_smem);
}

template <bool FP4, bool QUANT, int NB, int WAVES, int U>
__global__ __launch_bounds__(WAVES * 64) void grouped_few_rows_kernel(const GemmArgs a, const GroupArgs g) {
    const int blocks = (int)((a.N + 16 * NB - 1) / (16 * NB)), e = (int)blockIdx.x / blocks;
    const RowRange r = expert_rows(g.offsets, e, (int)a.M);
    if (r.begin == r.end) return;
    GemmArgs b = a;
    b.M = r.end - r.begin;
    b.A = static_cast<const uint8_t*>(a.A) + r.begin * a.lda * (FP4 && !QUANT ? 1 : 2);
    b.W = static_cast<const uint8_t*>(a.W) + e * g.w_stride * (FP4 ? 1 : 2);
    b.Y = a.Y + r.begin * a.ldy;
    if (a.bias) b.bias = a.bias + e * a.N;
    if constexpr (FP4) {
        b.w_scale = a.w_scale + e * a.N * 8;
        if constexpr (!QUANT) b.a_scale = a.a_scale + (int64_t)r.begin * 8;
    }
    few_rows<FP4, QUANT, NB, WAVES, U>(b, (int64_t)(blockIdx.x % blocks) * (16 * NB), few_smem);
}

template <bool FP4, bool QUANT, int NB, int WAVES, int U>
struct Few {
    static int64_t lds(int64_t M, int64_t K) { return WAVES * NB * 1024 + (QUANT ? few_lds_rows(M) * (few_code_pitch(K) + few_scale_pitch(K)) : 0); }
    static int64_t blocks(int64_t N) { return (N + 16 * NB - 1) / (16 * NB); }
    static hipError_t prepare() {
        auto limit = [](const void* k) { return hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, kFewLds); };
        hipError_t e = limit(reinterpret_cast<const void*>(grouped_few_rows_kernel<FP4, QUANT, NB, WAVES, U>));
        if constexpr (FP4 && NB == 1)
            if (e == hipSuccess) e = limit(reinterpret_cast<const void*>(few_rows_kernel<QUANT, NB, WAVES, U>));
        return e;
    }
    static hipError_t launch(const GemmArgs& a, hipStream_t stream) {
        hipLaunchKernelGGL((few_rows_kernel<QUANT, NB, WAVES, U>), dim3((unsigned)blocks(a.N)), dim3(WAVES * 64), (size_t)lds(a.M, a.K), stream, a);
        return hipGetLastError();
    }
    static hipError_t launch(const GemmArgs& a, const GroupArgs& g, hipStream_t stream) {
        hipLaunchKernelGGL((grouped_few_rows_kernel<FP4, QUANT, NB, WAVES, U>), dim3((unsigned)(g.experts * blocks(a.N))), dim3(WAVES * 64),
                           (size_t)lds(a.M, a.K), stream, a, g);
        return hipGetLastError();
    }
};
// 16 columns and eight lines of W per row in flight in a workgroup; 4-bit stacks of experts that fill the chip several times over take more columns per
// workgroup instead, fewer lines (kWide columns and more of experts that can have rows). us, [T, E, N, K] 4-bit, quantised inside: NB 1 U 2 | NB 4 U 1 | NB 4 U 2
// | NB 2 U 4: [24, 32, 2816, 2048] 12.1 | 11.1 | 13.9 | 20.4, [64, ..] 24.3 | 19.5; from codes NB 1 U 2 | NB 2 U 2: [64, ..] 23.0 | 20.2, [200, ..] 23.6 | 21.1. One row,
// [12288, 3072], launches back to back on one weight (7.2 traced one by one): NB 1 U 2 6.2, NB 1 U 4 6.7, NB 2 U 2 7.1, NB 4 U 2 7.4; eight waves 6.3
// to 8.5. bf16 [24, 32, 1408, 1024]: NB 1 U 4 9.2, U 2 10.8, NB 2 U 4 9.4, NB 4 U 4 12.4.
using FewQuant = Few<true, true, 1, 4, 2>;
using FewQuantWide = Few<true, true, 4, 4, 1>;
using FewCodes = Few<true, false, 1, 4, 2>;
using FewCodesWide = Few<true, false, 2, 4, 2>;
using FewBf16 = Few<false, false, 1, 4, 4>;
// (Just under the smallest stack that was better off wide, 24 x 2816 columns; 12288 columns were not; nothing between them is measured.)
constexpr int64_t kWide = 65536;

}  // namespace

FewRows few_rows_choice(int64_t M, int64_t most, int64_t K, bool fp4) {
    if (M > kFewRows) return FewRows::no;
    if (!fp4) return FewRows::direct;
    // Quantised by each workgroup for itself while there is little to quantise: one launch instead of two (2.5 us and the gap). [M, 12288, 3072], inside |
    // from codes: M = 1 6.3 | 6.4, 2 6.6 | 6.8, 8 10.3 | 7.6; [1, 3072, 12288] 7.9 | 7.0, [2, 3072, 12288] 10.1 | 7.1.
    return M * K <= 8192 && FewQuantWide::lds(most, K) <= kFewLds ? FewRows::quantise : FewRows::direct;
}

// us of a grouped launch that cannot be shorter than `stream` us: its workgroups, three to a unit at a time, each as long as its batches of lines and its
// expert's 16-row blocks (an expert of one and a half times the average rows). More than two rounds of workgroups read at a lower rate than tiles do: bf16
// [64, 64, 1024, 2048] 37.5 us against 29.5 with panels, where [24, 32, 1408, 1024], two rounds, takes 12.0 against 14.2 with 64 x 64 tiles (changing inputs).
// (An expert of many times the average is not priced, the offsets are on the device: 4-bit [512, 64, 1408, 1024] 16 us even, 48 with a quarter of the rows
// on one expert, 139 with all.)
double few_rows_us(int64_t T, int64_t E, int64_t N, int64_t K, bool fp4, double stream) {
    const double experts = group_experts(T, E), rows = (double)T / experts, cols = fp4 && (double)(E < T ? E : T) * (double)N >= (double)kWide ? 32 : 16;
    const double many = rows * 1.5 / 16, batches = (double)(fp4 ? (K + 2047) / 2048 : (K + 1023) / 1024);
    const double waves = experts * (double)(int64_t)(((double)N + cols - 1) / cols) / (256 * 3);
    const double chain = 2.0 + (waves > 1 ? waves : 1) * ((fp4 ? 1.0 : 2.0) + 1.4 * batches) * (many > 1 ? many : 1);
    const double read = stream * (waves > 2 ? 1 + 0.1 * (waves - 2) : 1);
    return chain > read ? chain : read;
}

hipError_t prepare_few_rows_kernels() {
    for (hipError_t e : {FewQuant::prepare(), FewQuantWide::prepare(), FewCodes::prepare(), FewCodesWide::prepare(), FewBf16::prepare()})
        if (e != hipSuccess) return e;
    return hipSuccess;
}
hipError_t launch_few_rows(const GemmArgs& a, hipStream_t stream) { return a.a_scale ? FewCodes::launch(a, stream) : FewQuant::launch(a, stream); }
hipError_t launch_grouped_few_rows(const GemmArgs& a, const GroupArgs& g, hipStream_t stream) {
    if (!a.fp4) return FewBf16::launch(a, g, stream);
    const bool wide = (a.M < g.experts ? a.M : g.experts) * a.N >= kWide;
    if (a.a_scale) return wide ? FewCodesWide::launch(a, g, stream) : FewCodes::launch(a, g, stream);
    return wide ? FewQuantWide::launch(a, g, stream) : FewQuant::launch(a, g, stream);
}
int64_t few_rows_grid(int64_t E, int64_t N) { return E * FewBf16::blocks(N); }

}  // namespace rtl
