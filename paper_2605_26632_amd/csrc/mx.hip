// Microscaled 4-bit floating point: E2M1 codes, two to a byte (even index in the low half), and for every 32 of them along the contraction
// a power of two, kept as its biased exponent. Quantiser (rows, columns, or both in one read) and its inverse.
//
//   e = floor(log2 max|x|) - 2 over the 32, at least -127;  code = E2M1 nearest to x / 2^e (ties to the even code, at most 6)
//
// In bf16 bits floor(log2 max|x|) is the exponent field of the largest magnitude: the scale byte is max(field - 2, 0). The division by the
// power of two, the rounding and the saturation are one conversion instruction for two values. A block with a NaN or an infinity gets the
// scale byte 0xFF (NaN), which makes all of it NaN: no finite value stands for something that was not finite.
// All of it is bound by memory: 2 bytes read and 17/32 written per value and direction. The same inputs again and again (so partly in the MALL):
// rows [4608, 12288] 21.0 us = 6.8 TB/s, back 22.6 us = 6.3 TB/s; columns and rows of [2111, 2048] in one read 7.7 us (144 workgroups: latency).
#include "mx_codes.h"

namespace rtl {
namespace {

// Along the rows. A workgroup takes 256 columns (one record of eight scale bytes) of 32 rows, four 16-byte loads per thread in flight; the
// records of its rows are one run of 256 bytes.
constexpr int kQuantRows = 32;
__global__ __launch_bounds__(256) void quantize_rows_kernel(const uint16_t* X, int64_t rows, int64_t cols, int64_t ld, uint8_t* Q, int64_t ldq,
                                                            uint8_t* S) {
    const int64_t col_blocks = (cols + 255) / 256;
    const int64_t cb = blockIdx.x % col_blocks, r0 = blockIdx.x / col_blocks * kQuantRows + threadIdx.x / 32;
    const int64_t col = cb * 256 + (threadIdx.x % 32) * 8;
    uint4 v[kQuantRows / 8];
#pragma unroll
    for (int p = 0; p < kQuantRows / 8; ++p) {
        v[p] = make_uint4(0, 0, 0, 0);
        if (r0 + 8 * p < rows && col < cols) v[p] = *reinterpret_cast<const uint4*>(X + (r0 + 8 * p) * ld + col);
    }
#pragma unroll
    for (int p = 0; p < kQuantRows / 8; ++p) {
        const int64_t row = r0 + 8 * p;
        const uint32_t byte = row_scale_byte(v[p]);
        const uint32_t word = word_of_bytes(byte);
        if (row >= rows) continue;
        if ((threadIdx.x & 15) == 0) *reinterpret_cast<uint32_t*>(S + (cb * rows + row) * 8 + (threadIdx.x & 16) / 4) = word;
        const uint32_t w[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
        if (col < cols) *reinterpret_cast<uint32_t*>(Q + row * ldq + col / 2) = codes8(w, byte);
    }
}

// Down the columns, the result transposed; with Q also along the rows from the same read. A workgroup takes 256 rows (one record of the
// transposed scales) of 128 columns through LDS; a thread then owns 32 rows of two neighbouring columns. Rows of the tile are 256 bytes,
// each 32 of them moved on by 32 bytes, so that the eight row blocks and eight column pairs of a wave's read meet 64 banks.
constexpr int kTRows = 256, kTCols = 128;
__device__ __forceinline__ int t_word(int row, int pair) { return row * (kTCols / 2) + (row / 32) * 8 + pair; }
__global__ __launch_bounds__(512) void quantize_cols_kernel(const uint16_t* X, int64_t rows, int64_t cols, int64_t ld, uint8_t* Q, int64_t ldq,
                                                            uint8_t* S, uint8_t* Qt, int64_t ldqt, uint8_t* St) {
    __shared__ __align__(16) uint32_t tile[kTRows * kTCols / 2 + 8 * 8];
    const int64_t col_blocks = (cols + kTCols - 1) / kTCols;
    const int64_t c0 = blockIdx.x % col_blocks * kTCols, rb0 = blockIdx.x / col_blocks, r0 = rb0 * kTRows;
    const int tid = threadIdx.x;
    {
        const int chunk = tid % 16;
        const int64_t col = c0 + chunk * 8;
        uint4 v[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const int64_t row = r0 + p * 32 + tid / 16;
            v[p] = make_uint4(0, 0, 0, 0);
            if (row < rows && col < cols) v[p] = *reinterpret_cast<const uint4*>(X + row * ld + col);
        }
#pragma unroll
        for (int p = 0; p < 8; ++p) *reinterpret_cast<uint4*>(tile + t_word(p * 32 + tid / 16, chunk * 4)) = v[p];
        if (Q) {
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                const int64_t row = r0 + p * 32 + tid / 16;
                const uint32_t byte = row_scale_byte(v[p]);
                const uint32_t word = word_of_bytes(byte);
                if (row >= rows) continue;
                uint32_t* rec = reinterpret_cast<uint32_t*>(S + (c0 / 256 * rows + row) * 8 + c0 % 256 / 32);
                if (chunk == 0) *rec = word;
                if (chunk == 0 && c0 % 256 == 0 && c0 + kTCols >= cols) rec[1] = 0;      // no tile has the record's other half
                const uint32_t w[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
                if (col < cols) *reinterpret_cast<uint32_t*>(Q + row * ldq + col / 2) = codes8(w, byte);
            }
        }
    }
    __syncthreads();
    const int rb = tid % 8, pair = tid / 8;
    const int64_t col = c0 + 2 * pair;
    if (col >= cols) return;
    uint32_t w[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) w[i] = tile[t_word(rb * 32 + i, pair)];
    u16x2 m = magnitudes(w[0]);
#pragma unroll
    for (int i = 1; i < 32; ++i) m = max2(m, magnitudes(w[i]));
    const bool inside = r0 + rb * 32 < rows;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t byte = scale_byte(m[h]);
        St[(rb0 * cols + col + h) * 8 + rb] = (uint8_t)byte;
        uint32_t out[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)        // rows 2 e, 2 e + 1 of the eight
                p[e] = __builtin_amdgcn_perm(w[8 * q + 2 * e + 1], w[8 * q + 2 * e], h ? 0x07060302u : 0x05040100u);
            out[q] = codes8(p, byte);
        }
        if (inside) *reinterpret_cast<uint4*>(Qt + (col + h) * ldqt + r0 / 2 + rb * 16) = make_uint4(out[0], out[1], out[2], out[3]);
    }
}

// The values of the codes. A thread turns eight codes into 16 bytes.
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t* Q, int64_t ldq, const uint8_t* S, int64_t rows, int64_t cols, uint16_t* X,
                                                         int64_t ld) {
    const int64_t chunks = cols / 8, all = rows * chunks;
    for (int64_t n = blockIdx.x * (int64_t)256 + threadIdx.x; n < all; n += (int64_t)gridDim.x * 256) {
        const int64_t row = n / chunks, c = n % chunks;
        const uint32_t q = *reinterpret_cast<const uint32_t*>(Q + row * ldq + c * 4);
        const uint32_t byte = S[(c / 32 * rows + row) * 8 + c / 4 % 8];
        const float s = byte == 255 ? __uint_as_float(0x7FC00000u) : scale_value(byte);
        uint32_t out[4];
        auto two = [&](f32x2 v) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[0] * s, v[1] * s}, bf16x2)); };
        out[0] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0));
        out[1] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1));
        out[2] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2));
        out[3] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3));
        *reinterpret_cast<uint4*>(X + row * ld + c * 8) = make_uint4(out[0], out[1], out[2], out[3]);
    }
}

}  // namespace

hipError_t prepare_mx_kernels() {
    for (const void* k : {reinterpret_cast<const void*>(quantize_rows_kernel), reinterpret_cast<const void*>(quantize_cols_kernel),
                          reinterpret_cast<const void*>(dequantize_kernel)}) {
        hipFuncAttributes attr;
        const hipError_t e = hipFuncGetAttributes(&attr, k);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// (whatever directions are asked for, so that a matrix that goes along its rows also goes down its columns)
bool quantize_mxfp4_fits(int64_t rows, int64_t cols) {
    const int64_t along = ((rows + kQuantRows - 1) / kQuantRows) * ((cols + 255) / 256) * 256;
    const int64_t down = ((rows + kTRows - 1) / kTRows) * ((cols + kTCols - 1) / kTCols) * 512;
    return along < (int64_t)1 << 32 && down < (int64_t)1 << 32;
}

hipError_t launch_quantize_mxfp4(const uint16_t* X, int64_t rows, int64_t cols, int64_t ld, uint8_t* Q, int64_t ldq, uint8_t* S, uint8_t* Qt,
                                 int64_t ldqt, uint8_t* St, hipStream_t stream) {
    if (Qt) {
        const int64_t grid = ((rows + kTRows - 1) / kTRows) * ((cols + kTCols - 1) / kTCols);
        hipLaunchKernelGGL(quantize_cols_kernel, dim3((unsigned)grid), dim3(512), 0, stream, X, rows, cols, ld, Q, ldq, S, Qt, ldqt, St);
    } else {
        const int64_t grid = ((rows + kQuantRows - 1) / kQuantRows) * ((cols + 255) / 256);
        hipLaunchKernelGGL(quantize_rows_kernel, dim3((unsigned)grid), dim3(256), 0, stream, X, rows, cols, ld, Q, ldq, S);
    }
    return hipGetLastError();
}

hipError_t launch_dequantize_mxfp4(const uint8_t* Q, int64_t ldq, const uint8_t* S, int64_t rows, int64_t cols, uint16_t* X, int64_t ld,
                                   hipStream_t stream) {
    const int64_t want = (rows * (cols / 8) + 255) / 256;
    hipLaunchKernelGGL(dequantize_kernel, dim3((unsigned)(want < 16384 ? want : 16384)), dim3(256), 0, stream, Q, ldq, S, rows, cols, X, ld);
    return hipGetLastError();
}

}  // namespace rtl
