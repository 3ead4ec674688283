// Norm and rotary positions of the heads of q and k, in one pass over both, and their gradients.
//
//   forward   n = w q / sqrt(mean q^2 + eps) (or q itself); with the angle pos[t, axis[j]] freq[j] pair j of n is turned by it, (a, b) -> (a cos - b sin,
//             a sin + b cos); pairs are (2 j, 2 j + 1) or (j, j + pairs), what lies behind the pairs passes
//   backward  the gradient is turned back by the angle; dw += d q r, and through the norm: dq = r (w d - q r mean(w d q r)), r = 1 / sqrt(mean q^2 + eps)
//
// Bound by memory (each head read once and written once). An angle belongs to a token: a lane holds 16 values of a head, so that the eight pairs that
// they make are the same for all heads of the token, and their sines are taken once per wave. The product of position and frequency is exact in 64
// bits and cut to a quarter turn there, since in 32 a far position's angle would be off by 2^-24 of itself; the rest is fp32.
#include "rtl_internal.h"

namespace rtl {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kHeadWaves = 4;            // waves of a workgroup

__device__ __forceinline__ void unpack(const uint4 v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(w[e] << 16);
        f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const f32x2 v = {f[2 * e], f[2 * e + 1]};
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));       // RNE
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Sum over the L neighbouring lanes of a head, in all of them.
template <int L>
__device__ __forceinline__ float head_sum(float v) {
    auto add = [&](auto ctrl) { v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(ctrl)::value, 0xF, 0xF, true)); };
    if constexpr (L >= 2) add(std::integral_constant<int, 0xB1>{});          // the neighbour, the other pair, the other four, the other eight
    if constexpr (L >= 4) add(std::integral_constant<int, 0x4E>{});
    if constexpr (L >= 8) add(std::integral_constant<int, 0x141>{});
    if constexpr (L >= 16) add(std::integral_constant<int, 0x140>{});
    if constexpr (L >= 32) v += __shfl_xor(v, 16);
    return v;
}

// Sine and cosine of pos * freq (exact product). The angle less the nearest multiple of a quarter turn, pi / 2 in two doubles, lies in [-pi/4, pi/4]; there the
// Taylor series to the ninth and the tenth power are off by less than 2e-9.
__device__ __forceinline__ void turn(float pos, float freq, float& sn, float& cs) {
    const double t = (double)pos * (double)freq;
    const double n = rint(t * 0.63661977236758134308);
    const float r = (float)fma(-n, 6.123233995736766e-17, fma(-n, 1.5707963267948966, t));
    const int quarter = (int)(n - 4.0 * floor(n * 0.25));
    const float r2 = r * r;
    const float s = r + r * r2 * (-1.6666667e-1f + r2 * (8.3333333e-3f + r2 * (-1.9841270e-4f + r2 * 2.7557319e-6f)));
    const float c = 1.0f + r2 * (-0.5f + r2 * (4.1666667e-2f + r2 * (-1.3888889e-3f + r2 * (2.4801587e-5f - r2 * 2.7557319e-7f))));
    const bool swap = quarter & 1;
    const float a = swap ? c : s, b = swap ? s : c;
    sn = quarter & 2 ? -a : a;
    cs = (quarter + 1) & 2 ? -b : b;
}

// What a lane does in every head: its two chunks of eight values (first value, or -1 for none), whether they turn, and its eight pairs' sines. HALVES: element e of
// the first chunk and of the second are pair e; else a chunk holds four pairs, of which the lane has the two chunks' eight.
struct LanePlan {
    int at[2];
    bool turns[2];
    int pair0;
};
template <bool HALVES>
__device__ __forceinline__ LanePlan lane_plan(int c, int D, int pairs) {
    LanePlan p;
    const int chunks = D / 8;
    if constexpr (HALVES) {
        const int half = pairs / 8;
        if (c < half) {
            p = LanePlan{{c * 8, (c + half) * 8}, {true, true}, c * 8};
        } else {
            const int rest = 2 * half + 2 * (c - half);
            p = LanePlan{{rest < chunks ? rest * 8 : -1, rest + 1 < chunks ? (rest + 1) * 8 : -1}, {false, false}, 0};
        }
    } else {
        const int i = 2 * c;
        p = LanePlan{{i < chunks ? i * 8 : -1, i + 1 < chunks ? (i + 1) * 8 : -1}, {i * 4 < pairs, i * 4 + 4 < pairs}, c * 8};
    }
    return p;
}

template <bool HALVES>
__device__ __forceinline__ void lane_turns(const RotaryArgs& a, const LanePlan& p, int64_t token, float (&sn)[8], float (&cs)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sn[e] = 0.f;
        cs[e] = 1.f;
        if (p.turns[HALVES ? 0 : e / 4]) {
            const int j = p.pair0 + e, ax = min(max(a.axis[j], 0), a.axes - 1);
            turn(a.pos[token * a.axes + ax], a.freq[j], sn[e], cs[e]);
        }
    }
}

// Both chunks turned; BACK: by the negative angle.
template <bool HALVES, bool BACK>
__device__ __forceinline__ void apply_turns(float (&v)[2][8], const float (&sn)[8], const float (&cs)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float& x = HALVES ? v[0][e] : v[e / 4][2 * (e % 4)];
        float& y = HALVES ? v[1][e] : v[e / 4][2 * (e % 4) + 1];
        const float s = BACK ? -sn[e] : sn[e], p = x * cs[e] - y * s, q = x * s + y * cs[e];
        x = p;
        y = q;
    }
}

__device__ __forceinline__ void load_chunks(const uint16_t* p, const LanePlan& plan, float (&v)[2][8]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = 0.f;
        if (plan.at[c] >= 0) unpack(*reinterpret_cast<const uint4*>(p + plan.at[c]), v[c]);
    }
}
__device__ __forceinline__ void store_chunks(uint16_t* p, const LanePlan& plan, const float (&v)[2][8]) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (plan.at[c] >= 0) *reinterpret_cast<uint4*>(p + plan.at[c]) = pack(v[c]);
}
__device__ __forceinline__ float square_sum(const float (&v)[2][8]) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[c][e] * v[c][e];
    return s;
}

// A wave takes one token and a.heads_per heads of it (those of q, then those of k), 64 / L at a time.
template <int L, bool HALVES>
__global__ __launch_bounds__(kHeadWaves * 64) void rotary_kernel(const RotaryArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t task = (int64_t)blockIdx.x * kHeadWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t token = task / a.splits;
    if (token >= a.T) return;
    const int heads = a.Hq + a.Hk, h0 = (int)(task % a.splits) * a.heads_per, h1 = min(h0 + a.heads_per, heads);
    const LanePlan plan = lane_plan<HALVES>(lane % L, a.D, a.pairs);
    float sn[8], cs[8], w[2][2][8];
    lane_turns<HALVES>(a, plan, token, sn, cs);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint16_t* p = k ? a.wk : a.wq;
        if (p) {
            load_chunks(p, plan, w[k]);
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) w[k][c][e] = 1.0f;
        }
    }
    for (int h = h0 + lane / L; h < h1; h += 64 / L) {
        const bool is_k = h >= a.Hq;
        const uint16_t* from = is_k ? a.k + token * a.ldk + (h - a.Hq) * a.sk : a.q + token * a.ldq + h * a.sq;
        uint16_t* to = is_k ? a.k_out + token * a.ldko + (h - a.Hq) * a.sko : a.q_out + token * a.ldqo + h * a.sqo;
        float v[2][8];
        load_chunks(from, plan, v);
        if (a.norm) {
            const float r = 1.0f / sqrtf(head_sum<L>(square_sum(v)) / (float)a.D + a.eps);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[c][e] = v[c][e] * r * (is_k ? w[1][c][e] : w[0][c][e]);
        }
        apply_turns<HALVES, false>(v, sn, cs);
        store_chunks(to, plan, v);
    }
}

// The same walk for the gradients; a wave goes on to further tokens, and what it has of the weights' gradients goes to the workspace at the end, a
// workgroup's four waves and a wave's 64 / L heads added up in order.
template <int L, bool HALVES>
__global__ __launch_bounds__(kHeadWaves * 64) void rotary_backward_kernel(const RotaryArgs a) {
    __shared__ float part[kHeadWaves][2][L * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = a.Hq + a.Hk;
    const LanePlan plan = lane_plan<HALVES>(lane % L, a.D, a.pairs);
    float w[2][2][8], dw[2][2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint16_t* p = k ? a.wk : a.wq;
        if (p) load_chunks(p, plan, w[k]);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!p) w[k][c][e] = 1.0f;
                dw[k][c][e] = 0.f;
            }
    }
    const int64_t tasks = a.T * a.splits;
    for (int64_t task = (int64_t)blockIdx.x * kHeadWaves + wave; task < tasks; task += (int64_t)gridDim.x * kHeadWaves) {
        const int64_t token = task / a.splits;
        const int h0 = (int)(task % a.splits) * a.heads_per, h1 = min(h0 + a.heads_per, heads);
        float sn[8], cs[8];
        lane_turns<HALVES>(a, plan, token, sn, cs);
        for (int h = h0 + lane / L; h < h1; h += 64 / L) {
            const bool is_k = h >= a.Hq;
            const int64_t hk = h - a.Hq;
            float d[2][8];
            load_chunks(is_k ? a.dk_out + token * a.lddko + hk * a.sdko : a.dq_out + token * a.lddqo + h * a.sdqo, plan, d);
            apply_turns<HALVES, true>(d, sn, cs);
            if (a.norm) {
                float v[2][8];
                load_chunks(is_k ? a.k + token * a.ldk + hk * a.sk : a.q + token * a.ldq + h * a.sq, plan, v);
                const float r = 1.0f / sqrtf(head_sum<L>(square_sum(v)) / (float)a.D + a.eps);
                float m = 0.f;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[c][e] *= r;
                        const float dn = d[c][e] * v[c][e];
                        if (is_k) dw[1][c][e] += dn;
                        else dw[0][c][e] += dn;
                        d[c][e] *= is_k ? w[1][c][e] : w[0][c][e];
                        m += d[c][e] * v[c][e];
                    }
                m = head_sum<L>(m) / (float)a.D;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[c][e] = r * (d[c][e] - v[c][e] * m);
            }
            store_chunks(is_k ? a.dk + token * a.lddk + hk * a.sdk : a.dq + token * a.lddq + h * a.sdq, plan, d);
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = dw[k][c][e];
#pragma unroll
                for (int step = L; step < 64; step *= 2) s += __shfl_xor(s, step);
                if (lane < L && plan.at[c] >= 0) part[wave][k][plan.at[c] + e] = s;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.D; i += kHeadWaves * 64) {
        const int k = i / a.D, col = i % a.D;
        float s = part[0][k][col];
#pragma unroll
        for (int v = 1; v < kHeadWaves; ++v) s += part[v][k][col];
        a.sums[(int64_t)blockIdx.x * 2 * a.D + i] = s;
    }
}

// The workgroups' sums, 16 columns to a workgroup, dealt to its 16 lane groups in turn and those added in order.
__global__ __launch_bounds__(256) void rotary_reduce_kernel(const RotaryArgs a, const int groups) {
    __shared__ float part[16][16];
    const int i = blockIdx.x * 16 + (threadIdx.x & 15), g = threadIdx.x >> 4;
    float s = 0.f;
    if (i < 2 * a.D)
        for (int b = g; b < groups; b += 16) s += a.sums[(int64_t)b * 2 * a.D + i];
    part[g][threadIdx.x & 15] = s;
    __syncthreads();
    if (g != 0 || i >= 2 * a.D) return;
    for (int v = 1; v < 16; ++v) s += part[v][threadIdx.x & 15];
    if (i < a.D) {
        if (a.dwq) a.dwq[i] = s;
    } else if (a.dwk) {
        a.dwk[i - a.D] = s;
    }
}

// f(lanes of a head)
template <class F>
hipError_t with_lanes(int D, F f) {
    using std::integral_constant;
    if (D <= 64) return f(integral_constant<int, 4>{});
    if (D <= 128) return f(integral_constant<int, 8>{});
    if (D <= 256) return f(integral_constant<int, 16>{});
    return f(integral_constant<int, 32>{});
}

constexpr int64_t kBackwardGroups = 1024;    // workgroups of the backward pass at most

// Heads of a wave: all of a token's, fewer while there are not enough tokens to fill the chip with waves.
void deal_heads(RotaryArgs& a, int lanes) {
    const int heads = a.Hq + a.Hk, step = 64 / lanes;
    int per = (heads + step - 1) / step;
    while (per > 1 && a.T * ((heads + per * step - 1) / (per * step)) < 4096) per = (per + 1) / 2;
    a.heads_per = per * step;
    a.splits = (heads + a.heads_per - 1) / a.heads_per;
}

}  // namespace

size_t rotary_backward_scratch(int64_t D) { return (size_t)kBackwardGroups * 2 * (size_t)D * sizeof(float); }

hipError_t launch_rotary(const RotaryArgs& a_in, hipStream_t stream) {
    return with_lanes(a_in.D, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        RotaryArgs a = a_in;
        deal_heads(a, L);
        const dim3 grid((unsigned)((a.T * a.splits + kHeadWaves - 1) / kHeadWaves)), block(kHeadWaves * 64);
        if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<L, false>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((rotary_kernel<L, true>), grid, block, 0, stream, a);
        return hipGetLastError();
    });
}

hipError_t launch_rotary_backward(const RotaryArgs& a_in, hipStream_t stream) {
    int64_t groups = 0;
    hipError_t e = with_lanes(a_in.D, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        RotaryArgs a = a_in;
        deal_heads(a, L);
        groups = (a.T * a.splits + kHeadWaves - 1) / kHeadWaves;
        if (groups > kBackwardGroups) groups = kBackwardGroups;
        const dim3 grid((unsigned)groups), block(kHeadWaves * 64);
        if (groups == 0) return hipSuccess;
        if (a.interleaved) hipLaunchKernelGGL((rotary_backward_kernel<L, false>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((rotary_backward_kernel<L, true>), grid, block, 0, stream, a);
        return hipGetLastError();
    });
    if (e == hipSuccess && a_in.sums) {
        hipLaunchKernelGGL(rotary_reduce_kernel, dim3((unsigned)((2 * a_in.D + 15) / 16)), dim3(256), 0, stream, a_in, (int)groups);
        e = hipGetLastError();
    }
    return e;
}

hipError_t prepare_rotary_kernels() {
    hipFuncAttributes f;
    return hipFuncGetAttributes(&f, reinterpret_cast<const void*>(rotary_reduce_kernel));        // loads the code object
}

}  // namespace rtl
