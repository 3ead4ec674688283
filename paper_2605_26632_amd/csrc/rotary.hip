// Norm and rotary positions of the heads of q and k, in one pass over both, and their gradients.
//
//   forward   n = w q / sqrt(mean q^2 + eps) (or q itself); with the angle pos[t, axis[j]] freq[j] pair j of n is turned by it, (a, b) -> (a cos - b sin,
//             a sin + b cos); pairs are (2 j, 2 j + 1) or (j, j + pairs), what lies behind the pairs passes
//   backward  the gradient is turned back by the angle; dw += d q r, and through the norm: dq = r (w d - q r mean(w d q r)), r = 1 / sqrt(mean q^2 + eps)
//
// Bound by memory (each head read once and written once). An angle belongs to a token: a wave takes heads of one token and has its lanes take the sines of
// a pair each, which they share in LDS. The product of position and frequency is exact in 64 bits and cut to a quarter turn there, since in 32 a far
// position's angle would be off by 2^-24 of itself; the rest is fp32. q and k are dealt to workgroups of their own, so that weights and strides are
// the same throughout a wave.
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

// What a lane does in every head: its two chunks of eight values (first value, or -1 for none) and its eight pairs. HALVES: element e of the first chunk and
// of the second are pair e; else a chunk holds four pairs, of which the lane has the two chunks' eight.
// Chunks that only pass are left alone: turned by zero, a value that is not finite would reach the other of its pair.
constexpr int kMostPairs = 256 + 8;
struct LanePlan {
    int at[2], pair0;
    bool turned[2];          // of each chunk (HALVES: of both)
};
template <bool HALVES>
__device__ __forceinline__ LanePlan lane_plan(int c, int D, int pairs) {
    const int chunks = D / 8, none = (pairs + 7) / 8 * 8;
    if constexpr (HALVES) {
        const int half = pairs / 8, rest = 2 * half + 2 * (c - half);
        if (c < half) return LanePlan{{c * 8, (c + half) * 8}, c * 8, {true, true}};
        return LanePlan{{rest < chunks ? rest * 8 : -1, rest + 1 < chunks ? (rest + 1) * 8 : -1}, none, {false, false}};
    } else {
        const int i = 2 * c;
        return LanePlan{{i < chunks ? i * 8 : -1, i + 1 < chunks ? (i + 1) * 8 : -1}, min(c * 8, none), {i * 4 < pairs, i * 4 + 4 < pairs}};
    }
}

// The token's sines, a pair to a lane, through the wave's own part of LDS (whose operations stay in order): those of the lane's pairs come back.
struct Turns {
    float sn[8], cs[8];
};
__device__ __forceinline__ Turns token_turns(const RotaryArgs& a, const LanePlan& p, int64_t token, float (*lds)[kMostPairs]) {
    const int fill = (a.pairs + 7) / 8 * 8 + 8;
    for (int j = threadIdx.x & 63; j < fill; j += 64) {
        float s = 0.f, c = 1.f;
        if (j < a.pairs) {
            const int ax = min(max(a.axis[j], 0), a.axes - 1);
            turn(a.pos[token * a.axes + ax], a.freq[j], s, c);
        }
        lds[0][j] = s;
        lds[1][j] = c;
    }
    __builtin_amdgcn_wave_barrier();
    Turns t;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        t.sn[e] = lds[0][p.pair0 + e];
        t.cs[e] = lds[1][p.pair0 + e];
    }
    __builtin_amdgcn_wave_barrier();
    return t;
}

// Both chunks turned; BACK: by the negative angle. PART: there are values behind the pairs. (Selections in place of the template took heads that are turned
// whole 1 % longer, [16896, 30 + 30, 128] 102 -> 103 us, branches 2 to 5 %.)
template <bool HALVES, bool BACK, bool PART>
__device__ __forceinline__ void apply_turns(float (&v)[2][8], const Turns& t, const LanePlan& plan) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float& x = HALVES ? v[0][e] : v[e / 4][2 * (e % 4)];
        float& y = HALVES ? v[1][e] : v[e / 4][2 * (e % 4) + 1];
        const float s = BACK ? -t.sn[e] : t.sn[e], p = x * t.cs[e] - y * s, q = x * s + y * t.cs[e];
        const bool turned = !PART || plan.turned[HALVES ? 0 : e / 4];
        x = turned ? p : x;
        y = turned ? q : y;
    }
}

__device__ __forceinline__ void load_chunks(const uint16_t* p, const LanePlan& plan, float (&v)[2][8]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (plan.at[c] >= 0) raw = *reinterpret_cast<const uint4*>(p + plan.at[c]);
        unpack(raw, v[c]);
    }
}
__device__ __forceinline__ void store_chunks(uint16_t* p, const LanePlan& plan, const float (&v)[2][8]) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (plan.at[c] >= 0) *reinterpret_cast<uint4*>(p + plan.at[c]) = pack(v[c]);
}
__device__ __forceinline__ void load_weights(const uint16_t* p, const LanePlan& plan, float (&w)[2][8]) {
    if (p) {
        load_chunks(p, plan, w);
    } else {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) w[c][e] = 1.0f;
    }
}
__device__ __forceinline__ float square_sum(const float (&v)[2][8]) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[c][e] * v[c][e];
    return s;
}

// A wave takes one token and side.per heads of it, 64 / L at a time: one time only, unless the launch would be too large. Then the four waves of a workgroup work on
// neighbouring heads, and memory gives more than to waves that go through a token each, though every wave takes the token's sines anew (us, a token to a wave |
// one time): [16896, 30 + 30, 128] 105 | 96, [16896, 40 + 40, 128] 139 | 123, [5000, 64 + 8, 128] 32.8 | 29.0, [1, 30 + 30, 128] 4.3 | 3.2;
// [4096, 24 + 24, 128] 17.7 | 18.1, [16896, 12 + 12, 256] 82.7 | 84.3. The first side[0].groups workgroups have the heads of q, the others those of k.
template <int L, bool HALVES, bool PART>
__global__ __launch_bounds__(kHeadWaves * 64) void rotary_kernel(const RotaryArgs a) {
    __shared__ float lds[kHeadWaves][2][kMostPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_k = blockIdx.x >= a.side[0].groups;
    const HeadSide& side = a.side[is_k];
    const uint32_t task = (blockIdx.x - (is_k ? a.side[0].groups : 0)) * kHeadWaves + wave, token = task / side.splits;
    if (token >= a.T) return;
    const int h0 = (int)(task % side.splits) * side.per, h1 = min(h0 + side.per, side.H);
    const LanePlan plan = lane_plan<HALVES>(lane % L, a.D, a.pairs);
    const Turns turns = token_turns(a, plan, token, lds[wave]);
    float w[2][8];
    load_weights(side.w, plan, w);
    const uint16_t* const in = side.in + token * side.ld;
    uint16_t* const out = side.out + token * side.ldo;
    for (int h = h0 + lane / L; h < h1; h += 64 / L) {
        float v[2][8];
        load_chunks(in + h * side.s, plan, v);
        if (a.norm) {
            const float r = 1.0f / sqrtf(head_sum<L>(square_sum(v)) * (1.0f / (float)a.D) + a.eps);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[c][e] *= r * w[c][e];
        }
        apply_turns<HALVES, false, PART>(v, turns, plan);
        store_chunks(out + h * side.so, plan, v);
    }
}

// The same walk for the gradients; a wave goes on to further tokens, and what it has of the weight's gradient goes to the workspace at the end, a
// workgroup's four waves and a wave's 64 / L heads added up in order. [4433, 30 + 30, 128] 34.5 us at the least, 204 MB (some of them in the cache behind
// L2), and 4 for the reduction.
template <int L, bool HALVES, bool PART>
__global__ __launch_bounds__(kHeadWaves * 64, 4) void rotary_backward_kernel(const RotaryArgs a) {
    __shared__ float lds[kHeadWaves][2][kMostPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_k = blockIdx.x >= a.side[0].groups;
    const HeadSide& side = a.side[is_k];
    const uint32_t tasks = (uint32_t)a.T * side.splits;
    const LanePlan plan = lane_plan<HALVES>(lane % L, a.D, a.pairs);
    const float inv = 1.0f / (float)a.D;
    float w[2][8], dw[2][8];
    load_weights(side.w, plan, w);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = 0.f;
    for (uint32_t task = (blockIdx.x - (is_k ? a.side[0].groups : 0)) * kHeadWaves + wave; task < tasks; task += side.groups * kHeadWaves) {
        const uint32_t token = task / side.splits;
        const int h0 = (int)(task % side.splits) * side.per, h1 = min(h0 + side.per, side.H);
        const Turns turns = token_turns(a, plan, token, lds[wave]);
        const uint16_t* const in = a.norm ? side.in + token * side.ld : nullptr;
        const uint16_t* const grad = side.grad + token * side.ldg;
        uint16_t* const out = side.out + token * side.ldo;
        for (int h = h0 + lane / L; h < h1; h += 64 / L) {
            float d[2][8];
            load_chunks(grad + h * side.sg, plan, d);
            if (a.norm) {
                float v[2][8];
                load_chunks(in + h * side.s, plan, v);
                apply_turns<HALVES, true, PART>(d, turns, plan);
                const float r = 1.0f / sqrtf(head_sum<L>(square_sum(v)) * inv + a.eps);
                float m = 0.f;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[c][e] *= r;
                        dw[c][e] += d[c][e] * v[c][e];
                        d[c][e] *= w[c][e];
                        m += d[c][e] * v[c][e];
                    }
                m = head_sum<L>(m) * inv;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[c][e] = r * (d[c][e] - v[c][e] * m);
            } else {
                apply_turns<HALVES, true, PART>(d, turns, plan);
            }
            store_chunks(out + h * side.so, plan, d);
        }
    }
    if (!side.sums) return;
    __syncthreads();
    float (*const part)[L * 16] = reinterpret_cast<float (*)[L * 16]>(&lds[0][0][0]);
    static_assert(kHeadWaves * L * 16 <= kHeadWaves * 2 * kMostPairs, "the waves' sums fit");
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float s = dw[c][e];
#pragma unroll
            for (int step = L; step < 64; step *= 2) s += __shfl_xor(s, step);
            if (lane < L && plan.at[c] >= 0) part[wave][plan.at[c] + e] = s;
        }
    __syncthreads();
    float* const to = side.sums + (int64_t)(blockIdx.x - (is_k ? a.side[0].groups : 0)) * a.D;
    for (int i = threadIdx.x; i < a.D; i += kHeadWaves * 64) {
        float s = part[0][i];
#pragma unroll
        for (int v = 1; v < kHeadWaves; ++v) s += part[v][i];
        to[i] = s;
    }
}

// The workgroups' sums of a side (blockIdx.y), 16 columns to a workgroup, dealt to its 64 groups of 16 lanes in turn and those added in order. Eight loads of a lane
// are under way at a time: one after the other they were most of the launch ([4433, 30 + 30, 128], both kernels, 40.5 -> 38.8 us).
constexpr int kAtOnce = 8;
__global__ __launch_bounds__(1024) void rotary_reduce_kernel(const RotaryArgs a) {
    __shared__ float part[64][16];
    const HeadSide& side = a.side[blockIdx.y];
    const int i = blockIdx.x * 16 + (threadIdx.x & 15), g = threadIdx.x >> 4;
    float s = 0.f;
    if (i < a.D && side.dw)
        for (uint32_t b = g; b < side.groups; b += 64 * kAtOnce) {
            float v[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) v[u] = side.sums[(int64_t)min(b + 64 * u, side.groups - 1) * a.D + i];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) s += b + 64 * u < side.groups ? v[u] : 0.f;
        }
    part[g][threadIdx.x & 15] = s;
    __syncthreads();
    if (g != 0 || i >= a.D || !side.dw) return;
    for (int v = 1; v < 64; ++v) s += part[v][threadIdx.x & 15];
    side.dw[i] = s;
}

// f(lanes of a head, pairs in halves, values behind the pairs)
template <class F>
hipError_t with_form(const RotaryArgs& a, F f) {
    using std::integral_constant;
    auto go = [&](auto lanes) {
        using T = std::true_type;
        using N = std::false_type;
        const bool part = 2 * a.pairs < a.D;
        if (a.interleaved) return part ? f(lanes, N{}, T{}) : f(lanes, N{}, N{});
        return part ? f(lanes, T{}, T{}) : f(lanes, T{}, N{});
    };
    if (a.D <= 64) return go(integral_constant<int, 4>{});
    if (a.D <= 128) return go(integral_constant<int, 8>{});
    if (a.D <= 256) return go(integral_constant<int, 16>{});
    return go(integral_constant<int, 32>{});
}

constexpr int64_t kMostTasks = (int64_t)1 << 23;         // of a side, where a task can be more than an iteration (a launch takes fewer than 2^32 threads)

// Deals the heads of a side to the waves of the backward pass: a task is a token and `per` of its heads. `waves` run at a time; a task costs about .7 of an
// iteration over 64 / L heads besides its iterations, and the last round of tasks counts in full. us, tokens as tasks | so | an iteration to a task:
// [1, 30 + 30, 128] 9.6 | 7.6 | 7.6, [5000, 64 + 8, 128] 62.7 | 56.1 | 59.6, [4096, 30 + 30, 128] 37.3 | 37.5 | 38.6, [16896, 12 + 12, 256] 129 | 129 | 141,
// [16896, 40 + 40, 128] 206 | 206 | 203.
void deal(HeadSide& side, int64_t T, int step, int64_t waves) {
    const int most = (side.H + step - 1) / step;
    double best = 0;
    for (int splits = 1; splits <= most; splits += 1 + splits / 16) {
        const int per = (most + splits - 1) / splits;
        const int64_t n = (most + per - 1) / per, rounds = (T * n + waves - 1) / waves;
        if (splits > 1 && T * n > kMostTasks) break;
        const double time = (double)rounds * (per + 0.7);
        if (splits == 1 || time < best) {
            best = time;
            side.per = per * step;
            side.splits = (int)n;
        }
    }
}

constexpr int64_t kGroups = 1024;            // workgroups of the backward pass, as many as the chip holds at a time

// One side's share of them, by the iterations that its tasks of whole tokens take. (Halves: [1024, 24 + 8] alike, [300, 48 + 2, 64] 9.4 -> 9.6.)
int64_t share(const RotaryArgs& a, int i, int step) {
    auto work = [&](int k) { return a.side[k].H > 0 ? (double)((a.side[k].H + step - 1) / step) + 0.7 : 0.0; };
    const int64_t n = (int64_t)((double)kGroups * work(i) / (work(0) + work(1)));
    return n > 0 ? n : 1;
}

}  // namespace

size_t rotary_backward_scratch(int64_t D) { return (size_t)(kGroups + 2) * (size_t)D * sizeof(float); }

hipError_t launch_rotary(const RotaryArgs& a_in, hipStream_t stream) {
    return with_form(a_in, [&](auto lanes, auto halves, auto part) {
        constexpr int L = decltype(lanes)::value;
        constexpr bool HALVES = decltype(halves)::value, PART = decltype(part)::value;
        RotaryArgs a = a_in;
        for (int i = 0; i < 2; ++i) {
            HeadSide& side = a.side[i];
            side.splits = 1;
            if (side.H > 0) {
                const int64_t most = (side.H + 64 / L - 1) / (64 / L), times = (a.T * most + kMostTasks - 1) / kMostTasks;
                side.per = (int)(times > 1 ? times : 1) * (64 / L);
                side.splits = (side.H + side.per - 1) / side.per;
            }
            side.groups = side.H > 0 ? (unsigned)((a.T * side.splits + kHeadWaves - 1) / kHeadWaves) : 0;
        }
        const dim3 grid(a.side[0].groups + a.side[1].groups), block(kHeadWaves * 64);
        hipLaunchKernelGGL((rotary_kernel<L, HALVES, PART>), grid, block, 0, stream, a);
        return hipGetLastError();
    });
}

hipError_t launch_rotary_backward(const RotaryArgs& a_in, float* sums, hipStream_t stream) {
    return with_form(a_in, [&](auto lanes, auto halves, auto part) {
        constexpr int L = decltype(lanes)::value;
        constexpr bool HALVES = decltype(halves)::value, PART = decltype(part)::value;
        RotaryArgs a = a_in;
        for (int i = 0; i < 2; ++i) {
            HeadSide& side = a.side[i];
            side.groups = 0;
            side.splits = 1;
            if (side.H > 0 && a.T > 0) {
                const int64_t most = share(a, i, 64 / L);
                deal(side, a.T, 64 / L, most * kHeadWaves);
                const int64_t groups = (a.T * side.splits + kHeadWaves - 1) / kHeadWaves;
                side.groups = (unsigned)(groups < most ? groups : most);
            }
            if (side.dw) side.sums = sums + (i ? (int64_t)a.side[0].groups * a.D : 0);
        }
        const unsigned groups = a.side[0].groups + a.side[1].groups;
        if (groups > 0) {
            hipLaunchKernelGGL((rotary_backward_kernel<L, HALVES, PART>), dim3(groups), dim3(kHeadWaves * 64), 0, stream, a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (a.side[0].dw || a.side[1].dw) hipLaunchKernelGGL(rotary_reduce_kernel, dim3((unsigned)((a.D + 15) / 16), 2), dim3(1024), 0, stream, a);
        return hipGetLastError();
    });
}

hipError_t prepare_rotary_kernels() {
    hipFuncAttributes f;
    return hipFuncGetAttributes(&f, reinterpret_cast<const void*>(rotary_reduce_kernel));        // loads the code object
}

}  // namespace rtl
