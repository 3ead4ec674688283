// The norms of a transformer block with its gate, residual and modulation in one pass over the rows, and their gradients.
//
//   forward   x' = alpha x + gate_s (w_post norm(y)),  h = w_pre norm(x') (1 + scale_s) + shift_s             for the rows of sequence s
//   backward  dn = dh w_pre (1 + scale_s), dt = dx' + J dn with J the norm's: layer r (dn - mean dn - n mean(dn n)), rms without mean dn;
//             dx = alpha dt, dy = J (w_post gate_s dt) over norm(y);
//             dgate_s = sum dt w_post norm(y), dscale_s = sum dh w_pre n, dshift_s = sum dh over the rows of s; the weights' sums go over all of them
//
// Bound by memory: forward reads x, y and writes x', h, backward reads dx', dh, x', y and writes dx, dy, each once; a row's values stay in the
// registers of its team (a wave or a workgroup) from the load to the last store, so that the statistics are taken in two steps, mean first,
// without reading anything again. Everything between the loads and the one rounding at each store is fp32.
#include <type_traits>
#include "rtl_internal.h"

namespace rtl {
namespace {

// A row's team is a wave or a workgroup; workgroups of 256 threads, or of the team's where that is more.
constexpr int team_threads(int waves) { return waves > 4 ? waves * 64 : 256; }

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void unpack8(const uint4 v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(w[e] << 16);
        f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const f32x2 v = {f[2 * e], f[2 * e + 1]};
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));       // RNE
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&f)[8]) { unpack8(*reinterpret_cast<const uint4*>(p), f); }
template <bool F32>
__device__ __forceinline__ void load8_as(const void* p, int64_t at, float (&f)[8]) {
    if constexpr (F32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        const float4 u = q[0], v = q[1];
        f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
    } else {
        load8(static_cast<const uint16_t*>(p) + at, f);
    }
}
template <bool F32>
__device__ __forceinline__ void store8_as(void* p, int64_t at, const float (&f)[8]) {
    if constexpr (F32) {
        float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
        q[0] = make_float4(f[0], f[1], f[2], f[3]);
        q[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = pack8(f);
    }
}

// Sum over the lanes of a wave, in all of them.
__device__ __forceinline__ float wave_sum(float v) {
    auto step = [](float x, auto ctrl, auto rows) {
        return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
    };
    using std::integral_constant;
    using all = integral_constant<int, 0xF>;
    v = step(v, integral_constant<int, 0x111>{}, all{});                          // from 1, 2, 4, 8 lanes below, inside 16
    v = step(v, integral_constant<int, 0x112>{}, all{});
    v = step(v, integral_constant<int, 0x114>{}, all{});
    v = step(v, integral_constant<int, 0x118>{}, all{});
    v = step(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});   // the 16 before, then the 32
    v = step(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// Sums of two values over a team of WAVES waves, in a fixed order. `slot` (team of several waves): LDS of 2 x 2 WAVES floats, used by turns, so that
// one barrier a sum is enough: a wave that writes a half again has passed the barrier behind which everybody has read it.
template <int WAVES>
struct TeamSum {
    float* slot;
    int turn = 0;
    __device__ __forceinline__ void operator()(float& a, float& b) {
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (WAVES > 1) {
            const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            float* s = slot + turn * 2 * WAVES;
            if (lane == 0) {
                s[2 * wave] = a;
                s[2 * wave + 1] = b;
            }
            __syncthreads();
            a = s[0];
            b = s[1];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                a += s[2 * w];
                b += s[2 * w + 1];
            }
            turn ^= 1;
        }
    }
};

// Sequence of a row: how many of the ends offsets[1 .. S] lie at or before it, 64 of them looked at in each step of a search that divides by 64; -1 for a
// row of no sequence. Any offsets lead to a sequence in [0, S) or to none.
__device__ __forceinline__ int sequence_of(const int* offsets, int S, int row) {
    if (!offsets) return 0;
    const int lane = threadIdx.x & 63;
    int step = 1, count = 0;
    while ((int64_t)step * 64 < S) step *= 64;
    for (;; step /= 64) {
        const int64_t at = count + (int64_t)(lane + 1) * step;
        const int end = at <= S ? offsets[at] : 0x7FFFFFFF;
        count += __builtin_popcountll(__ballot(end <= row)) * step;
        if (step == 1 || count >= S) break;
    }
    return count < S && offsets[0] <= row ? count : -1;
}

struct Stats {
    float mean, scale;
};

// Statistics of two rows at once (either may be without a norm). v: NCH chunks of eight of the lane, zeros behind the end of the row.
template <int WAVES, int NCH>
__device__ __forceinline__ void row_stats(const float (&u)[NCH][8], int kind_u, Stats& su, const float (&v)[NCH][8], int kind_v, Stats& sv, int team_lane, int D,
                                          float eps, TeamSum<WAVES>& sum) {
    su = sv = Stats{0.f, 1.f};
    const float inv = 1.0f / (float)D;
    if (kind_u == RTL_NORM_LAYER || kind_v == RTL_NORM_LAYER) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a += u[c][e];
                b += v[c][e];
            }
        sum(a, b);
        if (kind_u == RTL_NORM_LAYER) su.mean = a * inv;
        if (kind_v == RTL_NORM_LAYER) sv.mean = b * inv;
    }
    if (kind_u != RTL_NORM_NONE || kind_v != RTL_NORM_NONE) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
            if ((c * WAVES * 64 + team_lane) * 8 < D) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = u[c][e] - su.mean, q = v[c][e] - sv.mean;
                    a += p * p;
                    b += q * q;
                }
            }
        sum(a, b);
        if (kind_u != RTL_NORM_NONE) su.scale = 1.0f / sqrtf(a * inv + eps);
        if (kind_v != RTL_NORM_NONE) sv.scale = 1.0f / sqrtf(b * inv + eps);
    }
}

template <int WAVES, int NCH, bool F32>
__global__ __launch_bounds__(team_threads(WAVES)) void norm_kernel(const NormArgs a) {
    __shared__ float slots[4 * WAVES];
    constexpr int TEAM = WAVES * 64, TEAMS = team_threads(WAVES) / TEAM;
    const int tl = threadIdx.x % TEAM;
    const int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM;
    if (row >= a.T) return;
    const int D = (int)a.D;
    const int s = __builtin_amdgcn_readfirstlane(sequence_of(a.offsets, (int)a.S, (int)row));
    float x[NCH][8];
    if (s < 0) {
        if (!a.clear) return;
        const float zero[8] = {};
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * TEAM + tl) * 8;
            if (col < D) {
                if (a.x_out) store8_as<F32>(a.x_out, row * a.ldxo + col, zero);
                if (a.h) store8_as<false>(a.h, row * a.ldh + col, zero);
            }
        }
        return;
    }
    TeamSum<WAVES> sum{slots};
    float y[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * TEAM + tl) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = y[c][e] = 0.f;
        if (col < D) {
            load8_as<F32>(a.x, row * a.ldx + col, x[c]);
            if (a.y) load8(a.y + row * a.ldy + col, y[c]);
        }
    }
    Stats sy, sx;
    row_stats<WAVES, NCH>(y, a.y ? a.post : RTL_NORM_NONE, sy, y, RTL_NORM_NONE, sx, tl, D, a.eps, sum);
    {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * TEAM + tl) * 8;
            if (col < D) {
                float w[8], g[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = g[e] = 1.0f;
                if (a.w_post) load8(a.w_post + col, w);
                if (a.gate) load8(a.gate + s * a.ld_gate + col, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c][e] = a.alpha * x[c][e] + g[e] * (w[e] * ((y[c][e] - sy.mean) * sy.scale));
                if (a.x_out) store8_as<F32>(a.x_out, row * a.ldxo + col, x[c]);
            }
        }
    }
    if (!a.h) return;
    row_stats<WAVES, NCH>(x, a.pre, sx, x, RTL_NORM_NONE, sy, tl, D, a.eps, sum);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int col = (c * TEAM + tl) * 8;
        if (col < D) {
            float w[8], g[8], b[8], h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = 1.0f;
                g[e] = b[e] = 0.f;
            }
            if (a.w_pre) load8(a.w_pre + col, w);
            if (a.scale) load8(a.scale + s * a.ld_mod + col, g);
            if (a.shift) load8(a.shift + s * a.ld_mod + col, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = w[e] * ((x[c][e] - sx.mean) * sx.scale) * (1.0f + g[e]) + b[e];
            store8_as<false>(a.h, row * a.ldh + col, h);
        }
    }
}

// A team takes `rows` neighbouring rows and keeps the columns' sums of the sequence it is in; where the sequence changes, and behind the last row, they go to
// the workspace. Team b and sequence s have slot b + s: over a team's rows and from team to team one of the two grows and neither falls, so no two
// share a slot. Sums of a slot: [dt norm(y) | dh n | dh], D floats each.
template <int WAVES, int NCH, bool F32>
__global__ __launch_bounds__(team_threads(WAVES)) void norm_backward_kernel(const NormGradArgs a) {
    __shared__ float slots[4 * WAVES];
    constexpr int TEAM = WAVES * 64, TEAMS = team_threads(WAVES) / TEAM;
    const int tl = threadIdx.x % TEAM;
    const int64_t team = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM, first = team * a.rows;
    if (first >= a.T) return;
    const int64_t end = min(first + a.rows, a.T);
    const int D = (int)a.D;
    const float inv = 1.0f / (float)D;
    TeamSum<WAVES> sum{slots};
    float of_gate[NCH][8], of_scale[NCH][8], of_shift[NCH][8];
    int now = -1;
    auto leave = [&]() {
        if (now < 0 || !a.sums) return;
        float* to = a.sums + (team + now) * 3 * a.D;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * TEAM + tl) * 8;
            if (col < D) {
                store8_as<true>(to, col, of_gate[c]);
                store8_as<true>(to, a.D + col, of_scale[c]);
                store8_as<true>(to, 2 * a.D + col, of_shift[c]);
            }
        }
    };
    for (int64_t row = first; row < end; ++row) {
        const int s = __builtin_amdgcn_readfirstlane(sequence_of(a.offsets, (int)a.S, (int)row));
        if (s < 0) {
            if (a.clear) {
                const float zero[8] = {};
#pragma unroll
                for (int c = 0; c < NCH; ++c) {
                    const int col = (c * TEAM + tl) * 8;
                    if (col < D) {
                        if (a.dx) store8_as<F32>(a.dx, row * a.lddx + col, zero);
                        if (a.dy) store8_as<false>(a.dy, row * a.lddy + col, zero);
                    }
                }
            }
            continue;
        }
        if (s != now) {
            leave();
            now = s;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) of_gate[c][e] = of_scale[c][e] = of_shift[c][e] = 0.f;
        }
        float x[NCH][8], y[NCH][8], dh[NCH][8], dt[NCH][8];
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * TEAM + tl) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] = y[c][e] = dh[c][e] = dt[c][e] = 0.f;
            if (col < D) {
                if (a.dh) {
                    load8_as<F32>(a.x, row * a.ldx + col, x[c]);
                    load8(a.dh + row * a.lddh + col, dh[c]);
                }
                if (a.y) load8(a.y + row * a.ldy + col, y[c]);
                if (a.dx_out) load8_as<F32>(a.dx_out, row * a.lddxo + col, dt[c]);
            }
        }
        Stats sx, sy;
        row_stats<WAVES, NCH>(x, a.dh ? a.pre : RTL_NORM_NONE, sx, y, a.y ? a.post : RTL_NORM_NONE, sy, tl, D, a.eps, sum);
        // n in x's place, norm(y) in y's; the columns' sums of dh; then dn in dh's place
        float m = 0.f, mn = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * TEAM + tl) * 8;
            if (col < D) {
                float w[8], g[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = 1.0f;
                    g[e] = 0.f;
                }
                if (a.w_pre) load8(a.w_pre + col, w);
                if (a.scale) load8(a.scale + s * a.ld_mod + col, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[c][e] = (x[c][e] - sx.mean) * sx.scale;
                    y[c][e] = (y[c][e] - sy.mean) * sy.scale;
                    of_scale[c][e] += dh[c][e] * x[c][e];
                    of_shift[c][e] += dh[c][e];
                    dh[c][e] *= w[e] * (1.0f + g[e]);
                    m += dh[c][e];
                    mn += dh[c][e] * x[c][e];
                }
            }
        }
        if (a.dh && a.pre != RTL_NORM_NONE) {
            sum(m, mn);
            m = a.pre == RTL_NORM_LAYER ? m * inv : 0.f;
            mn *= inv;
        } else {
            m = mn = 0.f;
        }
        float p = 0.f, pn = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int col = (c * TEAM + tl) * 8;
            if (col < D) {
                float w[8], g[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = g[e] = 1.0f;
                if (a.w_post) load8(a.w_post + col, w);
                if (a.gate) load8(a.gate + s * a.ld_gate + col, g);
                float dx[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dt[c][e] += sx.scale * (dh[c][e] - m - x[c][e] * mn);
                    dx[e] = a.alpha * dt[c][e];
                    of_gate[c][e] += dt[c][e] * y[c][e];
                    dt[c][e] *= g[e] * w[e];
                    p += dt[c][e];
                    pn += dt[c][e] * y[c][e];
                }
                if (a.dx) store8_as<F32>(a.dx, row * a.lddx + col, dx);
            }
        }
        if (!a.y) continue;
        if (a.post != RTL_NORM_NONE) {
            sum(p, pn);
            p = a.post == RTL_NORM_LAYER ? p * inv : 0.f;
            pn *= inv;
        } else {
            p = pn = 0.f;
        }
        if (a.dy) {
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                const int col = (c * TEAM + tl) * 8;
                if (col < D) {
                    float dy[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) dy[e] = sy.scale * (dt[c][e] - p - y[c][e] * pn);
                    store8_as<false>(a.dy, row * a.lddy + col, dy);
                }
            }
        }
    }
    leave();
}

// Adds the slots of a sequence up in the order of its rows: 64 columns to a workgroup, the slots dealt to its four waves in turn and the four sums added in
// order. What the weights' gradients need of it goes to a.totals ([S][2][D]).
__global__ __launch_bounds__(256) void norm_reduce_kernel(const NormGradArgs a) {
    __shared__ float part[3][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane, s = blockIdx.y;
    int64_t b0 = 0, b1 = -1;
    const int64_t begin = a.offsets ? min(max((int64_t)a.offsets[s], (int64_t)0), a.T) : 0;
    const int64_t end = a.offsets ? min(max((int64_t)a.offsets[s + 1], (int64_t)0), a.T) : a.T;
    if (begin < end) {
        b0 = begin / a.rows;
        b1 = (end - 1) / a.rows;
    }
    float v[3] = {};
    if (col < a.D)
        for (int64_t b = b0 + wave; b <= b1; b += 4) {
            const float* p = a.sums + (b + s) * 3 * a.D + col;
#pragma unroll
            for (int k = 0; k < 3; ++k) v[k] += p[k * a.D];
        }
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][wave][lane] = v[k];
    __syncthreads();
    if (wave != 0 || col >= a.D) return;
#pragma unroll
    for (int k = 0; k < 3; ++k)
        for (int w = 1; w < 4; ++w) v[k] += part[k][w][lane];
    auto one = [](const uint16_t* p, int64_t at) { return p ? __uint_as_float((uint32_t)p[at] << 16) : 1.0f; };
    if (a.dgate) a.dgate[s * a.D + col] = v[0] * one(a.w_post, col);
    if (a.dscale) a.dscale[s * a.D + col] = v[1] * one(a.w_pre, col);
    if (a.dshift) a.dshift[s * a.D + col] = v[2];
    if (a.dw_post) a.totals[s * 2 * a.D + col] = v[0];
    if (a.dw_pre) a.totals[(s * 2 + 1) * a.D + col] = v[1];
}

// dw_post = sum_s gate_s totals_s, dw_pre = sum_s (1 + scale_s) totals_s, the sequences dealt to four waves as the slots above.
__global__ __launch_bounds__(256) void norm_weights_kernel(const NormGradArgs a) {
    __shared__ float part[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float v[2] = {};
    if (col < a.D)
        for (int64_t s = wave; s < a.S; s += 4) {
            if (a.dw_post) v[0] += a.totals[s * 2 * a.D + col] * (a.gate ? __uint_as_float((uint32_t)a.gate[s * a.ld_gate + col] << 16) : 1.0f);
            if (a.dw_pre) v[1] += a.totals[(s * 2 + 1) * a.D + col] * (1.0f + (a.scale ? __uint_as_float((uint32_t)a.scale[s * a.ld_mod + col] << 16) : 0.0f));
        }
    part[0][wave][lane] = v[0];
    part[1][wave][lane] = v[1];
    __syncthreads();
    if (wave != 0 || col >= a.D) return;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        for (int w = 1; w < 4; ++w) v[k] += part[k][w][lane];
    if (a.dw_post) a.dw_post[col] = v[0];
    if (a.dw_pre) a.dw_pre[col] = v[1];
}

// f(waves of a team, chunks of a lane) for rows of D values.
template <class F>
hipError_t with_team(int64_t D, F f) {
    using std::integral_constant;
    if (D <= 512) return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    if (D <= 1024) return f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    if (D <= 2048) return f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (D <= 4096) return f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    return f(integral_constant<int, 8>{}, integral_constant<int, 2>{});
}

constexpr int kBackwardRows = 16;            // rows of a team in the backward pass

}  // namespace

hipError_t launch_residual_norm(const NormArgs& a, hipStream_t stream) {
    return with_team(a.D, [&](auto waves, auto chunks) {
        constexpr int W = decltype(waves)::value, C = decltype(chunks)::value;
        const int64_t teams = team_threads(W) / (W * 64);
        const dim3 grid((unsigned)((a.T + teams - 1) / teams));
        if (a.x_f32) hipLaunchKernelGGL((norm_kernel<W, C, true>), grid, dim3(team_threads(W)), 0, stream, a);
        else hipLaunchKernelGGL((norm_kernel<W, C, false>), grid, dim3(team_threads(W)), 0, stream, a);
        return hipGetLastError();
    });
}

// [slots | totals], the slots' rows three times D floats
size_t residual_norm_backward_slots(int64_t T, int64_t S) { return (size_t)((T + kBackwardRows - 1) / kBackwardRows + S); }

hipError_t launch_residual_norm_backward(const NormGradArgs& a_in, hipStream_t stream) {
    NormGradArgs a = a_in;
    a.rows = kBackwardRows;
    hipError_t e = hipSuccess;
    if (a.T > 0)
        e = with_team(a.D, [&](auto waves, auto chunks) {
            constexpr int W = decltype(waves)::value, C = decltype(chunks)::value;
            const int64_t rows = team_threads(W) / (W * 64) * a.rows;
            const dim3 grid((unsigned)((a.T + rows - 1) / rows));
            if (a.x_f32) hipLaunchKernelGGL((norm_backward_kernel<W, C, true>), grid, dim3(team_threads(W)), 0, stream, a);
            else hipLaunchKernelGGL((norm_backward_kernel<W, C, false>), grid, dim3(team_threads(W)), 0, stream, a);
            return hipGetLastError();
        });
    const unsigned cols = (unsigned)((a.D + 63) / 64);
    const bool weights = a.dw_post || a.dw_pre;
    if (e == hipSuccess && a.S > 0 && (weights || a.dgate || a.dscale || a.dshift)) {
        hipLaunchKernelGGL(norm_reduce_kernel, dim3(cols, (unsigned)a.S), dim3(256), 0, stream, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && weights) {
        hipLaunchKernelGGL(norm_weights_kernel, dim3(cols), dim3(256), 0, stream, a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t prepare_norm_kernels() {
    hipFuncAttributes f;
    hipError_t e = hipFuncGetAttributes(&f, reinterpret_cast<const void*>(norm_reduce_kernel));        // loads the code object
    return e;
}

}  // namespace rtl
