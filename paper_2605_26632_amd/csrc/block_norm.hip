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
// A row's address is the same in all lanes of a team (scalar registers), the column a 32-bit offset from it.
template <bool F32>
__device__ __forceinline__ const void* row_at(const void* p, int64_t at) { return static_cast<const uint8_t*>(p) + at * (F32 ? 4 : 2); }
__device__ __forceinline__ void load8(const uint16_t* row, uint32_t col, float (&f)[8]) { unpack8(*reinterpret_cast<const uint4*>(row + col), f); }
template <bool F32>
__device__ __forceinline__ void load8_as(const void* p, int64_t at, uint32_t col, float (&f)[8]) {
    const void* row = row_at<F32>(p, at);
    if constexpr (F32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(row) + col);
        const float4 u = q[0], v = q[1];
        f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
    } else {
        load8(static_cast<const uint16_t*>(row), col, f);
    }
}
template <bool F32>
__device__ __forceinline__ void store8_as(void* p, int64_t at, uint32_t col, const float (&f)[8]) {
    void* row = const_cast<void*>(row_at<F32>(p, at));
    if constexpr (F32) {
        float4* q = reinterpret_cast<float4*>(static_cast<float*>(row) + col);
        q[0] = make_float4(f[0], f[1], f[2], f[3]);
        q[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(row) + col) = pack8(f);
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
    const int64_t row = (int64_t)blockIdx.x * TEAMS + __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM);
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
                if (a.x_out) store8_as<F32>(a.x_out, row * a.ldxo, col, zero);
                if (a.h) store8_as<false>(a.h, row * a.ldh, col, zero);
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
            load8_as<F32>(a.x, row * a.ldx, col, x[c]);
            if (a.y) load8(a.y + row * a.ldy, col, y[c]);
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
                if (a.w_post) load8(a.w_post, col, w);
                if (a.gate) load8(a.gate + s * a.ld_gate, col, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c][e] = a.alpha * x[c][e] + g[e] * (w[e] * ((y[c][e] - sy.mean) * sy.scale));
                if (a.x_out) store8_as<F32>(a.x_out, row * a.ldxo, col, x[c]);
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
            if (a.w_pre) load8(a.w_pre, col, w);
            if (a.scale) load8(a.scale + s * a.ld_mod, col, g);
            if (a.shift) load8(a.shift + s * a.ld_mod, col, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = w[e] * ((x[c][e] - sx.mean) * sx.scale) * (1.0f + g[e]) + b[e];
            store8_as<false>(a.h, row * a.ldh, col, h);
        }
    }
}

// Sums of two values over the workgroup's waves (any number up to 16), in a fixed order: the waves' sums meet in LDS, and the lanes of each row of sixteen add
// all of them up. `slot`: 2 x 32 floats, used by turns as in TeamSum.
__device__ __forceinline__ void group_sum(float& a, float& b, float* slot, int& turn, int waves) {
    a = wave_sum(a);
    b = wave_sum(b);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float* s = slot + turn * 32;
    turn ^= 1;
    if (lane == 0) {
        s[wave] = a;
        s[16 + wave] = b;
    }
    __syncthreads();
    const int at = lane & 15;
    a = at < waves ? s[at] : 0.f;
    b = at < waves ? s[16 + at] : 0.f;
    auto step = [](float& x, auto ctrl) { x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    auto both = [&](auto ctrl) {
        step(a, ctrl);
        step(b, ctrl);
    };
    both(std::integral_constant<int, 0xB1>{});           // the neighbour, the other pair, the other four, the other eight
    both(std::integral_constant<int, 0x4E>{});
    both(std::integral_constant<int, 0x141>{});
    both(std::integral_constant<int, 0x140>{});
}

// Eight values as they lie in memory.
template <bool F32>
struct Raw8 {
    uint4 v[F32 ? 2 : 1];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (uint4& q : v) q = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void load(const void* p, int64_t at, uint32_t col) {
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(row_at<F32>(p, at)) + col * (F32 ? 4 : 2));
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) v[i] = q[i];
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f[4 * i] = __uint_as_float(v[i].x);
                f[4 * i + 1] = __uint_as_float(v[i].y);
                f[4 * i + 2] = __uint_as_float(v[i].z);
                f[4 * i + 3] = __uint_as_float(v[i].w);
            }
        } else {
            unpack8(v[0], f);
        }
    }
};

// A team of a.waves waves, a chunk of eight columns to a lane, takes a.rows neighbouring rows and keeps the columns' sums of the sequence it is in; where the
// sequence changes, and behind the last row, they go to the workspace. Team b and sequence s have slot b + s: over a team's rows and from team to team one of
// the two grows and neither falls, so no two share a slot. Sums of a slot: [dt norm(y) | dh n | dh], D floats each.
// The next row is under way while a row is worked on, and the factors of a sequence stay in registers as products: a row takes three or four sums over the
// team one after the other, and the few teams that a compute unit holds would not hide the loads behind them.
// Lanes behind the end of the row work on the row's first columns and are left out of the sums and stores only: branches around the arithmetic made the
// compiler keep two copies of what lives across them, and spill.
// SOLO: a wave to a team, four teams to a workgroup. POST: norm(y) is not y.
template <bool F32, bool SOLO, bool POST>
__global__ __launch_bounds__(SOLO ? 256 : 1024, 4) void norm_backward_kernel(const NormGradArgs a) {
    __shared__ float slots[64];
    const int tl = SOLO ? threadIdx.x & 63 : threadIdx.x, D = (int)a.D;
    const int team = SOLO ? (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : (int)blockIdx.x;
    const int first = team * a.rows;
    if (first >= a.T) return;
    const int end = (int)min((int64_t)first + a.rows, a.T);
    const bool mine = tl * 8 < D;
    const uint32_t own = mine ? tl * 8 : 0;
    // (formed anew where it is used: kept across the loops, the sums of the arrays' addresses and the column took 26 registers)
    auto column = [&]() {
        uint32_t c = own;
        asm volatile("" : "+v"(c));
        return c;
    };
    const float inv = 1.0f / (float)D;
    int turn = 0;
    auto sum = [&](float& u, float& v) {
        u = mine ? u : 0.f;
        v = mine ? v : 0.f;
        if constexpr (SOLO) {
            u = wave_sum(u);
            v = wave_sum(v);
        } else {
            group_sum(u, v, slots, turn, a.waves);
        }
    };
    const bool layer_pre = a.pre == RTL_NORM_LAYER, norm_pre = a.dh && a.pre != RTL_NORM_NONE, layer_post = POST && a.post == RTL_NORM_LAYER;

    for (int row = first; row < end;) {
        // a run of rows of one sequence
        const int s = __builtin_amdgcn_readfirstlane(sequence_of(a.offsets, (int)a.S, row));
        if (s < 0) {
            if (a.clear && mine) {
                const uint32_t col = column();
                const float zero[8] = {};
                if (a.dx) store8_as<F32>(a.dx, (int64_t)row * a.lddx, col, zero);
                if (a.dy) store8_as<false>(a.dy, (int64_t)row * a.lddy, col, zero);
            }
            ++row;
            continue;
        }
        const int run_end = a.offsets ? max(min(a.offsets[s + 1], end), row + 1) : end;
        Raw8<F32> rx, rd;
        Raw8<false> ry, rh;
        rx.zero();
        rd.zero();
        ry.zero();
        rh.zero();
        auto fetch = [&](int64_t row) {
            const uint32_t col = column();
            if (a.dh) {
                rx.load(a.x, row * a.ldx, col);
                rh.load(a.dh, row * a.lddh, col);
            }
            if (a.y) ry.load(a.y, row * a.ldy, col);
            if (a.dx_out) rd.load(a.dx_out, row * a.lddxo, col);
        };
        fetch(row);
        float of_gate[8], of_scale[8], of_shift[8], f_pre[8], f_post[8];       // f_pre = w_pre (1 + scale), f_post = gate w_post
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            of_gate[e] = of_scale[e] = of_shift[e] = 0.f;
            f_pre[e] = f_post[e] = 1.0f;
        }
        const uint32_t col = column();
        if (a.w_pre) load8(a.w_pre, col, f_pre);
        if (a.w_post) load8(a.w_post, col, f_post);
        if (a.scale) {
            float v[8];
            load8(a.scale + s * a.ld_mod, col, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) f_pre[e] *= 1.0f + v[e];
        }
        if (a.gate) {
            float v[8];
            load8(a.gate + s * a.ld_gate, col, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) f_post[e] *= v[e];
        }
#pragma unroll 1
      for (; row < run_end; ++row) {
        float x[8], y[8], dh[8], dt[8];
        rx.get(x);
        ry.get(y);
        rh.get(dh);
        rd.get(dt);
        if (row + 1 < run_end) fetch(row + 1);
        float mx = 0.f, rsx = 1.0f, my = 0.f, rsy = 1.0f;
        if (layer_pre || layer_post) {
            float u = 0.f, v = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u += x[e];
                v += y[e];
            }
            sum(u, v);
            if (layer_pre) mx = u * inv;
            if (layer_post) my = v * inv;
        }
        if (norm_pre || POST) {
            float u = 0.f, v = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] -= mx;
                u += x[e] * x[e];
                if constexpr (POST) {
                    y[e] -= my;
                    v += y[e] * y[e];
                }
            }
            sum(u, v);
            if (norm_pre) rsx = 1.0f / sqrtf(u * inv + a.eps);
            if constexpr (POST) rsy = 1.0f / sqrtf(v * inv + a.eps);
        }
        // n in x's place, norm(y) in y's; the columns' sums; dn in dh's place
        float m = 0.f, mn = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] *= rsx;
            if constexpr (POST) y[e] *= rsy;
            of_scale[e] += dh[e] * x[e];
            of_shift[e] += dh[e];
            dh[e] *= f_pre[e];
            m += dh[e];
            mn += dh[e] * x[e];
        }
        if (norm_pre) {
            sum(m, mn);
            m = layer_pre ? m * inv : 0.f;
            mn *= inv;
        } else {
            m = mn = 0.f;
        }
        float p = 0.f, pn = 0.f, out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dt[e] += rsx * (dh[e] - m - x[e] * mn);
            out[e] = a.alpha * dt[e];
            of_gate[e] += dt[e] * y[e];
            dt[e] *= f_post[e];
            if constexpr (POST) {
                p += dt[e];
                pn += dt[e] * y[e];
            }
        }
        if (a.dx && mine) store8_as<F32>(a.dx, (int64_t)row * a.lddx, column(), out);
        if constexpr (POST) {
            sum(p, pn);
            p = layer_post ? p * inv : 0.f;
            pn *= inv;
#pragma unroll
            for (int e = 0; e < 8; ++e) dt[e] = rsy * (dt[e] - p - y[e] * pn);
        }
        if (a.dy && mine) store8_as<false>(a.dy, (int64_t)row * a.lddy, column(), dt);
      }
        if (a.sums && mine) {
            float* to = a.sums + (int64_t)(team + s) * 3 * a.D;
            const uint32_t at = column();
            store8_as<true>(to, 0, at, of_gate);
            store8_as<true>(to, a.D, at, of_scale);
            store8_as<true>(to, 2 * a.D, at, of_shift);
        }
    }
}

// Adds the slots of a sequence up in the order of its rows: 64 columns to a workgroup, the slots dealt to its waves in turn and the waves' sums added in order.
// What the weights' gradients need of it goes to a.totals ([S][2][D]); of a single sequence they are made here.
constexpr int kReduceWaves = 16;
__global__ __launch_bounds__(kReduceWaves * 64) void norm_reduce_kernel(const NormGradArgs a) {
    __shared__ float part[3][kReduceWaves][64];
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
    if (col < a.D) {
        const float* p = a.sums + (b0 + wave + s) * 3 * a.D + col;
#pragma unroll 4
        for (int64_t b = b0 + wave; b <= b1; b += kReduceWaves, p += kReduceWaves * 3 * a.D) {
#pragma unroll
            for (int k = 0; k < 3; ++k) v[k] += p[k * a.D];
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][wave][lane] = v[k];
    __syncthreads();
    if (wave != 0 || col >= a.D) return;
#pragma unroll
    for (int k = 0; k < 3; ++k)
        for (int w = 1; w < kReduceWaves; ++w) v[k] += part[k][w][lane];
    auto one = [](const uint16_t* p, int64_t at) { return p ? __uint_as_float((uint32_t)p[at] << 16) : 1.0f; };
    if (a.dgate) a.dgate[s * a.D + col] = v[0] * one(a.w_post, col);
    if (a.dscale) a.dscale[s * a.D + col] = v[1] * one(a.w_pre, col);
    if (a.dshift) a.dshift[s * a.D + col] = v[2];
    if (a.S == 1) {
        if (a.dw_post) a.dw_post[col] = v[0] * one(a.gate, col);
        if (a.dw_pre) a.dw_pre[col] = v[1] * (a.scale ? 1.0f + one(a.scale, col) : 1.0f);
    } else {
        if (a.dw_post) a.totals[s * 2 * a.D + col] = v[0];
        if (a.dw_pre) a.totals[(s * 2 + 1) * a.D + col] = v[1];
    }
}

// dw_post = sum_s gate_s totals_s, dw_pre = sum_s (1 + scale_s) totals_s, the sequences dealt to the waves as the slots above.
__global__ __launch_bounds__(kReduceWaves * 64) void norm_weights_kernel(const NormGradArgs a) {
    __shared__ float part[2][kReduceWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float v[2] = {};
    if (col < a.D)
        for (int64_t s = wave; s < a.S; s += kReduceWaves) {
            if (a.dw_post) v[0] += a.totals[s * 2 * a.D + col] * (a.gate ? __uint_as_float((uint32_t)a.gate[s * a.ld_gate + col] << 16) : 1.0f);
            if (a.dw_pre) v[1] += a.totals[(s * 2 + 1) * a.D + col] * (1.0f + (a.scale ? __uint_as_float((uint32_t)a.scale[s * a.ld_mod + col] << 16) : 0.0f));
        }
    part[0][wave][lane] = v[0];
    part[1][wave][lane] = v[1];
    __syncthreads();
    if (wave != 0 || col >= a.D) return;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        for (int w = 1; w < kReduceWaves; ++w) v[k] += part[k][w][lane];
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

// Backward pass: waves of a team, and rows of one: the rows dealt once over the teams that the chip holds, 16 waves to a compute unit.
int team_waves(int64_t D) { return (int)((D + 511) / 512); }
int64_t team_rows(int64_t T, int64_t D) {
    const int64_t teams = 256 * (16 / team_waves(D));
    return T > teams ? (T + teams - 1) / teams : 1;
}

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

size_t residual_norm_backward_slots(int64_t T, int64_t S, int64_t D) {
    const int64_t rows = team_rows(T, D);
    return (size_t)((T + rows - 1) / rows + S);
}

hipError_t launch_residual_norm_backward(const NormGradArgs& a_in, hipStream_t stream) {
    NormGradArgs a = a_in;
    a.rows = (int)team_rows(a.T, a.D);
    a.waves = team_waves(a.D);
    hipError_t e = hipSuccess;
    if (a.T > 0) {
        const int64_t teams = (a.T + a.rows - 1) / a.rows;
        auto go = [&](auto f32, auto solo, auto post) {
            constexpr bool F32 = decltype(f32)::value, SOLO = decltype(solo)::value, POST = decltype(post)::value;
            hipLaunchKernelGGL((norm_backward_kernel<F32, SOLO, POST>), dim3((unsigned)(SOLO ? (teams + 3) / 4 : teams)), dim3(SOLO ? 256 : a.waves * 64), 0, stream, a);
        };
        using T = std::true_type;
        using F = std::false_type;
        const bool solo = a.waves == 1, post = a.y && a.post != RTL_NORM_NONE;
        if (a.x_f32) {
            if (solo) post ? go(T{}, T{}, T{}) : go(T{}, T{}, F{});
            else post ? go(T{}, F{}, T{}) : go(T{}, F{}, F{});
        } else {
            if (solo) post ? go(F{}, T{}, T{}) : go(F{}, T{}, F{});
            else post ? go(F{}, F{}, T{}) : go(F{}, F{}, F{});
        }
        e = hipGetLastError();
    }
    const unsigned cols = (unsigned)((a.D + 63) / 64);
    const bool weights = a.dw_post || a.dw_pre;
    if (e == hipSuccess && a.S > 0 && (weights || a.dgate || a.dscale || a.dshift)) {
        hipLaunchKernelGGL(norm_reduce_kernel, dim3(cols, (unsigned)a.S), dim3(kReduceWaves * 64), 0, stream, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && weights && a.S != 1) {
        hipLaunchKernelGGL(norm_weights_kernel, dim3(cols), dim3(kReduceWaves * 64), 0, stream, a);
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
