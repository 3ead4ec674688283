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

// A row's team is a wave, four of which make a workgroup, or a workgroup.
constexpr int team_threads(int waves) { return waves > 1 ? waves * 64 : 256; }

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

// Sum over a team of WAVES waves, in a fixed order. `slot` (team of several waves): LDS of 2 x WAVES floats, used by turns, so that one barrier a sum is
// enough: a wave that writes a half again has passed the barrier behind which everybody has read it.
template <int WAVES>
struct TeamSum {
    float* slot;
    int turn = 0;
    __device__ __forceinline__ float operator()(float a) {
        a = wave_sum(a);
        if constexpr (WAVES > 1) {
            float* s = slot + turn * WAVES;
            if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
            __syncthreads();
            a = s[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) a += s[w];
            turn ^= 1;
        }
        return a;
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

// Statistics of a row. v: NCH chunks of eight of the lane, zeros behind the end of the row.
template <int WAVES, int NCH>
__device__ __forceinline__ Stats row_stats(const float (&v)[NCH][8], int kind, int team_lane, int D, float eps, TeamSum<WAVES>& sum) {
    Stats s{0.f, 1.f};
    const float inv = 1.0f / (float)D;
    if (kind == RTL_NORM_LAYER) {
        float a = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) a += v[c][e];
        s.mean = sum(a) * inv;
    }
    if (kind != RTL_NORM_NONE) {
        float a = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
            if ((c * WAVES * 64 + team_lane) * 8 < D) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = v[c][e] - s.mean;
                    a += p * p;
                }
            }
        s.scale = 1.0f / sqrtf(sum(a) * inv + eps);
    }
    return s;
}

// A lane has NCH chunks of eight columns. [16896, 3840] with everything 101 us, 5.1 TB/s, what a copy reaches.
template <int WAVES, int NCH, bool F32>
__global__ __launch_bounds__(team_threads(WAVES)) void norm_kernel(const NormArgs a) {
    __shared__ float slots[2 * WAVES];
    constexpr int TEAM = WAVES * 64, TEAMS = team_threads(WAVES) / TEAM;
    const int tl = threadIdx.x % TEAM;
    const int64_t row = a.first + (int64_t)blockIdx.x * TEAMS + __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM);
    if (row >= a.T) return;
    const int D = (int)a.D;
    auto column = [&](int c) { return (uint32_t)((c * TEAM + tl) * 8); };
    const int s = __builtin_amdgcn_readfirstlane(sequence_of(a.offsets, (int)a.S, (int)row));
    if (s < 0) {
        if (!a.clear) return;
        const float zero[8] = {};
#pragma unroll
        for (int c = 0; c < NCH; ++c)
            if (column(c) < (uint32_t)D) {
                if (a.x_out) store8_as<F32>(a.x_out, row * a.ldxo, column(c), zero);
                if (a.h) store8_as<false>(a.h, row * a.ldh, column(c), zero);
            }
        return;
    }
    TeamSum<WAVES> sum{slots};
    // a chunk of a vector, `none` where there is no vector
    constexpr uint32_t kOnes = 0x3F803F80u;
    auto vector = [&](const uint16_t* p, int64_t at, int c, uint32_t none, float (&f)[8]) {
        uint4 v = make_uint4(none, none, none, none);
        if (p && column(c) < (uint32_t)D) v = *reinterpret_cast<const uint4*>(p + at + column(c));
        unpack8(v, f);
    };
    // Without y its vectors count as ones, whatever they hold, and its values as -0: alpha x plus that is alpha x, the sign of a zero too.
    // (Branches around the vectors took 3 to 4 % longer, [16896, 3840] 102 -> 105 us.)
    const float none = a.y ? 0.f : -0.f;
    float x[NCH][8], y[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[c][e] = 0.f;
            y[c][e] = none;
        }
        if (column(c) < (uint32_t)D) {
            load8_as<F32>(a.x, row * a.ldx, column(c), x[c]);
            if (a.y) load8(a.y + row * a.ldy, column(c), y[c]);
        }
    }
    const Stats sy = row_stats<WAVES, NCH>(y, a.y ? a.post : RTL_NORM_NONE, tl, D, a.eps, sum);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        float w[8], g[8];
        vector(a.y ? a.w_post : nullptr, 0, c, kOnes, w);
        vector(a.y ? a.gate : nullptr, s * a.ld_gate, c, kOnes, g);
        if (column(c) < (uint32_t)D) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[c][e] = a.alpha * x[c][e] + g[e] * (w[e] * ((y[c][e] - sy.mean) * sy.scale));
            if (a.x_out) store8_as<F32>(a.x_out, row * a.ldxo, column(c), x[c]);
        }
    }
    if (!a.h) return;
    const Stats sx = row_stats<WAVES, NCH>(x, a.pre, tl, D, a.eps, sum);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        float w[8], g[8], b[8], h[8];
        vector(a.w_pre, 0, c, kOnes, w);
        vector(a.scale, s * a.ld_mod, c, 0, g);
        vector(a.shift, s * a.ld_mod, c, 0, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = w[e] * ((x[c][e] - sx.mean) * sx.scale) * (1.0f + g[e]) + b[e];
        if (column(c) < (uint32_t)D) store8_as<false>(a.h, row * a.ldh, column(c), h);
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
// [8192, 3840], one of the norms, 74 to 78 us, 386 MB at 5.0 TB/s, and 4.5 for the reduction; fp32 [2111, 2048] with both norms and five sequences 19 to 20, 4.5 to 5 and 3.5.
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
        if (a.w_pre && a.dh) load8(a.w_pre, col, f_pre);          // (without dh neither is looked at: zeros times them need not be zeros)
        if (a.w_post) load8(a.w_post, col, f_post);
        if (a.scale && a.dh) {
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

// Adds the slots of a sequence up (blockIdx.y): kReduceCols columns to a workgroup, the slots dealt to its kReduceSlices rows of threads in turn, their sums
// added in order. What the weights' gradients need of it goes to a.totals ([S][2][D]); those of a single sequence are made here. (A workgroup that takes all
// the sequences one after the other, which spares norm_weights_kernel, took 7 us longer with five.)
constexpr int kReduceCols = 32, kReduceSlices = 32;
__device__ __forceinline__ float bf16_or(const uint16_t* p, int64_t at, float none) { return p ? __uint_as_float((uint32_t)p[at] << 16) : none; }
__global__ __launch_bounds__(kReduceCols * kReduceSlices) void norm_reduce_kernel(const NormGradArgs a) {
    __shared__ float part[3][kReduceSlices][kReduceCols];
    const int lane = threadIdx.x % kReduceCols, slice = threadIdx.x / kReduceCols, D = (int)a.D, T = (int)a.T, s = blockIdx.y;
    const int col0 = blockIdx.x * kReduceCols, col = min(col0 + lane, D - 1);
    const int begin = a.offsets ? min(max(a.offsets[s], 0), T) : 0, end = a.offsets ? min(max(a.offsets[s + 1], 0), T) : T;
    const int b0 = (int)((uint32_t)begin / (uint32_t)a.rows), b1 = begin < end ? (int)((uint32_t)(end - 1) / (uint32_t)a.rows) : b0 - 1;
    float v[3] = {};
    const float* p = a.sums + (int64_t)(b0 + slice + s) * 3 * D + col;
#pragma unroll 4
    for (int b = b0 + slice; b <= b1; b += kReduceSlices, p += (int64_t)kReduceSlices * 3 * D)
#pragma unroll
        for (int k = 0; k < 3; ++k) v[k] += p[k * D];
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][slice][lane] = v[k];
    __syncthreads();
    if (slice >= 3 || col0 + lane >= D) return;                  // the first three rows of threads finish one sum each
    float sum = part[slice][0][lane];
    for (int w = 1; w < kReduceSlices; ++w) sum += part[slice][w][lane];
    const int64_t at = (int64_t)s * D + col;
    // Zero where there is nothing to sum up, whatever the vectors of a sequence without rows, or of a gradient that is not there, hold.
    const bool any = begin < end, any_h = any && a.dh;
    if (slice == 0) {
        if (a.dgate) a.dgate[at] = any ? sum * bf16_or(a.w_post, col, 1.0f) : 0.f;
        if (a.dw_post && a.S == 1) a.dw_post[col] = any ? sum * bf16_or(a.gate, col, 1.0f) : 0.f;
        else if (a.dw_post) a.totals[(int64_t)s * 2 * D + col] = sum;
    } else if (slice == 1) {
        if (a.dscale) a.dscale[at] = any_h ? sum * bf16_or(a.w_pre, col, 1.0f) : 0.f;
        if (a.dw_pre && a.S == 1) a.dw_pre[col] = any_h ? sum * (1.0f + bf16_or(a.scale, col, 0.0f)) : 0.f;
        else if (a.dw_pre) a.totals[((int64_t)s * 2 + 1) * D + col] = sum;
    } else if (a.dshift) {
        a.dshift[at] = sum;
    }
}

// dw_post = sum_s gate_s totals_s, dw_pre = sum_s (1 + scale_s) totals_s over the sequences that have rows, dealt as the slots above.
__global__ __launch_bounds__(kReduceCols * kReduceSlices) void norm_weights_kernel(const NormGradArgs a) {
    __shared__ float part[2][kReduceSlices][kReduceCols];
    const int lane = threadIdx.x % kReduceCols, slice = threadIdx.x / kReduceCols, D = (int)a.D;
    const int col0 = blockIdx.x * kReduceCols, col = min(col0 + lane, D - 1);
    float v[2] = {};
    for (int64_t s = slice; s < a.S; s += kReduceSlices) {
        const bool any = min(max(a.offsets[s], 0), (int)a.T) < min(max(a.offsets[s + 1], 0), (int)a.T);       // (several sequences or none: there are offsets)
        if (a.dw_post) {
            const float total = a.totals[s * 2 * D + col], factor = bf16_or(a.gate, s * a.ld_gate + col, 1.0f);
            v[0] = any ? v[0] + total * factor : v[0];
        }
        if (a.dw_pre && a.dh) {
            const float total = a.totals[(s * 2 + 1) * D + col], factor = 1.0f + bf16_or(a.scale, s * a.ld_mod + col, 0.0f);
            v[1] = any ? v[1] + total * factor : v[1];
        }
    }
    part[0][slice][lane] = v[0];
    part[1][slice][lane] = v[1];
    __syncthreads();
    if (slice >= 2 || col0 + lane >= D) return;
    float sum = part[slice][0][lane];
    for (int w = 1; w < kReduceSlices; ++w) sum += part[slice][w][lane];
    float* const to = slice ? a.dw_pre : a.dw_post;
    if (to) to[col] = sum;
}

// f(waves of a team, chunks of a lane) for T rows of D values. With few rows a launch is as long as a row, and one chunk to a lane is soonest through it; with
// many, half the waves at two chunks spare barriers and workgroups. us, one | two chunks: [4, 1024] 3.3 | 4.4, [4, 3840] 3.6 | 4.8, [512, 3840] 5.5 | 6.0,
// [4, 8192] 4.1 | 4.9, [2048, 1024] 5.5 | 5.9, [2048, 3840] 14.2 | 14.4; [33792, 1024] 51.9 | 51.0, [16896, 3840] 106.3 | 105.3, [4096, 8192] 45.0 | 44.1.
// (One wave: [33792, 512] 24.7, two of one row 30.3. Four of one chunk: [16896, 2048] 51.9, two of two 51.6, one of four 53.8.)
constexpr int64_t kFewNormRows = 2048;
template <class F>
hipError_t with_team(int64_t T, int64_t D, F f) {
    using std::integral_constant;
    const bool few = T <= kFewNormRows;
    if (D <= 512) return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    if (D <= 1024) return few ? f(integral_constant<int, 2>{}, integral_constant<int, 1>{}) : f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    if (D <= 2048) return f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (D <= 4096) return few ? f(integral_constant<int, 8>{}, integral_constant<int, 1>{}) : f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    return few ? f(integral_constant<int, 16>{}, integral_constant<int, 1>{}) : f(integral_constant<int, 8>{}, integral_constant<int, 2>{});
}

// Backward pass: waves of a team, and rows of one: the rows dealt once over teams of eight waves to a compute unit. Sixteen read at the same rate and leave
// twice the sums: [16896, 3840] 175 -> 167 us, [16896, 2048] 104 -> 97, [8192, 3840] 90 -> 85, [16896, 512] 40 -> 34, fp32 [2111, 2048] 28.7 -> 27.4.
int team_waves(int64_t D) { return (int)((D + 511) / 512); }
int64_t team_rows(int64_t T, int64_t D) {
    const int waves = team_waves(D);
    const int64_t teams = 256 * (waves < 8 ? 8 / waves : 1);
    return T > teams ? (T + teams - 1) / teams : 1;
}

}  // namespace

// Workgroups of one launch, which takes fewer than 2^32 threads: 2^23 rows of more than 4096 columns, 512 threads each, would have as many.
constexpr int64_t kMostNormGroups = (int64_t)1 << 22;

hipError_t launch_residual_norm(const NormArgs& a_in, hipStream_t stream) {
    NormArgs a = a_in;
    return with_team(a.T, a.D, [&](auto waves, auto chunks) {
        constexpr int W = decltype(waves)::value, C = decltype(chunks)::value;
        constexpr int64_t teams = team_threads(W) / (W * 64), most = kMostNormGroups * teams;
        hipError_t e = hipSuccess;
        for (a.first = 0; a.first < a.T && e == hipSuccess; a.first += most) {
            const int64_t rows = a.T - a.first < most ? a.T - a.first : most;
            const dim3 grid((unsigned)((rows + teams - 1) / teams)), block(team_threads(W));
            if (a.x_f32) hipLaunchKernelGGL((norm_kernel<W, C, true>), grid, block, 0, stream, a);
            else hipLaunchKernelGGL((norm_kernel<W, C, false>), grid, block, 0, stream, a);
            e = hipGetLastError();
        }
        return e;
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
    const unsigned cols = (unsigned)((a.D + kReduceCols - 1) / kReduceCols), threads = kReduceCols * kReduceSlices;
    const bool weights = a.dw_post || a.dw_pre;
    if (e != hipSuccess || !(weights || a.dgate || a.dscale || a.dshift)) return e;
    if (a.S > 0) {
        hipLaunchKernelGGL(norm_reduce_kernel, dim3(cols, (unsigned)a.S), dim3(threads), 0, stream, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && weights && a.S != 1) {
        hipLaunchKernelGGL(norm_weights_kernel, dim3(cols), dim3(threads), 0, stream, a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t prepare_norm_kernels() {
    hipFuncAttributes f;
    hipError_t e = hipFuncGetAttributes(&f, reinterpret_cast<const void*>(norm_weights_kernel));        // loads the code object
    return e;
}

}  // namespace rtl
