// Rows grouped by expert: which tile of which expert a workgroup owns, found on the device from the experts' offsets.
#pragma once
#include "gemm_tile.h"

namespace rtl {
namespace {

// Rows [begin, end) of expert e. Offsets are read as they come: cut to [0, T], and an end before its begin is an expert without rows, so that
// no offsets lead outside of the tensors.
struct RowRange {
    int begin, end;
};
__device__ __forceinline__ RowRange expert_rows(const int* offsets, int e, int T) {
    const int b = min(max(offsets[e], 0), T), n = min(max(offsets[e + 1], 0), T);
    return RowRange{b, max(b, n)};
}

// Over the lanes of a wave, in lane moves (a few cycles each; shuffles through LDS took 1.5 us of a workgroup's start): inclusive sums, and the
// smallest number, which lands in lane 63.
template <class F>
__device__ __forceinline__ int over_lanes(int v, int none, F f) {
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x111, 0xF, 0xF, false));       // from 1, 2, 4, 8 lanes below, inside 16
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x112, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x114, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x118, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x142, 0xA, 0xF, false));       // the 16 before, then the 32
    v = f(v, __builtin_amdgcn_update_dpp(none, v, 0x143, 0xC, 0xF, false));
    return v;
}
__device__ __forceinline__ int lane_scan(int n) {
    return over_lanes(n, 0, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int lane_min(int n) {
    return __builtin_amdgcn_readlane(over_lanes(n, 0x7FFFFFFF, [](int a, int b) { return min(a, b); }), 63);
}

struct GroupTile {
    int expert, begin, rows, tile;       // tile: index in the walk of the expert's own grid of tiles
};

// The tile of this workgroup: experts in order, ceil(rows / bm) * tiles_n tiles each, the list dealt to the XCDs in contiguous shares. False for a
// workgroup without one: the grid is an upper bound, since the host does not know the offsets. Every wave finds it for itself, 64 experts
// at a time, one to a lane. (Counts are cut to the grid's size, which is under kMaxGroupGrid = 2^24, so that no offsets overflow the sums.)
__device__ __forceinline__ bool group_tile(const int* offsets, int E, int T, int bm, int tiles_n, GroupTile& out) {
    const int lane = threadIdx.x & 63, grid = (int)gridDim.x;
    auto lane_rows = [&](int e0) {
        RowRange r{0, 0};
        if (e0 + lane < E) r = expert_rows(offsets, e0 + lane, T);
        return r;
    };
    auto count = [&](const RowRange& r) { return (int)min((int64_t)((r.end - r.begin + bm - 1) / bm) * tiles_n, (int64_t)grid); };
    RowRange r = lane_rows(0);
    int n = count(r), upto = lane_scan(n), total = min(__builtin_amdgcn_readlane(upto, 63), grid);
    for (int e0 = 64; e0 < E; e0 += 64) total = min(total + __builtin_amdgcn_readlane(lane_scan(count(lane_rows(e0))), 63), grid);
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8;
    const int t = xcd_share_start(total, xcd) + local;
    if (t >= xcd_share_start(total, xcd + 1)) return false;
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        if (e0 > 0) {
            r = lane_rows(e0);
            n = count(r);
            upto = lane_scan(n);
        }
        const uint64_t hit = __ballot(before + upto > t);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            out.expert = e0 + l;
            out.begin = __builtin_amdgcn_readlane(r.begin, l);
            out.rows = __builtin_amdgcn_readlane(r.end, l) - out.begin;
            out.tile = t - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Two tile heights in one launch, for experts of many rows: 256 rows for as many panels as suit, 128 for the rest of the rows. An expert's last rows are
// seldom a full panel, and uniform tiles leave the last round mostly empty (8192 rows over eight experts: 37 panels, with 2048 columns 296 tiles of
// 256 x 256, 1.16 rounds that cost 2). (192 rows as a third height end launches sooner by this count and not by the clock: the matrix instructions run at the power
// limit, and lower tiles take more energy per product. Sustained, on inputs that change: [8192, 4096, 2048] over uneven experts 163 us without, 177 with, medians of three runs.)
struct MixedTile {
    bool tall;
    int expert, begin, rows, panels, tile;       // begin, rows: the expert's rows that are cut into `panels` of this height
};
constexpr int kUnits = 256;              // compute units
// us of a tile of 256 columns with every unit at work: 8 and this for each stage of 128 bytes of the contraction. Measured, 8 and 32 (4-bit) or 64 stages:
// 128 rows bf16 14.7 / 62, 4-bit 16.4 / 33.9, input gradient 14.7 / 57; 256 rows 21.8 / 106, 23.1 / 60, 22.4 / 105.
constexpr float kTileFixed = 8.0f, kTile128 = 0.78f, kTile256 = 1.5f;

// Time of `tall` tiles and then `half` tiles on the chip, in those of a tall tile (c: time of a half tile in those), each tile to the unit that frees
// first: after the whole rounds of tall tiles x units work at one more, the others at half tiles, whose k-th ends at k c there and at 1 + k c on the x.
__device__ __forceinline__ float mixed_time(int tall, int half, float c) {
    const int x = tall % kUnits, rest = kUnits - x;
    const float least = max(((float)half * c + (float)x) / kUnits, x ? 1.0f : 0.0f);
    auto held = [&](float t) { return rest * (int)(t / c + 0.01f) + x * (int)(max(t - 1.0f, 0.0f) / c + 0.01f); };
    float best = 1e9f;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const float a = max((ceilf(least / c - 0.01f) + k) * c, least), b = 1.0f + (ceilf(max(least - 1.0f, 0.0f) / c - 0.01f) + k) * c;
        if (held(a) >= half) best = min(best, a);
        if (x && held(b) >= half) best = min(best, b);
    }
    return (float)(tall / kUnits) + best;
}

__device__ __forceinline__ int half_panels(int rows) { return (rows + 127) / 128; }

struct MixedPlan {
    int p, tall, half;                   // tall panels, tall tiles, half tiles
};
__device__ __forceinline__ MixedPlan plan_mixed(const int* offsets, int E, int T, int tiles_n, int stages) {
    const int lane = threadIdx.x & 63, most = T / 128 + min(E, T);                   // no offsets that ascend make more panels
    int full = 0, rest = 0;
    auto add = [&](int& sum, int n) { sum = min(sum + __builtin_amdgcn_readlane(lane_scan(n), 63), most); };
    for (int e0 = 0; e0 < E; e0 += 64) {
        int n = 0;
        if (e0 + lane < E) {
            const RowRange r = expert_rows(offsets, e0 + lane, T);
            n = r.end - r.begin;
        }
        add(full, n / 256);
        add(rest, half_panels(n % 256));
    }
    // how many panels are tall: each lane prices one number, all full panels or fewer, in steps of 16 tiles or more
    const int mine = max(full - lane * max(1, 16 / tiles_n), 0), left = (full - mine) * 2 + rest;
    const float cost128 = kTileFixed + kTile128 * stages, cost256 = kTileFixed + kTile256 * stages;
    const float us = mixed_time(mine * tiles_n, left * tiles_n, cost128 / cost256) * cost256;
    const int pick = lane_min((int)min(us * 16.0f, 3e7f) << 6 | lane) & 63;          // (the lowest lane among equals)
    const int p = __builtin_amdgcn_readlane(mine, pick);
    return MixedPlan{p, p * tiles_n, ((full - p) * 2 + rest) * tiles_n};
}

// Number t of the tall (body) or of the half tiles: the tall panels go to the first experts.
__device__ __forceinline__ bool find_mixed(const int* offsets, int E, int T, int tiles_n, const MixedPlan& plan, bool body, int t, MixedTile& out) {
    const int lane = threadIdx.x & 63, panel = t / tiles_n;
    int before = 0, full_before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        RowRange r{0, 0};
        if (e0 + lane < E) r = expert_rows(offsets, e0 + lane, T);
        const int n = r.end - r.begin, f = n / 256, f_upto = lane_scan(f), taken = min(max(plan.p - (full_before + f_upto - f), 0), f);
        const int count = body ? taken : half_panels(n - taken * 256), upto = lane_scan(count);
        const uint64_t hit = __ballot(before + upto > panel);
        if (hit) {
            const int l = __builtin_ctzll(hit), cut = __builtin_amdgcn_readlane(taken, l) * 256;
            const int begin = __builtin_amdgcn_readlane(r.begin, l), end = __builtin_amdgcn_readlane(r.end, l);
            out.tall = body;
            out.expert = e0 + l;
            out.begin = body ? begin : begin + cut;
            out.rows = body ? cut : end - begin - cut;
            out.panels = __builtin_amdgcn_readlane(count, l);
            out.tile = t - (before + __builtin_amdgcn_readlane(upto, l) - out.panels) * tiles_n;
            return true;
        }
        before = min(before + __builtin_amdgcn_readlane(upto, 63), 1 << 28);
        full_before = min(full_before + __builtin_amdgcn_readlane(f_upto, 63), 1 << 28);
    }
    return false;
}

// All tiles of the launch on kUnits workgroups: an XCD's share of the list (tall tiles first) is dealt to its workgroups to and fro, so that who got a
// late, small tile gets an early one next. (Left to the hardware a tile waits for a unit of the shader engine that is next in turn, whatever
// units are free elsewhere: input gradient of 248 tall tiles and 16 half ones, 64 stages, 151 -> 126 us; forward of 496 and 32, 32 stages, 137 -> 128.) `work` is called with each tile of this workgroup.
template <class Work>
__device__ __forceinline__ void mixed_tiles(const int* offsets, int E, int T, int tiles_n, int stages, Work work) {
    const MixedPlan plan = plan_mixed(offsets, E, T, tiles_n, stages);
    constexpr int kPer = kUnits / 8;
    const int xcd = (int)blockIdx.x % 8, l = (int)blockIdx.x / 8;
    const int nb = plan.tall, all = plan.tall + plan.half, nb0 = xcd_share_start(nb, xcd), nb_x = nb / 8 + (xcd < nb % 8);
    const int first = xcd_share_start(all, xcd), n = all / 8 + (xcd < all % 8);
    for (int k = 0; k * kPer < n; ++k) {
        const int local = k * kPer + (k % 2 ? kPer - 1 - l : l);
        if (local >= n) continue;
        MixedTile t;
        if (!find_mixed(offsets, E, T, tiles_n, plan, local < nb_x, local < nb_x ? nb0 + local : first - nb0 + (local - nb_x), t)) return;
        if (k > 0) __syncthreads();                      // the last tile's rows have left LDS
        work(t);
    }
}

}  // namespace
}  // namespace rtl
