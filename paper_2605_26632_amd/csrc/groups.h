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
    auto scan = [&](int n) {             // inclusive
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int up = __shfl_up(n, d);
            if (lane >= d) n += up;
        }
        return n;
    };
    RowRange r = lane_rows(0);
    int n = count(r), upto = scan(n), total = min(__builtin_amdgcn_readlane(upto, 63), grid);
    for (int e0 = 64; e0 < E; e0 += 64) total = min(total + __builtin_amdgcn_readlane(scan(count(lane_rows(e0))), 63), grid);
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8;
    const int t = xcd_share_start(total, xcd) + local;
    if (t >= xcd_share_start(total, xcd + 1)) return false;
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        if (e0 > 0) {
            r = lane_rows(e0);
            n = count(r);
            upto = scan(n);
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

// Two tile heights in one launch, for experts of many rows: as many 256-row panels as fill whole rounds of the chip, the rest of the rows in 128-row
// ones. An expert's last rows are seldom a full panel, and uniform tiles leave the last round mostly empty (8192 rows over eight experts: 37 panels, with
// 2048 columns 296 tiles, 1.16 rounds that cost 2).
struct MixedTile {
    bool tall;                           // 256 rows, else 128
    int expert, begin, rows, panels, tile;       // begin, rows: the expert's rows that are cut into `panels` of this height
};
constexpr int kUnits = 256;              // compute units
constexpr float kHalfCost = 0.6f;        // time of a 128 x 256 tile in those of a 256 x 256 one

// Time of `tall` tiles and then `half` tiles on the chip, in those of a tall tile, each tile to the unit that frees first: after the whole rounds
// of tall tiles x units work at one more, the others at half tiles, whose k-th ends at k c there and at 1 + k c on the x.
__device__ __forceinline__ float mixed_time(int tall, int half) {
    constexpr float c = kHalfCost;
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

__device__ __forceinline__ bool group_tile_mixed(const int* offsets, int E, int T, int tiles_n, MixedTile& out) {
    const int lane = threadIdx.x & 63, grid = (int)gridDim.x, most = grid / tiles_n;
    auto lane_rows = [&](int e0) {
        RowRange r{0, 0};
        if (e0 + lane < E) r = expert_rows(offsets, e0 + lane, T);
        return r;
    };
    auto scan = [&](int n) {             // inclusive
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int up = __shfl_up(n, d);
            if (lane >= d) n += up;
        }
        return n;
    };
    // panels of all experts: full ones, and 128-row ones of what is left of each (sums cut to the grid's size: see group_tile)
    RowRange r = lane_rows(0);
    int full = 0, rest = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const RowRange x = e0 ? lane_rows(e0) : r;
        const int n = x.end - x.begin;
        full = min(full + __builtin_amdgcn_readlane(scan(n / 256), 63), most);
        rest = min(rest + __builtin_amdgcn_readlane(scan((n % 256 + 127) / 128), 63), most);
    }
    // how many full panels are tall ones: each lane prices one number, the fewest halves among equals
    const int mine = max(full - lane, 0);
    float best = mixed_time(mine * tiles_n, (2 * (full - mine) + rest) * tiles_n);
    int p = mine;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        const float t = __shfl_xor(best, d);
        const int q = __shfl_xor(p, d);
        if (t < best - 1e-4f || (t < best + 1e-4f && q > p)) {
            best = t;
            p = q;
        }
    }
    p = __builtin_amdgcn_readfirstlane(p);
    const int nb = p * tiles_n, nt = (2 * (full - p) + rest) * tiles_n;
    const int xcd = (int)blockIdx.x % 8, local = (int)blockIdx.x / 8, nb_x = nb / 8 + (xcd < nb % 8);
    if (local >= xcd_share_start(nb + nt, xcd + 1) - xcd_share_start(nb + nt, xcd)) return false;
    out.tall = local < nb_x;
    const int t = out.tall ? xcd_share_start(nb, xcd) + local : xcd_share_start(nb + nt, xcd) - xcd_share_start(nb, xcd) + (local - nb_x);
    const int panel = t / tiles_n;
    int before = 0, full_before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        if (e0) r = lane_rows(e0);
        const int n = r.end - r.begin, f = n / 256, f_upto = scan(f);
        const int taken = min(max(p - (full_before + f_upto - f), 0), f);         // tall panels of the lane's expert
        const int count = out.tall ? taken : 2 * (f - taken) + (n % 256 + 127) / 128, upto = scan(count);
        const uint64_t hit = __ballot(before + upto > panel);
        if (hit) {
            const int l = __builtin_ctzll(hit), cut = __builtin_amdgcn_readlane(taken, l) * 256;
            const int begin = __builtin_amdgcn_readlane(r.begin, l), end = __builtin_amdgcn_readlane(r.end, l);
            out.expert = e0 + l;
            out.begin = out.tall ? begin : begin + cut;
            out.rows = out.tall ? cut : end - begin - cut;
            out.panels = __builtin_amdgcn_readlane(count, l);
            out.tile = t - (before + __builtin_amdgcn_readlane(upto, l) - out.panels) * tiles_n;
            return true;
        }
        before = min(before + __builtin_amdgcn_readlane(upto, 63), 1 << 28);
        full_before = min(full_before + __builtin_amdgcn_readlane(f_upto, 63), 1 << 28);
    }
    return false;
}

}  // namespace
}  // namespace rtl
