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

}  // namespace
}  // namespace rtl
