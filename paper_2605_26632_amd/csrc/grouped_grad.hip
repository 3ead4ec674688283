// Gradients of the linears grouped by expert, bf16 operands, fp32 accumulation (v_mfma_f32_16x16x32_bf16):
//
//   input  : dX[rows of e] = dY[rows of e] W[e]              contraction over N: dY is contiguous along it, W is not
//   weight : dW[e] = dY[rows of e]^T X[rows of e]            contraction over the expert's rows: neither operand is contiguous along it
//   bias   : db[e] = sum of the rows of dY                   beside the weight gradient, by the tiles of its first columns
//
// The matrix instruction wants eight values along the contraction from each lane. An operand that is not contiguous along it is staged as it
// lies in memory (64 rows of the contraction, BM or BN columns) and transposed on the way out of LDS: ds_read_b64_tr_b16 hands lane i of
// 16 lanes the i-th column of the 4 x 16 block that the sixteen addressed (lane l points at row l / 4, columns 4 (l % 4) ..; measured), so two of them
// make a fragment.
// One tile loop for both: a stage is 64 of the contraction, travels to LDS by direct loads through a ring, and is worked off in two
// halves of 32; the fragments of a half are read behind the matrix instructions of the half before it.
// A contraction that is no multiple of 64 takes its last, partial block first: there the places behind its end are filled with zeros instead
// of loaded (on both sides: what lies in memory behind an expert's rows may be NaN), at no cost to the loop.
// 8192 rows, [4096, 2048], eight experts, inputs that change: input gradient 122 us with 1024 rows each, 161 with 484 to 1997 (216 tall and 104 half
// tiles: the units are active 65 % of the launch); weight gradient 141 and 143. Matrix cores busy 42 and 43 % at 2.18 GHz, uneven.
#include "groups.h"

namespace rtl {
namespace {

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
struct GradSmem {
    static constexpr int kA = BM * 128, kB = BN * 128, kStage = kA + kB, kRing = STAGES * kStage;
    static constexpr int kEpiRow = (BN / WAVES_N) * 2 + 16;
    static constexpr int kEpi = WAVES_M * WAVES_N * (BM / WAVES_M) * kEpiRow;
    static constexpr int kTotal = kRing > kEpi ? kRing : kEpi;
    static_assert(kTotal <= 160 * 1024, "LDS budget of a CU");
};

// Tiles of an operand staged as it lies in memory: rows of W columns, in chunks of 32 bytes. A wave's transposing read is served 32 lanes at a
// time, which are eight rows (0 .. 3 and 8 .. 11 of a run of 16, or the same plus 4) of one 32-byte column chunk: the chunk is XORed with a
// number that differs for all eight, so that they meet 64 different banks.
__device__ __forceinline__ int row_key(int row) { return (row & 3) | ((row >> 3) & 1) << 2; }

struct GradArgs {
    const uint16_t* A;       // A_COL: A(c, i) at A[c * lda + i], else at A[i * lda + c]
    const uint16_t* B;       // B(c, j) at B[c * ldb + j]
    void* C;                 // C(i, j) = sum over c of A(c, i) B(c, j), at C[i * ldc + j], bf16 or fp32
    void* row_sums;          // weight gradient, nullable: the sums over c of A(c, i) at [i], the type of C, by the tiles of j = 0
    int64_t lda, ldb, ldc;
    int64_t m, n, depth;     // extents of i, j (both from the tile's own matrix) and c
};

template <bool A_COL, bool F32, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__device__ __forceinline__ void grad_tile(const GradArgs a, const int64_t m0, const int64_t n0, const int part = 0, const int parts = 1) {
    using L = GradSmem<BM, BN, WAVES_M, WAVES_N, STAGES>;
    constexpr int NW = WAVES_M * WAVES_N, WTM = BM / WAVES_M, WTN = BN / WAVES_N, TM = WTM / 16, TN = WTN / 16;
    static_assert(!A_COL || BM % 128 == 0, "eight 32-byte chunks to a row");
    static_assert(BN % 128 == 0, "eight 32-byte chunks to a row");
    static_assert((!A_COL || BM == 128 || NW == 8) && (BN == 128 || NW == 8) && NW % 4 == 0, "order of a wave's requests (col_unit)");
    constexpr int A_PER_W = L::kA / 1024 / NW, B_PER_W = L::kB / 1024 / NW, LOADS = A_PER_W + B_PER_W;
    static_assert(L::kA % (1024 * NW) == 0 && L::kB % (1024 * NW) == 0, "tile loads must divide over the waves");

    extern __shared__ __align__(1024) uint8_t smem[];
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                                // (in a loop over tiles: formed anew for each, not kept across it)
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)smem;
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;
    const int64_t rows_a = a.m - m0, cols_b = a.n - n0;
    // part `part` of `parts` of the contraction: an even share of its blocks
    const int blocks = (int)((a.depth + 63) / 64), tail = (int)(a.depth % 64);
    const int blk0 = (int)((int64_t)blocks * part / parts), KT = (int)((int64_t)blocks * (part + 1) / parts) - blk0;
    const bool tail_first = tail && blk0 == 0;

    // ---- global -> LDS: a lane's chunks; beyond the matrix's edge it repeats the last one (only outputs that are not stored see it) ----
    const int64_t step_a = A_COL ? 64 * a.lda * 2 : 128, step_b = 64 * a.ldb * 2;
    const uint8_t* base_a = reinterpret_cast<const uint8_t*>(a.A + (A_COL ? m0 : m0 * a.lda));
    const uint8_t* base_b = reinterpret_cast<const uint8_t*>(a.B + n0);
    // block b > 0 is block b - 1 of memory when the last one is not full and comes first
    if (tail) {
        base_a -= step_a;
        base_b -= step_b;
    }
    base_a += blk0 * step_a;
    base_b += blk0 * step_b;
    base_a = reinterpret_cast<const uint8_t*>(uniform64(base_a));
    base_b = reinterpret_cast<const uint8_t*>(uniform64(base_b));
    using wA = std::integral_constant<int, BM>;
    using wB = std::integral_constant<int, BN>;
    // An operand staged as it lies in memory: a request fills 1 KiB of consecutive rows (512 / width of them). A wave takes requests whose rows
    // have one and the same key in every lane, so that one register of lane offsets serves them all and the rows between them are scalar.
    auto col_unit = [&](auto width, int s) {               // request s of this wave, counted in 1 KiB pieces of the tile
        constexpr int W = decltype(width)::value;
        if constexpr (W == 256) return (wave & 1) | (s & 1) << 1 | (wave >> 1 & 1) << 2 | (s >> 1) << 3 | (wave >> 2) << 4;   // 2 rows each
        else return wave + s * NW;                                                                                  // 4 rows each
    };
    uint32_t oa, ob;
    int a_row = 0;                                         // row-major A: the lane's row of request 0; oa its chunk in the row
    auto row_unit = [&](int s) { return (wave & 1) + 2 * s + (wave >> 1) * (2 * A_PER_W); };      // 8 rows each, one chunk order
    auto col_offset = [&](auto width, int64_t ld, int64_t valid) {
        constexpr int W = decltype(width)::value, CH = W / 8;
        const int row = col_unit(width, 0) * (512 / W) + lane / CH, c = (lane % CH) ^ (row_key(row) << 1);
        return (uint32_t)(lane / CH * ld * 2 + min((int64_t)c * 8, valid - 8) * 2);
    };
    if constexpr (A_COL) {
        oa = col_offset(wA{}, a.lda, rows_a);
    } else {
        int c;
        unswz8(row_unit(0) * 64 + lane, a_row, c);
        oa = c * 16;
    }
    ob = col_offset(wB{}, a.ldb, cols_b);
    auto gload_one = [&](int kt, int buf, auto n_tag) {
        constexpr int n = decltype(n_tag)::value;
        const uint32_t base = lds0 + buf * L::kStage;
        if constexpr (n < A_PER_W && A_COL) {
            const int u = col_unit(wA{}, n);
            lds_dma16_so(base_a + kt * step_a + u * (512 / BM) * a.lda * 2, oa, base + u * 1024);
        } else if constexpr (n < A_PER_W) {
            // (formed anew for each request: as four registers the offsets did not fit beside the fragments)
            int row = a_row;
            asm volatile("" : "+v"(row));
            row = min(row + 16 * n, (int)rows_a - 1);
            lds_dma16_so(base_a + kt * step_a, (uint32_t)row * (uint32_t)(a.lda * 2) + oa, base + row_unit(n) * 1024);
        } else if constexpr (n < LOADS) {
            const int u = col_unit(wB{}, n - A_PER_W);
            lds_dma16_so(base_b + kt * step_b + u * (512 / BN) * a.ldb * 2, ob, base + L::kA + u * 1024);
        }
    };
    auto gload = [&](int kt, int buf) { static_for<LOADS>([&](auto n) { gload_one(kt, buf, n); }); };
    auto gload_tail = [&]() {                                          // stage 0 when it is the partial block
        static_for<LOADS>([&](auto n_tag) {
            constexpr int n = decltype(n_tag)::value;
            int at;
            bool in;
            if constexpr (n < A_PER_W && !A_COL) {
                in = (int)oa / 2 < tail;
                at = row_unit(n) * 1024;
            } else if constexpr (n < A_PER_W && A_COL) {
                const int u = col_unit(wA{}, n);
                in = u * (512 / BM) + lane / (BM / 8) < tail;
                at = u * 1024;
            } else {
                const int u = col_unit(wB{}, n - A_PER_W);
                in = u * (512 / BN) + lane / (BN / 8) < tail;
                at = L::kA + u * 1024;
            }
            if (in) gload_one(blocks, 0, n_tag);
            else *reinterpret_cast<uint4*>(smem + at + lane * 16) = make_uint4(0, 0, 0, 0);
        });
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // ---- fragments: two sets, one per half of a stage ----------------------------------------------------
    const int li = lane & 15, kb = lane >> 4;
    struct Frags {
        Frag8 a[TM], b[TN];
    } f[2];
    // Column block q of a tile staged as it lies in memory: (q ^ key) * 32 is lane_key ^ (q * 32) with everything else in the lane's address
    // a multiple of 256 or below 32, so that one exclusive or with a constant leads from block to block.
    typedef __attribute__((address_space(3))) uint8_t* lds_ptr;
    const int tr_row = 8 * kb + (li >> 2), tr_lane = (row_key(tr_row) << 5) + (li & 3) * 8;
    uint32_t tr_a = lds0 + tr_row * (BM * 2) + tr_lane + wm * TM * 32, tr_b = lds0 + L::kA + tr_row * (BN * 2) + tr_lane + wn * TN * 32;
    static_assert(TM == 8 || !A_COL || (TM == 4 && BM == 128), "column blocks of a wave: an aligned run of at most eight");
    static_assert(TN == 8 || TN == 4 || TN == 2, "likewise");
    if constexpr (TM < 8) tr_a = lds0 + tr_row * (BM * 2) + (tr_lane ^ (wm * TM * 32 & 255)) + (wm * TM * 32 & ~255);
    if constexpr (TN < 8) tr_b = lds0 + L::kA + tr_row * (BN * 2) + (tr_lane ^ (wn * TN * 32 & 255)) + (wn * TN * 32 & ~255);
    auto tr_frag = [&](uint32_t at, auto width, auto half) {
        constexpr int W = decltype(width)::value * 2, H = decltype(half)::value;
        typedef __attribute__((address_space(3))) bf16x4* lds4;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4)((lds_ptr)(uintptr_t)at + 32 * H * W));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4)((lds_ptr)(uintptr_t)at + 32 * H * W + 4 * W));
        return bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    auto read_item = [&](int buf, auto half_tag, auto e_tag) {         // tr_a and tr_b point into buffer buf already
        constexpr int H = decltype(half_tag)::value, e = decltype(e_tag)::value;
        if constexpr (e < TM && A_COL) {
            f[H].a[e].v = tr_frag(tr_a ^ (e * 32), wA{}, half_tag);
        } else if constexpr (e < TM) {
            f[H].a[e].u = *reinterpret_cast<const uint4*>(smem + buf * L::kStage + swz8(wm * WTM + e * 16 + li, 4 * H + kb));
        } else {
            f[H].b[e - TM].v = tr_frag(tr_b ^ ((e - TM) * 32), wB{}, half_tag);
        }
    };
    // Sums of A (the bias gradient): A times a matrix of ones, the row blocks of a wave's row of tiles dealt over the waves that share them.
    constexpr int SUMS = A_COL ? TM / WAVES_N : 0;
    static_assert(!A_COL || TM % WAVES_N == 0, "row blocks divide over the waves");
    const bool sum_rows = A_COL && a.row_sums && n0 == 0;
    f32x4 sums[SUMS ? SUMS : 1];
    sums[0] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (SUMS > 1)
#pragma unroll
        for (int u = 1; u < SUMS; ++u) sums[u] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add_rows = [&](auto h_tag) {
        constexpr int H = decltype(h_tag)::value;
        const bf16x8 one = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        static_for<(H < 2 ? WAVES_N : 0)>([&](auto w_tag) {
            constexpr int w = decltype(w_tag)::value;
            if (wn == w)
                static_for<SUMS>([&](auto u) {
                    constexpr int i = w * SUMS + decltype(u)::value;
                    sums[decltype(u)::value] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[H].a[i].v, one, sums[decltype(u)::value], 0, 0, 0);
                });
        });
    };
    constexpr int NMMA = TM * TN, ITEMS = TM + TN;
    // Matrix work of half H; behind it the fragments of the other half (of buffer rbuf) and LO <= n < HI of the requests of stage kt_load.
    auto half = [&](auto h_tag, auto read_tag, int rbuf, auto lo_tag, auto hi_tag, int kt_load, int buf) {
        constexpr int H = decltype(h_tag)::value, LO = decltype(lo_tag)::value, CNT = decltype(hi_tag)::value - LO;
        constexpr int RPM = (ITEMS + NMMA - 1) / NMMA, LPM = (CNT + NMMA - 1) / NMMA;
        asm volatile("" : "+v"(tr_b));                  // one register, not an address per column block kept through the loop
        if constexpr (A_COL) asm volatile("" : "+v"(tr_a));
        static_for<NMMA>([&](auto n_tag) {
            constexpr int n = decltype(n_tag)::value, i = n % TM, j = n / TM;
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[H].a[i].v, f[H].b[j].v, acc[i][j], 0, 0, 0);
            if constexpr (decltype(read_tag)::value) {
                constexpr int r0 = n * RPM < ITEMS ? n * RPM : ITEMS, r1 = (n + 1) * RPM < ITEMS ? (n + 1) * RPM : ITEMS;
                static_for<r1 - r0>([&](auto e) { read_item(rbuf, std::integral_constant<int, 1 - H>{}, std::integral_constant<int, r0 + decltype(e)::value>{}); });
            }
            constexpr int g0 = n * LPM < CNT ? n * LPM : CNT, g1 = (n + 1) * LPM < CNT ? (n + 1) * LPM : CNT;
            static_for<g1 - g0>([&](auto e) { gload_one(kt_load, buf, std::integral_constant<int, LO + g0 + decltype(e)::value>{}); });
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (A_COL)
            if (sum_rows) add_rows(h_tag);
    };
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    if (KT > 0) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s)
            if (s < KT) {
                if (s == 0 && tail_first) gload_tail();
                else gload(s, s);
            }
        if (KT >= STAGES) wait_vmcnt_lgkm0<(STAGES - 1) * LOADS>();
        else wait_vmcnt_lgkm0<0>();
        barrier();
        static_for<ITEMS>([&](auto e) { read_item(0, std::integral_constant<int, 0>{}, e); });
        wait_vmcnt_lgkm0<63>();
        // Inside stage kt: first half of its matrix work, the reads of its second half, (ring of three and more) the rest of the requests of
        // stage kt + STAGES - 1 | own reads done, stage kt + 1 landed | barrier | second half, the first reads of stage kt + 1 and the
        // requests of stage kt + STAGES into the buffer that nobody reads any more.
        constexpr int SPLIT = STAGES == 2 ? LOADS : (LOADS + 1) / 2;
        using c0 = std::integral_constant<int, 0>;
        using c1 = std::integral_constant<int, 1>;
        using cS = std::integral_constant<int, SPLIT>;
        using cL = std::integral_constant<int, LOADS>;
        using T = std::true_type;
        using F = std::false_type;
        int cur = 0;
        auto stage_step = [&](int kt, auto load_a, auto load_b, auto has_next, auto pending) {
            const int nxt = cur + 1 == STAGES ? 0 : cur + 1, prv = cur == 0 ? STAGES - 1 : cur - 1;
            using a_lo = std::conditional_t<decltype(load_a)::value, cS, c0>;
            using a_hi = std::conditional_t<decltype(load_a)::value, cL, c0>;
            using b_hi = std::conditional_t<decltype(load_b)::value, cS, c0>;
            half(c0{}, T{}, cur, a_lo{}, a_hi{}, kt + STAGES - 1, prv);
            wait_vmcnt_lgkm0<decltype(pending)::value * LOADS>();
            barrier();
            tr_a += (nxt - cur) * L::kStage;
            tr_b += (nxt - cur) * L::kStage;
            half(c1{}, has_next, nxt, c0{}, b_hi{}, kt + STAGES, cur);
            cur = nxt;
        };
        using P = std::integral_constant<int, STAGES - 2>;
        static_assert(STAGES == 2 || STAGES == 3 || STAGES == 4, "ring depth");
        int kt = 0;
        if constexpr (STAGES == 2) {
            for (; kt < KT - 2; ++kt) stage_step(kt, F{}, T{}, T{}, P{});
            // (the last stage reads fragments that nobody uses: a step of its own without them came out of the compiler with spills)
            for (; kt < KT; ++kt) stage_step(kt, F{}, F{}, T{}, P{});
        } else {
          if (KT > STAGES) {
            stage_step(kt, F{}, T{}, T{}, P{});
            for (kt = 1; kt < KT - STAGES; ++kt) stage_step(kt, T{}, T{}, T{}, P{});
            stage_step(kt, T{}, F{}, T{}, P{});
            ++kt;
          }
          if constexpr (STAGES >= 4) {
            if (kt == KT - 4) { stage_step(kt, F{}, F{}, T{}, std::integral_constant<int, 2>{}); ++kt; }
          }
          if (kt == KT - 3) { stage_step(kt, F{}, F{}, T{}, std::integral_constant<int, 1>{}); ++kt; }
          if (kt == KT - 2) { stage_step(kt, F{}, F{}, T{}, std::integral_constant<int, 0>{}); ++kt; }
          stage_step(kt, F{}, F{}, F{}, std::integral_constant<int, 0>{});
        }
    }

    // ---- store: register r of a block is row 4 kb + r, column li -----------------------------------------
    if constexpr (A_COL) {
        if (sum_rows && li == 0) {
#pragma unroll
            for (int u = 0; u < SUMS; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t row = m0 + wm * WTM + (wn * SUMS + u) * 16 + 4 * kb + r;
                    if (row >= a.m) continue;
                    if constexpr (F32) static_cast<float*>(a.row_sums)[row] = sums[u][r];
                    else static_cast<uint16_t*>(a.row_sums)[row] = (uint16_t)f32_to_bf16_rne(sums[u][r]);
                }
        }
    }
    if constexpr (F32) {
        // row block by row block through LDS, so that rows leave in whole lines
        wait_vmcnt_lgkm0<0>();
        barrier();                                   // the ring is free
        constexpr int ROWB = WTN * 4 + 16, CPR = WTN / 4;
        static_assert(NW * 16 * ROWB <= L::kTotal, "row blocks fit in the ring");
        uint8_t* ep = smem + wave * (16 * ROWB);
        float* C = static_cast<float*>(a.C);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) *reinterpret_cast<float*>(ep + (4 * kb + r) * ROWB + (j * 16 + li) * 4) = acc[i][j][r];
            // (LDS operations of a wave complete in order)
#pragma unroll
            for (int q0 = 0; q0 < 16 * CPR; q0 += 64) {
                const int rl = (q0 + lane) / CPR, c = (q0 + lane) % CPR;
                const int64_t row = m0 + wm * WTM + i * 16 + rl, col = n0 + wn * WTN + c * 4;
                const float4 v = *reinterpret_cast<const float4*>(ep + rl * ROWB + c * 16);
                if (row < a.m && col < a.n) *reinterpret_cast<float4*>(C + row * a.ldc + col) = v;
            }
        }
    } else {
        // (the lane's numbers formed again: kept through the loop they cost registers there)
        int lane = threadIdx.x;
        asm volatile("" : "+v"(lane));
        lane &= 63;
        const int li = lane & 15, kb = lane >> 4;
        // through LDS, so that rows leave in 16-byte pieces; two lanes of neighbouring columns first trade halves, so that each writes two
        // columns of one row
        wait_vmcnt_lgkm0<0>();
        barrier();                                   // the ring is free
        uint8_t* ep = smem + wave * (WTM * L::kEpiRow);
        const bool odd = lane & 1;
        const uint32_t sel = odd ? 0x03020706u : 0x05040100u;
        uint8_t* const ep_lane = ep + (4 * kb + (odd ? 2 : 0)) * L::kEpiRow + (li & ~1) * 2;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const f32x2 pv = {acc[i][j][r], acc[i][j][r + 2]};
                    const uint32_t own = __builtin_bit_cast(uint32_t, __builtin_convertvector(pv, bf16x2));      // RNE
                    const uint32_t partner = (uint32_t)__builtin_amdgcn_mov_dpp((int)own, 0xB1, 0xF, 0xF, true);
                    *reinterpret_cast<uint32_t*>(ep_lane + (i * 16 + r) * L::kEpiRow + j * 32) = __builtin_amdgcn_perm(partner, own, sel);
                }
        uint16_t* C = static_cast<uint16_t*>(a.C);
        constexpr int CPR = WTN / 8, CHUNKS = WTM * CPR;
#pragma unroll
        for (int q0 = 0; q0 < CHUNKS; q0 += 64) {
            const int q = q0 + lane, rl = q / CPR, c = q % CPR;
            const int64_t row = m0 + wm * WTM + rl, col = n0 + wn * WTN + c * 8;
            if (q < CHUNKS && row < a.m && col < a.n)
                *reinterpret_cast<uint4*>(C + row * a.ldc + col) = *reinterpret_cast<const uint4*>(ep + rl * L::kEpiRow + c * 16);
        }
    }
}

__device__ __forceinline__ GradArgs dgrad_problem(const GroupedGradArgs& a, int expert, int begin, int rows) {
    GradArgs g;
    g.A = a.dY + begin * a.lddy;
    g.lda = a.lddy;
    g.B = a.W + expert * a.w_stride;
    g.ldb = a.ldw;
    g.C = static_cast<uint16_t*>(a.out) + begin * a.ldo;
    g.ldc = a.ldo;
    g.m = rows;
    g.n = a.K;
    g.depth = a.N;
    return g;
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64) void dgrad_kernel(const GroupedGradArgs a) {
    GroupTile t;
    const int tiles_n = (int)((a.K + BN - 1) / BN);
    if (!group_tile(a.offsets, a.experts, (int)a.T, BM, tiles_n, t)) return;
    int pm, pn;
    tile_walk<16>(t.tile, (t.rows + BM - 1) / BM, tiles_n, pm, pn);
    grad_tile<false, false, BM, BN, WAVES_M, WAVES_N, STAGES>(dgrad_problem(a, t.expert, t.begin, t.rows), (int64_t)pm * BM, (int64_t)pn * BN);
}

__global__ __launch_bounds__(512) void dgrad_mixed_kernel(const GroupedGradArgs a) {
    const int tiles_n = (int)((a.K + 255) / 256);
    mixed_tiles(a.offsets, a.experts, (int)a.T, tiles_n, (int)((a.N + 63) / 64), [&](const MixedTile& t) {
        const GradArgs g = dgrad_problem(a, t.expert, t.begin, t.rows);
        int pm, pn;
        if (t.tall) {
            tile_walk<8>(t.tile, t.panels, tiles_n, pm, pn);
            grad_tile<false, false, 256, 256, 2, 4, 2>(g, (int64_t)pm * 256, (int64_t)pn * 256);
        } else {
            tile_walk<16>(t.tile, t.panels, tiles_n, pm, pn);
            grad_tile<false, false, 128, 256, 2, 4, 3>(g, (int64_t)pm * 128, (int64_t)pn * 256);
        }
    });
}

template <bool F32, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64) void wgrad_kernel(const GroupedGradArgs a) {
    // Every XCD takes an eighth of every expert's tiles (neighbours in the walk), so that uneven experts do not make uneven XCDs; which
    // eighth turns with the expert, for experts of fewer than eight tiles.
    const int tiles_m = (int)((a.N + BM - 1) / BM), tiles_n = (int)((a.K + BN - 1) / BN), tiles = tiles_m * tiles_n, per = (tiles + 7) / 8;
    const int one = a.experts * 8 * per, part = (int)blockIdx.x / one, id = (int)blockIdx.x % one;
    const int e = id / 8 / per, share = (id + e + part) % 8;
    const int t = xcd_share_start(tiles, share) + id / 8 % per;
    if (t >= xcd_share_start(tiles, share + 1)) return;
    const RowRange r = expert_rows(a.offsets, e, (int)a.T);
    GradArgs g;
    g.A = a.dY + r.begin * a.lddy;
    g.lda = a.lddy;
    g.B = a.X + r.begin * a.ldx;
    g.ldb = a.ldx;
    if constexpr (F32) g.C = static_cast<float*>(a.out) + (part * a.experts + e) * a.o_stride;
    else g.C = static_cast<uint16_t*>(a.out) + e * a.o_stride;
    g.ldc = a.ldo;
    g.m = a.N;
    g.n = a.K;
    g.depth = r.end - r.begin;
    if constexpr (F32) g.row_sums = a.bias_out ? static_cast<float*>(a.bias_out) + (part * a.experts + e) * a.N : nullptr;
    else g.row_sums = a.bias_out ? static_cast<uint16_t*>(a.bias_out) + e * a.N : nullptr;
    int pm, pn;
    tile_walk<8>(t, tiles_m, tiles_n, pm, pn);
    grad_tile<true, F32, BM, BN, WAVES_M, WAVES_N, STAGES>(g, (int64_t)pm * BM, (int64_t)pn * BN, part, a.parts);
}

// Adds the parts' planes up in order: dW four columns to a thread, behind them the bias gradient one element to a thread.
__global__ __launch_bounds__(256) void wgrad_reduce_kernel(const GroupedGradArgs a, const float* planes, const float* bias_planes) {
    const int64_t all = (int64_t)a.experts * a.N * (a.K / 4), q = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (q < all) {
        const int64_t row = q / (a.K / 4), col = q % (a.K / 4) * 4, e = row / a.N, n = row % a.N;
        const float* p = planes + row * a.K + col;
        float4 s = *reinterpret_cast<const float4*>(p);
        for (int i = 1; i < a.parts; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(p + i * ((int64_t)a.experts * a.N * a.K));
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const int64_t at = e * a.o_stride + n * a.ldo + col;
        if (a.f32) {
            *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = s;
        } else {
            const uint32_t lo = f32_to_bf16_rne(s.x) | f32_to_bf16_rne(s.y) << 16, hi = f32_to_bf16_rne(s.z) | f32_to_bf16_rne(s.w) << 16;
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = make_uint2(lo, hi);
        }
    } else if (a.bias_out && q - all < a.experts * a.N) {
        const int64_t n = q - all;
        float s = bias_planes[n];
        for (int i = 1; i < a.parts; ++i) s += bias_planes[i * (a.experts * a.N) + n];
        if (a.f32) static_cast<float*>(a.bias_out)[n] = s;
        else static_cast<uint16_t*>(a.bias_out)[n] = (uint16_t)f32_to_bf16_rne(s);
    }
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
struct Grad {
    using L = GradSmem<BM, BN, WAVES_M, WAVES_N, STAGES>;
    static int64_t dgrad_grid(int64_t T, int64_t E, int64_t K) { return group_grid(T, E, K, BM, BN); }
    static int64_t wgrad_grid(int64_t E, int64_t N, int64_t K) { return E * 8 * ((((N + BM - 1) / BM) * ((K + BN - 1) / BN) + 7) / 8); }
    static constexpr dim3 block() { return dim3(WAVES_M * WAVES_N * 64); }
    static hipError_t limit(const void* k) { return hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, L::kTotal); }
    static hipError_t prepare_dgrad() { return limit(reinterpret_cast<const void*>(dgrad_kernel<BM, BN, WAVES_M, WAVES_N, STAGES>)); }
    static hipError_t prepare_wgrad() {
        const hipError_t e = limit(reinterpret_cast<const void*>(wgrad_kernel<false, BM, BN, WAVES_M, WAVES_N, STAGES>));
        return e != hipSuccess ? e : limit(reinterpret_cast<const void*>(wgrad_kernel<true, BM, BN, WAVES_M, WAVES_N, STAGES>));
    }
    static hipError_t dgrad(const GroupedGradArgs& a, hipStream_t stream) {
        hipLaunchKernelGGL((dgrad_kernel<BM, BN, WAVES_M, WAVES_N, STAGES>), dim3((unsigned)dgrad_grid(a.T, a.experts, a.K)), block(),
                           L::kTotal, stream, a);
        return hipGetLastError();
    }
    static hipError_t wgrad(const GroupedGradArgs& a, hipStream_t stream) {
        const dim3 grid((unsigned)(wgrad_grid(a.experts, a.N, a.K) * a.parts));
        if (a.f32) hipLaunchKernelGGL((wgrad_kernel<true, BM, BN, WAVES_M, WAVES_N, STAGES>), grid, block(), L::kTotal, stream, a);
        else hipLaunchKernelGGL((wgrad_kernel<false, BM, BN, WAVES_M, WAVES_N, STAGES>), grid, block(), L::kTotal, stream, a);
        return hipGetLastError();
    }
};

struct DgradMixed {
    using L0 = GradSmem<256, 256, 2, 4, 2>;
    using L1 = GradSmem<128, 256, 2, 4, 3>;
    static constexpr int kLds = L0::kTotal > L1::kTotal ? L0::kTotal : L1::kTotal;
    static int64_t dgrad_grid(int64_t T, int64_t E, int64_t K) { return group_grid(T, E, K, 128, 256); }
    static hipError_t prepare_dgrad() {
        return hipFuncSetAttribute(reinterpret_cast<const void*>(dgrad_mixed_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    }
    static hipError_t dgrad(const GroupedGradArgs& a, hipStream_t stream) {
        hipLaunchKernelGGL(dgrad_mixed_kernel, dim3(kUnits), dim3(512), kLds, stream, a);
        return hipGetLastError();
    }
};

template <class Op>
auto with_dgrad(int shape, Op op) {
    switch (shape) {
        case 0: return op(Grad<64, 128, 1, 4, 4>{});
        case 1: return op(Grad<128, 128, 2, 2, 4>{});
        default: return op(DgradMixed{});
    }
}
template <class Op>
auto with_wgrad(int shape, Op op) {
    if (shape == 0) return op(Grad<128, 128, 2, 2, 4>{});
    if (shape == 2) return op(Grad<128, 128, 2, 2, 2>{});
    return op(Grad<256, 256, 2, 4, 2>{});
}

}  // namespace

// The tile with the least estimated time (as in grouped.hip; `stage`: 64 of the contraction). Over 315 problems as there the input gradient's choice is 3 %, the
// weight gradient's 1 % slower in the mean than the best.
int dgrad_shape(int64_t T, int64_t E, int64_t N, int64_t K) {
    const double stages = (double)((N + 63) / 64), halves = group_panels(T, E, 128) * (double)((K + 255) / 256), rounds = halves > 256 ? halves / 256 : 1;
    double best = 6.0 + (rounds - 1) * 4.5 + (0.6 + 0.15 * (halves < 256 ? halves / 256 : 1)) * stages * rounds;
    int pick = 2;
    for (int i = 0; i < 2; ++i) {
        const double tiles = group_panels(T, E, i ? 128 : 64) * (double)((K + 127) / 128), passes = tiles > 256 ? tiles / 256 : 1;
        const double fixed = i ? 4.8 : 3.8, stage = (i ? 0.53 : 0.305) * (1 + (i ? 0.06 : 0.13) * (passes < 2 ? passes - 1 : 1));
        const double us = fixed * (1 + 0.6 * (passes - 1)) + stage * stages * passes;
        if (us < best) {
            best = us;
            pick = i;
        }
    }
    return pick;
}
// Weight gradient: the tile, and in how many parts the rows are cut where the tiles leave units idle and there are many rows to an expert: each part leaves an fp32
// plane in the workspace and a second launch adds them up (3.5 us and the planes' way there and back at 3.5 TB/s).
struct WgradPlan {
    int shape, parts;
};
static size_t wgrad_plane(int64_t E, int64_t N, int64_t K) { return (size_t)E * (size_t)N * (size_t)(K + 1) * 4; }
static WgradPlan wgrad_plan(int64_t T, int64_t E, int64_t N, int64_t K, size_t room) {
    const double rows = T > 0 ? (double)T / (double)(E < T ? E : T) : 0, stages = rows / 64 + 0.5;
    auto us = [&](int shape, int parts) {
        const int64_t side = shape == 1 ? 256 : 128;
        const double tiles = (double)parts * (double)(E * ((N + side - 1) / side) * ((K + side - 1) / side)), passes = tiles > 256 ? tiles / 256 : 1;
        const double fixed = shape == 0 ? 4.8 : shape == 1 ? 9.0 : 4.0;
        // (a ring of two leaves room for two workgroups a unit, which pull more slowly each)
        const double stage = shape == 0 ? 0.53 : shape == 1 ? 1.5 : passes < 2 ? 0.785 - 0.255 * (passes - 1) : 0.53;
        return fixed * (1 + (shape == 1 ? 0.9 : 0.78) * (passes - 1)) + stage * (stages / parts) * passes;
    };
    WgradPlan plan{0, 1};
    double best = us(0, 1);
    for (int shape = 1; shape < 3; ++shape)
        if (us(shape, 1) < best) {
            best = us(shape, 1);
            plan.shape = shape;
        }
    for (int parts = 2; parts <= 64 && parts * 2 <= stages; parts *= 2) {
        const double bytes = (double)parts * (double)wgrad_plane(E, N, K);
        if (bytes > (double)room) break;
        const double t = us(0, parts) + 3.5 + bytes * 2 / 3.5e6;
        if (t < best * 0.95) {
            best = t;
            plan = WgradPlan{0, parts};
        }
    }
    return plan;
}
void wgrad_choice(int64_t T, int64_t E, int64_t N, int64_t K, size_t room, int out[2]) {
    const WgradPlan plan = wgrad_plan(T, E, N, K, room);
    out[0] = plan.shape;
    out[1] = plan.parts;
}
size_t wgrad_workspace(int64_t T, int64_t E, int64_t N, int64_t K, size_t room) {
    const int parts = wgrad_plan(T, E, N, K, room).parts;
    return parts > 1 ? (size_t)parts * wgrad_plane(E, N, K) : 0;
}

int64_t dgrad_grid(int64_t T, int64_t E, int64_t N, int64_t K) {
    return with_dgrad(dgrad_shape(T, E, N, K), [&](auto k) { return decltype(k)::dgrad_grid(T, E, K); });
}
int64_t wgrad_grid(int64_t T, int64_t E, int64_t N, int64_t K, size_t room) {
    const WgradPlan plan = wgrad_plan(T, E, N, K, room);
    return with_wgrad(plan.shape, [&](auto k) { return decltype(k)::wgrad_grid(E, N, K) * (decltype(k)::block().x / 256); }) * plan.parts;
}

hipError_t prepare_grouped_grad_kernels() {
    hipError_t e = hipSuccess;
    for (int i = 0; i < 3 && e == hipSuccess; ++i) e = with_dgrad(i, [](auto k) { return decltype(k)::prepare_dgrad(); });
    for (int i = 0; i < 3 && e == hipSuccess; ++i) e = with_wgrad(i, [](auto k) { return decltype(k)::prepare_wgrad(); });
    hipFuncAttributes attr;
    if (e == hipSuccess) e = hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(wgrad_reduce_kernel));
    return e;
}

hipError_t launch_grouped_dgrad(const GroupedGradArgs& a, hipStream_t stream) {
    return with_dgrad(dgrad_shape(a.T, a.experts, a.N, a.K), [&](auto k) { return decltype(k)::dgrad(a, stream); });
}

hipError_t launch_grouped_wgrad(const GroupedGradArgs& a_in, void* workspace, size_t room, hipStream_t stream) {
    GroupedGradArgs a = a_in;
    const WgradPlan plan = wgrad_plan(a.T, a.experts, a.N, a.K, room);
    a.parts = plan.parts;
    if (plan.parts == 1) return with_wgrad(plan.shape, [&](auto k) { return decltype(k)::wgrad(a, stream); });
    GroupedGradArgs part = a;
    float* planes = static_cast<float*>(workspace);
    float* bias_planes = planes + (size_t)plan.parts * a.experts * a.N * a.K;
    part.f32 = true;
    part.out = planes;
    part.bias_out = a.bias_out ? bias_planes : nullptr;
    part.ldo = a.K;
    part.o_stride = a.N * a.K;
    const hipError_t e = with_wgrad(plan.shape, [&](auto k) { return decltype(k)::wgrad(part, stream); });
    if (e != hipSuccess) return e;
    const int64_t work = a.experts * a.N * (a.K / 4) + (a.bias_out ? a.experts * a.N : 0);
    hipLaunchKernelGGL(wgrad_reduce_kernel, dim3((unsigned)((work + 255) / 256)), dim3(256), 0, stream, a, planes, bias_planes);
    return hipGetLastError();
}

}  // namespace rtl
