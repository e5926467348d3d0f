// Grouped product of 8-bit rows and weights with a ring of operand units: the scheme of gemm_ring.hpp (units of 64 or 128 rows of 128 bytes,
// read one phase before they are multiplied, refilled two slabs ahead at one barrier a phase) on the scaled 8-bit matrix
// instructions.  A slab is one block of 128 k, so a row of it has one scale, and so has a 128-column block of the weights:
//   * the scales of a slab travel with its unit A0: every wave loads one line of 256 bytes, wave 0 those of the tile's rows, wave 1 the word
//     that holds those of its column blocks; they lie behind the stage's operands in LDS;
//   * a lane reads its rows' bytes together with A0 and hands them to the instruction, which multiplies them in.
// What bounds it: the latency of the units, 2 us under load, against 7 of 8 slots in flight (112 KB a CU with two workgroups, 84 KB with one of 128 x
// 256), and the epilogue, which adds to it: 64 groups x 256 rows, 1024 -> 4096, GELU and 8-bit rows: 81 us without an epilogue, 118 without its
// stores, 131 in all (1.05 PFLOP/s; its bytes take 68, 52 of them the weights).  Per slab 128 x 128 moves 64 KB through L2 for 1024 matrix
// cycles of a CU, two workgroups side by side; 8192 x 8192 x 8192 2.2 PFLOP/s (2.4 in tiles of 128 x 256; a library product 2.9, at the 1.6 GHz
// that the power limit leaves).  Tried and taken back: the epilogue in slices beside the next tile's phases from a second set of accumulators
// (no gain: one wave issues a vector instruction every 5.5 cycles), 256 x 256 tiles (spill), requests into L2 a tile ahead (slower).
// GELU with its 8-bit output takes 25 vector instructions an output.
//
// The 8-bit epilogue needs the largest magnitude of a row in a block of 128 columns, which two waves share (and, in tiles of 128 columns,
// both parts of each): the waves exchange theirs through LDS.
#pragma once

#include <type_traits>

#include "fp8_internal.hpp"
#include "fp8_mfma.hpp"

namespace smile {

namespace {

enum { kFp8Y, kFp8Rows, kFp8Slope };   // y alone; 8-bit rows too; both times the activation's derivative at kept 8-bit rows

// QA0, QA1 / QB0, QB1: 32-wide blocks per wave in the units A0, A1 / B0, B1.  KIND: what the epilogue does.  ACT: the activation, 0 none, 1 ReLU, 3 GELU
// (of the kernel, not of the call: the branches would copy every accumulator).
template <int QA0, int QA1, int QB0, int QB1, int OCC, int KIND, int ACT>
__global__ __launch_bounds__(256, OCC) void fp8_gemm_ring_kernel(Fp8Gemm a)
{
#ifdef __HIP_DEVICE_COMPILE__   // (the host has no type for a buffer resource)
    constexpr int NW = 4, BM = 64 * (QA0 + QA1), BN = 64 * (QB0 + QB1), TM = QA0 + QA1, TN = QB0 + QB1, CB = BN / kFp8Block;
    enum { A0, B0, B1, A1 };                                            // units of a slab, in the order of the ring
    constexpr int kExt[4] = {64 * QA0, 64 * QB0, 64 * QB1, 64 * QA1};   // rows (columns) of a unit
    constexpr int kOff[4] = {0, kExt[0] * 128, (kExt[0] + kExt[1]) * 128, (kExt[0] + kExt[1] + kExt[2]) * 128};
    constexpr int kCnt[4] = {2 * QA0 + 1, 2 * QB0, 2 * QB1, 2 * QA1};   // load instructions per wave; the last of A0: scales
    constexpr int kCode[4] = {2 * QA0, 2 * QB0, 2 * QB1, 2 * QA1};      // ... of codes
    constexpr int kFirst[4] = {0, kCode[0], kCode[0] + kCode[1], kCode[0] + kCode[1] + kCode[2]};
    constexpr int kReads[4] = {4 * QA0 + TM + 1, 4 * QB0, 4 * QB1, 4 * QA1};   // LDS reads per wave
    constexpr int GPW = 2 * (TM + TN), SCALES = (BM + BN) * 128, STAGE = SCALES + NW * 256;
    constexpr int QB = QB0;                                       // both parts of a tile's columns are as wide
    constexpr int SROW = QB * 64 + 16;                            // bytes of a staged row
    constexpr int STAGING = NW * 32 * SROW, LARGEST = KIND != kFp8Y ? 2 * CB * BM * 4 : 0;   // one exchange of magnitudes: [wn][block][row]
    static_assert(QB0 == QB1 && (CB == 1 || CB == 2) && BN == CB * kFp8Block && QA0 >= 1 && QA1 >= 1 && QA0 <= 2 && QA1 <= 2, "tile shapes");
    static_assert((2 * STAGE + STAGING + 2 * LARGEST) * OCC <= kLdsPerCu, "LDS");
    __shared__ __attribute__((aligned(16))) char ring_lds[2 * STAGE + STAGING + 2 * LARGEST];
    lds_char *const lds = (lds_char *)ring_lds;
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
    typedef __attribute__((address_space(3))) uint32_t lds_u32;
    typedef __attribute__((address_space(3))) uint8_t lds_u8;

    const int S = a.KB, pitch = a.KB * kFp8Block;
    LiveTileWalk<BM> walk;
    walk.init(a.rows, a.N, a.C, a.col_tiles, false);
    struct Tile {
        int e, rt, ct, rows;
    };
    // The walk's order, row tiles fastest, would pass through all rows of a large group for each of its column tiles: bands of eight row tiles instead
    // (16384 x 1024 -> 4096: 101 -> 81 us; 8192 x 8192 x 8192 638 -> 498), so that what an XCD's workgroups share stays in its L2
    auto select = [&](Tile &t) __attribute__((always_inline)) {
        if (!walk.tile(t.e, t.rt, t.ct, t.rows)) return false;
        constexpr int BAND = 8;
        const int cnt = (t.rows + BM - 1) / BM;
        if (cnt > BAND) {
            const int u = t.ct * cnt + t.rt, band = u / (BAND * a.col_tiles), v = u - band * BAND * a.col_tiles, n = min(BAND, cnt - band * BAND);
            t.ct = v / n;
            t.rt = band * BAND + v - t.ct * n;
        }
        return true;
    };
    // Per-lane indices are derived afresh wherever they are needed, from an opaque copy of the thread id, so that nothing
    // computed from them stays in registers from one part of a tile to the next.
    auto thread_id = [&]() {
        int t = threadIdx.x;
        asm volatile("" : "+v"(t));
        return t;
    };
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;

    // ---- loader.  off: this lane's byte offset from the tile's operand (xb / wb, slab 0) in each load instruction of a slab; soff, sb, sadv: the
    // same of its wave's scales
    // (buffer loads: a scalar offset for the slab, no vector arithmetic; what lies behind the last valid row is not touched)
    uint32_t off[GPW], soff;
    struct Source {   // of a buffer resource: address and bytes, put together where it is used and through readfirstlane, since a resource in
        uint32_t lo, hi, size;   // vector registers costs a loop around each load
        __device__ __forceinline__ void set(const uint8_t *p, size_t bytes)
        {
            const uint64_t at = reinterpret_cast<uint64_t>(p);
            lo = (uint32_t)at, hi = (uint32_t)(at >> 32), size = bytes < 0xffffffffu ? (uint32_t)bytes : 0xffffffffu;
        }
        __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource() const
        {
            const uint32_t l = __builtin_amdgcn_readfirstlane(lo), h = __builtin_amdgcn_readfirstlane(hi);
            return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(((uint64_t)h << 32) | l), 0, (int)__builtin_amdgcn_readfirstlane(size), 0x00027000);
        }
    } xb = {}, wb = {}, scb = {};
    const uint32_t sadv = wave & 1 ? a.Ws : a.Cs;
    auto set_sources = [&](const Tile &t) __attribute__((always_inline)) {
        const int row0 = t.rt * BM, col0 = t.ct * BN;
        xb.set(a.x + ((size_t)t.e * a.C + row0) * pitch, (size_t)(t.rows - row0) * pitch);
        wb.set(a.w + ((size_t)t.e * a.Nout + col0) * pitch, (size_t)(a.Nout - col0) * pitch);
        const int lane = thread_id() & 63;
        for_constants<4>([&](auto type) {
            constexpr int T = decltype(type)::value;
            constexpr bool IS_X = T == A0 || T == A1;
            constexpr int FIRST = T == A1 ? kExt[A0] : T == B1 ? kExt[B0] : 0;
            const int last = IS_X ? t.rows - 1 - row0 : a.Nout - 1 - col0;   // rows beyond the last valid one re-read it
#pragma unroll
            for (int i = 0; i < kCode[T]; ++i) {
                const int r = (wave + i * NW) * 8 + (lane >> 3), piece = (lane & 7) ^ ((r >> 1) & 7);
                off[kFirst[T] + i] = (uint32_t)min(FIRST + r, last) * pitch + piece * 16;
            }
        });
        // (selected without a branch: the compiler would move matrix instructions behind it)
        const bool w = wave & 1;
        scb.set((w ? a.ws : a.xs) + (size_t)t.e * S * sadv, (size_t)S * sadv);
        soff = w ? t.ct * CB & ~3 : min(row0 + 4 * lane, a.Cs - 4);
    };
    // load instruction i of unit `type` of slab `slab`, into the stage `stage` bytes into LDS
    auto load_one = [&](auto type, int i, int slab, int stage) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        if (T == A0 && i == kCode[A0]) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(scb.resource(), SMILE_LPTR(lds + stage + SCALES + wave * 256), 4, soff, slab * sadv, 0, 0);
            return;
        }
        __builtin_amdgcn_raw_ptr_buffer_load_lds((T == A0 || T == A1 ? xb : wb).resource(), SMILE_LPTR(lds + stage + kOff[T] + (wave + i * NW) * 1024), 16,
                                                 off[kFirst[T] + min_int(i, kCode[T] - 1)], slab * kFp8Block, 0, 0);
    };
    auto load_unit = [&](auto type, int slab, int stage) __attribute__((always_inline)) {
        for_constants<kCnt[decltype(type)::value]>([&](auto i) { load_one(type, decltype(i)::value, slab, stage); });
    };
    // the first units of a tile whose first slab lies in `stage`, as far as it has them
    auto load_first = [&](int units, int stage) __attribute__((always_inline)) {
        for_constants<7>([&](auto v) {
            constexpr int V = decltype(v)::value;
            if (V < units) load_unit(std::integral_constant<int, V & 3>{}, V / 4, V < 4 ? stage : STAGE - stage);
        });
    };
    Tile cur;
    if (!select(cur)) return;
    set_sources(cur);
    int stage0 = 0;   // where the tile's slab 0 lies in LDS (0 or STAGE)
    load_first(4 * S, stage0);

    // The kept rows whose derivative multiplies the tile: requested in front of the next tile's units, since loads return in order.  Pieces of
    // 16 codes per lane as the epilogue stages them, and the scales of this lane's rows.
    constexpr int P8 = QB * 2, SLOPES = KIND == kFp8Slope ? TM * 2 : 1, SLOPE_SCALES = KIND == kFp8Slope ? TM * CB : 1;
    constexpr int SLOPE_LOADS = KIND == kFp8Slope ? TM * 2 * (P8 / 2) + TM * CB : 0;
    u32x4 slope[SLOPES][P8 / 2];
    uint8_t slope_scale[SLOPE_SCALES];
    auto request_slope = [&]() __attribute__((always_inline)) {
        if constexpr (KIND == kFp8Slope) {
            const int l = thread_id() & 63, blocks = (a.Nout + kFp8Block - 1) / kFp8Block;
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const int row0 = cur.rt * BM + (j < QA0 ? j * 64 : kExt[A0] + (j - QA0) * 64) + wm * 32;
#pragma unroll
                for (int H = 0; H < 2; ++H)
#pragma unroll
                    for (int it = 0; it < P8 / 2; ++it) {   // rows and columns beyond the matrix: the last ones
                        const int id = it * 64 + l, lrow = id / P8, row = min(row0 + lrow, cur.rows - 1);
                        const int col = min(cur.ct * BN + H * kExt[B0] + wn * QB * 32 + (id - lrow * P8) * 16, blocks * kFp8Block - 16);
                        slope[j * 2 + H][it] = *reinterpret_cast<const u32x4 *>(a.g8 + ((size_t)cur.e * a.C + row) * ((size_t)blocks * kFp8Block) + col);
                    }
#pragma unroll
                for (int b = 0; b < CB; ++b)
                    slope_scale[j * CB + b] = a.gs[((size_t)cur.e * blocks + min(cur.ct * CB + b, blocks - 1)) * a.Cs + min(row0 + (l & 31), cur.rows - 1)];
            }
        }
    };

    for (;;) {
    walk.advance();
    Tile nxt;
    const bool more = select(nxt);
    if (!more) nxt = cur;   // the last tile's first units are requested once more, so that the wait counts of a contraction have no branches

    // ---- fragment addressing: byte offsets of this lane in a unit; piece kk of a row at (2 kk + fhi) ^ swizzle
    const int lane = thread_id() & 63, frow = lane & 31, fhi = lane >> 5;
    int noff[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) noff[kk] = frow * 128 + (((2 * kk + fhi) ^ ((frow >> 1) & 7)) * 16);
    i32x8 fa0[QA0][2], fa1[QA1][2], fb[2][QB][2];   // whole operands of the instruction: halves would be copied together
    uint32_t sx[TM], sw, sxn[TM], swn;              // scales of this slab and of the next one
    const int wshift = 8 * (cur.ct * CB & 3);
    auto read_one = [&](auto type, auto index, const lds_char *stage) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value, Q = T == A0 ? QA0 : T == A1 ? QA1 : QB, I = decltype(index)::value;
        if constexpr (T == A0 && I >= 4 * QA0) {
            if constexpr (I == kReads[A0] - 1) {
                swn = *(const lds_u32 *)(stage + SCALES + 256);
            } else {
                constexpr int j = I - 4 * QA0;
                sxn[j] = *(const lds_u8 *)(stage + SCALES + (j < QA0 ? j * 64 : kExt[A0] + (j - QA0) * 64) + wm * 32 + frow);
            }
        } else {
            constexpr int KK = I / Q, q = I % Q;
            const int first = T == A0 || T == A1 ? wm * 32 + q * 64 : wn * Q * 32 + q * 32;
            const u32x4 v = *(const lds_u32x4 *)(stage + kOff[T] + first * 128 + noff[KK]);
            const auto take = [&](i32x8 &f) __attribute__((always_inline)) { f = KK % 2 ? set_high(f, v) : set_low(v); };
            if constexpr (T == A0) take(fa0[q][KK / 2]);
            else if constexpr (T == A1) take(fa1[q][KK / 2]);
            else take(fb[T == B1][q][KK / 2]);
        }
    };

    f32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // The products of a slab go A0 B0, A0 B1, A1 B0, A1 B1: each unit's registers are free when its next one is due.
    // Phase f: waits for unit f (every wave is then also done reading unit f - 1, whose slot is free), reads it, requests the
    // unit seven places on and multiplies fragments JA, JB (0 / 1; -1: none).  Unit f is of type f mod 4; D = f - U (U units in the
    // tile), or -32 in the steady state.  Behind unit f six units have been requested when it is waited for: of this tile, then of
    // the next one (unit v in phase U - 7 + v) if it follows.  from, to: stages of unit f and of unit f + 7; slab7: its slab.
    constexpr auto behind = [](int type, int n) {   // load instructions of the n units after one of type `type`
        int c = 0;
        for (int i = 1; i <= n; ++i) c += kCnt[(type + i) & 3];
        return c;
    };
    auto phase = [&](auto ja, auto jb, auto type, auto d, auto follow, int from, int slab7, int to) __attribute__((always_inline)) {
        constexpr int JA = decltype(ja)::value, JB = decltype(jb)::value, RT = decltype(type)::value, D = decltype(d)::value, LT = (RT + 3) & 3;
        constexpr bool FOLLOWS = decltype(follow)::value;   // the next tile's first seven units follow this tile's without a gap
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): this wave's reads of unit f - 1
        if constexpr (D <= -7) wait_vmcnt<behind(RT, 6)>();
        else if constexpr (D < 0) {
            wait_vmcnt<behind(RT, -1 - D) + (FOLLOWS ? SLOPE_LOADS + behind(3, D + 7) : 0)>();
        }
        if constexpr (D < 1) __builtin_amdgcn_s_barrier();
        if constexpr (FOLLOWS && D >= -7 && D < 0) {
            if constexpr (D == -7) {
                request_slope();
                set_sources(nxt);
            }
            load_unit(std::integral_constant<int, LT>{}, (D + 7) / 4, to);
        }
        constexpr int QA = JA < 0 ? 0 : JA == 0 ? QA0 : QA1, NQB = JB < 0 ? 0 : QB;
        constexpr int NM = QA * NQB * 2, NR = D >= 0 ? 0 : kReads[RT], NL = D < -7 ? kCnt[LT] : 0;
        // the stage read and the stage filled do not overlap (see gemm_transposed.hip on restrict)
        auto body = [&](const lds_char *__restrict stage) __attribute__((always_inline)) {
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (NM == 0) {
                for_constants<NL>([&](auto l) { load_one(std::integral_constant<int, LT>{}, decltype(l)::value, slab7, to); });
                for_constants<NR>([&](auto r) { read_one(std::integral_constant<int, RT>{}, r, stage); });
            } else {
                // reads in the first half of the MFMAs, so that the others cover their latency; loads spread over all (pinned order)
                constexpr int RPM = NM ? (2 * NR + NM - 1) / NM : 0;
                for_constants<NM>([&](auto m) {
                    constexpr int M = decltype(m)::value, KK = M / (QA * NQB), q = M % (QA * NQB), i = q / QA, j = q % QA;
                    constexpr int ai = JB * QB + i, aj = (JA == 0 ? 0 : QA0) + j;
                    const uint32_t scale = CB == 2 && JB == 1 ? sw >> 8 : sw;
                    if constexpr (JA == 0) acc[ai][aj] = mfma_scaled(fb[JB][i][KK], fa0[j][KK], acc[ai][aj], scale, sx[aj]);
                    else acc[ai][aj] = mfma_scaled(fb[JB][i][KK], fa1[j][KK], acc[ai][aj], scale, sx[aj]);
                    constexpr int R0 = min_int(NR, RPM * M), R1 = min_int(NR, RPM * (M + 1));
                    for_constants<R1 - R0>([&](auto r) { read_one(std::integral_constant<int, RT>{}, std::integral_constant<int, R0 + decltype(r)::value>{}, stage); });
                    constexpr int L0 = NL * M / NM, L1 = NL * (M + 1) / NM;
                    for_constants<L1 - L0>([&](auto l) { load_one(std::integral_constant<int, LT>{}, L0 + decltype(l)::value, slab7, to); });
                    __builtin_amdgcn_sched_barrier(0);
                });
            }
        };
        body(lds + from);
        // The products of the last slabs have no use before the end of the tile: without this the compiler moves all of them there
        if constexpr (JA >= 0 && D != -32) {
#pragma unroll
            for (int i = 0; i < QB; ++i)
#pragma unroll
                for (int j = 0; j < QA; ++j) {
                    f32x16 &c = acc[JB * QB + i][(JA == 0 ? 0 : QA0) + j];
                    if constexpr (OCC == 1) asm volatile("" : "+a"(c));
                    else asm volatile("" : "+v"(c));
                }
        }
    };
    auto take_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TM; ++j) sx[j] = sxn[j];
        sw = swn >> wshift;
    };
#define SMILE_IC(v) std::integral_constant<int, (v)>{}
    // The four phases 4 s + 2 .. 4 s + 5 of slab s, which lies in `stage`; D of the first of them, or -32.  Units f + 7 of the first
    // three are of slab s + 2 (same stage), of the last of slab s + 3.
    auto slab = [&](auto d, auto follow, int s, int stage) __attribute__((always_inline)) {
        constexpr int D = decltype(d)::value, N1 = D == -32 ? 0 : 1;
        phase(SMILE_IC(0), SMILE_IC(0), SMILE_IC(B1), SMILE_IC(D), follow, stage, s + 2, stage);
        phase(SMILE_IC(0), SMILE_IC(1), SMILE_IC(A1), SMILE_IC(D + N1), follow, stage, s + 2, stage);
        phase(SMILE_IC(1), SMILE_IC(0), SMILE_IC(A0), SMILE_IC(D + 2 * N1), follow, STAGE - stage, s + 2, stage);
        phase(SMILE_IC(1), SMILE_IC(1), SMILE_IC(B0), SMILE_IC(D + 3 * N1), follow, STAGE - stage, s + 3, STAGE - stage);
        take_scales();
    };
    const std::integral_constant<int, -1> none{};
    if (S >= 3) {
        const std::true_type follow{};
        phase(none, none, SMILE_IC(A0), SMILE_IC(-32), follow, stage0, 1, STAGE - stage0);
        phase(none, none, SMILE_IC(B0), SMILE_IC(-32), follow, stage0, 2, stage0);
        take_scales();
        int s = 0, stage = stage0;
        for (; s + 3 < S; ++s, stage = STAGE - stage) slab(SMILE_IC(-32), follow, s, stage);
        slab(SMILE_IC(-10), follow, s, stage);
        slab(SMILE_IC(-6), follow, s + 1, STAGE - stage);
        slab(SMILE_IC(-2), follow, s + 2, stage);
        stage0 = STAGE - stage;   // the next tile's slabs follow
    } else {
        // one or two slabs: nothing of the next tile is requested in between
        const std::false_type follow{};
        if (S == 2) {
            phase(none, none, SMILE_IC(A0), SMILE_IC(-8), follow, stage0, 1, STAGE - stage0);
            phase(none, none, SMILE_IC(B0), SMILE_IC(-7), follow, stage0, 0, stage0);
            take_scales();
            slab(SMILE_IC(-6), follow, 0, stage0);
            slab(SMILE_IC(-2), follow, 1, STAGE - stage0);
        } else {
            phase(none, none, SMILE_IC(A0), SMILE_IC(-4), follow, stage0, 0, 0);
            phase(none, none, SMILE_IC(B0), SMILE_IC(-3), follow, stage0, 0, 0);
            take_scales();
            slab(SMILE_IC(-2), follow, 0, stage0);
            stage0 = STAGE - stage0;
        }
        asm volatile("; one or two slabs" ::);   // no common code with the longer ones: their last products stay in front of the joint
    }
#undef SMILE_IC
    if (S < 3) request_slope();
    if (S < 3 && more) {   // its first units all at once; their slots were last read two phases and a barrier ago
        set_sources(nxt);
        load_first(4 * S, stage0);
    }

    // ---- epilogue.  Accumulator element v of a lane is (column 8*(v/4) + 4*(lane/32) + v%4, row lane%32) of its 32 x 32 block.
    const int e = cur.e, rows = cur.rows, Nout = a.Nout;
    const int olane = thread_id() & 63, orow = olane & 31, ohi = olane >> 5;
    lds_char *const stg = lds + 2 * STAGE + wave * 32 * SROW;
    auto row_at = [&](int j) { return (j < QA0 ? j * 64 : kExt[A0] + (j - QA0) * 64) + wm * 32; };            // first row of block j in the tile
    auto col_at = [&](int H) { return cur.ct * BN + H * kExt[B0] + wn * QB * 32; };                           // first column of part H
    auto activate_all = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            // Blocks without a row (128 groups x 20 rows, 768 -> 3072: 71 -> 59 us, 64 x 8, 1024 -> 4096 51 -> 45; full tiles: the same).  Neither ReLU nor
            // the search for the largest magnitude is worth it.
            if (ACT == 3 && cur.rt * BM + row_at(j) >= rows) break;
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = fp8_activate<ACT>(acc[i][j][v]);
        }
    };
    // y: rounded, staged as [32 rows][QB * 32 columns] of 16 bits (or half as many columns of fp32), stored row-contiguously
    auto store_y = [&]() __attribute__((always_inline)) {
        constexpr int P = QB * 4;   // 16-byte pieces of a staged row
        const auto blocks = [&](auto store) __attribute__((always_inline)) {   // store(j, H, first row, first column) of every live 32 x 32 QB block
            for_constants<TM>([&](auto j) {
                const int row0 = cur.rt * BM + row_at(decltype(j)::value);
                if (row0 >= rows) return;
                for_constants<2>([&](auto part) {
                    const int col0 = col_at(decltype(part)::value);
                    if (col0 < Nout) store(j, part, row0, col0);
                });
            });
        };
        const auto half_type = [&](auto type) __attribute__((always_inline)) {
            typedef Half<decltype(type)> HT;
            blocks([&](auto jj, auto part, int row0, int col0) __attribute__((always_inline)) {
                constexpr int j = decltype(jj)::value, H = decltype(part)::value;
#pragma unroll
                for (int i = 0; i < QB; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16 &c = acc[H * QB + i][j];
                        *(lds_u32x2 *)(stg + orow * SROW + (i * 32 + 8 * q + 4 * ohi) * 2) = u32x2{HT::pack(c[4 * q], c[4 * q + 1]), HT::pack(c[4 * q + 2], c[4 * q + 3])};
                    }
#pragma unroll
                for (int it = 0; it < P / 2; ++it) {
                    const int id = it * 64 + olane, lrow = id / P, row = row0 + lrow, col = col0 + (id - lrow * P) * 8;
                    const u32x4 v = *(const lds_u32x4 *)(stg + lrow * SROW + (id - lrow * P) * 16);
                    if (row < rows && col < Nout)
                        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.y) + ((size_t)e * a.C + row) * Nout + col) = v;
                }
            });
        };
        if (a.dtype == SMILE_DTYPE_BF16) {
            half_type(__bf16());
        } else if (a.dtype == SMILE_DTYPE_F16) {
            half_type(_Float16());
        } else {
            blocks([&](auto jj, auto part, int row0, int col0) __attribute__((always_inline)) {
                constexpr int j = decltype(jj)::value, H = decltype(part)::value;
                for_constants<2>([&](auto half) {
                    constexpr int F = decltype(half)::value;
#pragma unroll
                    for (int k = 0; k < 2 * QB; ++k) {
                        const int i = QB == 2 ? F : 0, q = QB == 2 ? k : 2 * F + k;
                        const f32x16 &c = acc[H * QB + i][j];
                        *(lds_u32x4 *)(stg + orow * SROW + (8 * k + 4 * ohi) * 4) =
                            u32x4{__float_as_uint(c[4 * q]), __float_as_uint(c[4 * q + 1]), __float_as_uint(c[4 * q + 2]), __float_as_uint(c[4 * q + 3])};
                    }
#pragma unroll
                    for (int it = 0; it < P / 2; ++it) {
                        const int id = it * 64 + olane, lrow = id / P, row = row0 + lrow, col = col0 + F * 16 * QB + (id - lrow * P) * 4;
                        const u32x4 v = *(const lds_u32x4 *)(stg + lrow * SROW + (id - lrow * P) * 16);
                        if (row < rows && col < Nout)
                            *reinterpret_cast<u32x4 *>(static_cast<float *>(a.y) + ((size_t)e * a.C + row) * Nout + col) = v;
                    }
                });
            });
        }
    };
    // Bias by scalar loads, which nothing else of the tile waits for: eight columns' words, of which a lane takes its half
    if (KIND != kFp8Slope && a.bias) {
        const auto add_bias = [&](auto words, auto value) __attribute__((always_inline)) {   // words: of eight columns; value(words of four, k)
            constexpr int W = decltype(words)::value;
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int col = min(col_at(i / QB) + i % QB * 32 + 8 * q, Nout - 8);
                    const auto *p = (const __attribute__((address_space(4))) uint32_t *)a.bias + ((size_t)e * Nout + col) / 8 * W;
                    uint32_t w[W / 2];
#pragma unroll
                    for (int k = 0; k < W / 2; ++k) {   // (through readfirstlane: a choice of addresses would be a vector load)
                        const uint32_t even = __builtin_amdgcn_readfirstlane(p[k]), odd = __builtin_amdgcn_readfirstlane(p[W / 2 + k]);
                        w[k] = ohi ? odd : even;
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float b = value(w, k);
#pragma unroll
                        for (int j = 0; j < TM; ++j) acc[i][j][4 * q + k] += b;
                    }
                }
        };
        if (a.dtype == SMILE_DTYPE_F32) add_bias(std::integral_constant<int, 8>{}, [](const uint32_t *w, int k) { return __uint_as_float(w[k]); });
        else if (a.dtype == SMILE_DTYPE_BF16) add_bias(std::integral_constant<int, 4>{}, [](const uint32_t *w, int k) { return k % 2 ? Half<__bf16>::hi(w[k / 2]) : Half<__bf16>::lo(w[k / 2]); });
        else add_bias(std::integral_constant<int, 4>{}, [](const uint32_t *w, int k) { return k % 2 ? Half<_Float16>::hi(w[k / 2]) : Half<_Float16>::lo(w[k / 2]); });
    }
    if constexpr (KIND == kFp8Y) {
        activate_all();
        store_y();
    } else {
        constexpr int SROW8 = QB * 32 + 16;
        const int NB = (Nout + kFp8Block - 1) / kFp8Block, ypitch = NB * kFp8Block;
        if (cur.ct * BN + BN > Nout) {         // columns beyond the matrix are zero codes
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (col_at(i / QB) + i % QB * 32 + 8 * (v / 4) + 4 * ohi + v % 4 >= Nout) {
#pragma unroll
                        for (int j = 0; j < TM; ++j) acc[i][j][v] = 0.f;
                    }
        }
        // The tile as 8-bit rows: each wave's largest magnitudes meet those of the wave that has the rest of the block's columns
        auto store_rows8 = [&](uint8_t *codes, uint8_t *scales, lds_char *largest) __attribute__((always_inline)) {
            uint32_t mine[TM][CB];   // magnitude_key's
            bool infinite = false;
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int b = 0; b < CB; ++b) {
                    float m = 0.f;
#pragma unroll
                    for (int i = CB == 2 ? b * QB : 0; i < (CB == 2 ? b * QB + QB : TN); ++i)
#pragma unroll
                        for (int v = 0; v < 16; v += 2) m = max_magnitude(m, acc[i][j][v], acc[i][j][v + 1]);
                    mine[j][b] = magnitude_key(m);
                    infinite |= __float_as_uint(m) >= 0x7f800000u;
                }
            if (__any(infinite)) {   // infinities do not count
#pragma unroll
                for (int j = 0; j < TM; ++j)
#pragma unroll
                    for (int b = 0; b < CB; ++b) {
                        uint32_t m = 0;
#pragma unroll
                        for (int i = CB == 2 ? b * QB : 0; i < (CB == 2 ? b * QB + QB : TN); ++i)
#pragma unroll
                            for (int v = 0; v < 16; ++v) m = max(m, magnitude_key(acc[i][j][v]));
                        mine[j][b] = m;
                    }
            }
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int b = 0; b < CB; ++b) {
                    mine[j][b] = max(mine[j][b], (uint32_t)__shfl_xor((int)mine[j][b], 32, 64));
                    if (ohi == 0) *(lds_u32 *)(largest + ((wn * CB + b) * BM + row_at(j) + orow) * 4) = mine[j][b];
                }
            __builtin_amdgcn_s_waitcnt(0xC07F);
            __builtin_amdgcn_s_barrier();
            for_constants<TM>([&](auto jj) {
                constexpr int j = decltype(jj)::value;
                const int row0 = cur.rt * BM + row_at(j);
                if (row0 >= rows) return;
                uint32_t byte[CB];
#pragma unroll
                for (int b = 0; b < CB; ++b)
                    byte[b] = scale_byte(magnitude_of(max(mine[j][b], *(const lds_u32 *)(largest + (((1 - wn) * CB + b) * BM + row_at(j) + orow) * 4))));
                for_constants<2>([&](auto part) {
                    constexpr int H = decltype(part)::value, b = CB == 2 ? H : 0;
                    const int col0 = col_at(H), block = cur.ct * CB + b;
                    if (block >= NB) return;
                    const float r = scale_value(byte[b]);
#pragma unroll
                    for (int i = 0; i < QB; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f32x16 &c = acc[H * QB + i][j];
                            *(lds_u32 *)(stg + orow * SROW8 + i * 32 + 8 * q + 4 * ohi) = pack4(c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3], r);
                        }
#pragma unroll
                    for (int it = 0; it < P8 / 2; ++it) {
                        const int id = it * 64 + olane, lrow = id / P8, row = row0 + lrow, at = (id - lrow * P8) * 16;
                        const u32x4 v = *(const lds_u32x4 *)(stg + lrow * SROW8 + at);
                        if (row < rows) *reinterpret_cast<u32x4 *>(codes + ((size_t)e * a.C + row) * ypitch + col0 + at) = v;
                    }
                    if (wn == 0 && ohi == 0 && (CB == 2 || H == 0) && row0 + orow < rows)
                        scales[((size_t)e * NB + block) * a.Cs + row0 + orow] = (uint8_t)byte[b];
                });
            });
        };
        lds_char *const largest = lds + 2 * STAGE + STAGING;
        if (KIND == kFp8Rows && a.p8) store_rows8(a.p8, a.ps, largest);
        // times the activation's derivative at the kept rows, which take the way through LDS that 8-bit rows take out
        const auto times_slope = [&](auto act) __attribute__((always_inline)) {
            for_constants<TM>([&](auto jj) {
                constexpr int j = decltype(jj)::value;
                if (cur.rt * BM + row_at(j) >= rows) return;
                for_constants<2>([&](auto part) {
                    constexpr int H = decltype(part)::value, b = CB == 2 ? H : 0;
                    if (cur.ct * CB + b >= NB) return;
#pragma unroll
                    for (int it = 0; it < P8 / 2; ++it) {
                        const int id = it * 64 + olane, lrow = id / P8;
                        *(lds_u32x4 *)(stg + lrow * SROW8 + (id - lrow * P8) * 16) = slope[j * 2 + H][it];
                    }
                    const float s = scale_value(slope_scale[j * CB + b]);
#pragma unroll
                    for (int i = 0; i < QB; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float g[4];
                            unpack4(*(const lds_u32 *)(stg + orow * SROW8 + i * 32 + 8 * q + 4 * ohi), s, g);
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[H * QB + i][j][4 * q + k] *= fp8_slope<decltype(act)::value>(g[k]);
                        }
                });
            });
        };
        if constexpr (KIND == kFp8Slope) {
            times_slope(std::integral_constant<int, ACT>{});
        } else {
            activate_all();
        }
        if (a.y8) store_rows8(a.y8, a.ys, largest + LARGEST);
        if (a.y) store_y();
    }
    if (!more) break;
    cur = nxt;
    }   // tile loop
    wait_vmcnt<0>();   // what was requested once more must not land in the LDS of another workgroup
#endif
}

template <int QB, int OCC, int KIND, int ACT>
hipError_t launch_fp8_ring(Fp8Gemm a, const Tuning &tune, hipStream_t s)
{
    constexpr int BM = 128, BN = 128 * QB;
    a.col_tiles = (a.Nout + BN - 1) / BN;
    const long long tiles = (long long)a.N * ((a.C + BM - 1) / BM) * a.col_tiles;
    const int slots = workgroup_slots(tune, OCC);
    const int grid = tiles < slots ? (int)((tiles + 7) / 8 * 8) : slots;
    SMILE_LAUNCH((fp8_gemm_ring_kernel<1, 1, QB, QB, OCC, KIND, ACT>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

}  // namespace smile
