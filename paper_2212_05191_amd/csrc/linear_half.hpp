// Products over sorted rows on the 16-bit matrix instructions (v_mfma_f32_32x32x16): rows (forward, gradient of x) and the weights' gradient.
//
// A workgroup of WM x WN waves computes BM x BN outputs at a time, a wave (64 QA) x 64 of them, and walks the tiles of the launch.  A slab (64 terms) is four
// units: the rows of X of the first and of the second half of every wave's blocks (A0, A1), and the same of W (B0, B1).  It is multiplied in two phases: A0 with B0
// and B1, then A1; a phase reads what it does not hold yet from LDS, then multiplies.  LDS holds two slabs; a unit's slot is refilled one phase after its reading, two
// slabs ahead, so that four to five of the eight units are in flight at any time.  Four phases of one product each, twice the barriers, were slower (8192^3 1017 against
// 971 us when both were tried); so was reading between the products of the phase before, with the fragments of two phases in registers (128 x 128 tiles, 4096 rows 1024
// -> 1024: 19.0 against 17.5 us).  The stream of slabs runs on through the tiles: the epilogue finds the next tile's first two slabs requested.  Behind the last tile the
// last slab is requested again, so that every wait counts the same.
//
// What bounds it: the matrix cores, if what they are fed with keeps up.  A wave that reads its fragments (up to 16 of 16 bytes a lane) cannot multiply, so two waves
// of a SIMD take turns (STAGGER): the waves are two halves, one a barrier behind the other; while one multiplies the other reads and requests.  With
// four waves (128 x 128 tiles, two workgroups on a CU) the workgroups do so by themselves, at one barrier a phase.  On a full chip a slab of 256 x 256 takes 1.5 us (1430
// TFLOP/s between epilogues), of 128 x 128 two on a CU 1.0 (1070); an epilogue about 5.5 and 3 us, 11 and 5 with GELU.  8192^3: 783 us (1404 TFLOP/s).
//
// Operand units in LDS.  Normal: [row][64 k], piece c (16 bytes) of a row at c ^ ((row >> 1) & 7).  Transposed: as in memory, [64 k][columns], fragments by
// transposing reads; pieces rotated by 4 (k & 3) in rows of 16 pieces, by 4 ((k >> 1) & 1) in rows of 8, so that successive k-rows fall on distinct banks.
// A wave's 64 columns are neighbours (32 of B0, 32 of B1): whole lines in the epilogue.  Terms beyond the sum's length are zero in both operands; rows and
// columns beyond a matrix repeat its last ones, whose outputs are not stored.
#pragma once

#include "linear_walk.hpp"

namespace smile {

namespace {

constexpr int kHalfBand = 8;

template <int WM, int WN, int QA>
constexpr int half_lds() { return 2 * (2 * 32 * QA * WM + 2 * 32 * WN) * 128 + WM * WN * 4096; }

// ACT: of the epilogue (rows); GRAD: the weights' gradient, both operands transposed; WT: w transposed
template <typename E, int WM, int WN, int QA, bool GRAD, bool WT, int ACT>
__global__ __launch_bounds__(WM *WN * 64, 2) void linear_half_kernel(LinearGemm a)
{
    typedef typename Half<E>::vec8 vec8;
    typedef __attribute__((__vector_size__(4 * sizeof(E)))) E vec4;
    static_assert(!GRAD || WT, "the weights' gradient takes both operands transposed");
    constexpr bool XT = GRAD, STAGGER = WM * WN == 8;
    constexpr int NW = WM * WN, UA = 32 * QA * WM, UB = 32 * WN, BM = 2 * UA, BN = 2 * UB, TM = 2 * QA;
    enum { A0, B0, B1, A1 };
    constexpr int kExt[4] = {UA, UB, UB, UA};
    constexpr int kOff[4] = {0, UA * 128, (UA + UB) * 128, (UA + 2 * UB) * 128};
    constexpr int STAGE = 2 * (UA + UB) * 128;
    static_assert(UA == UB && UA / (8 * NW) == 2, "two load instructions a wave and unit");
    constexpr int kAhead = 8;    // load instructions behind the units that the next phase reads: four units
    __shared__ __attribute__((aligned(16))) char half_lds_[half_lds<WM, WN, QA>()];
    lds_char *const lds = (lds_char *)half_lds_;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = wave % WN, wm = wave / WN;

    std::conditional_t<GRAD, GradWalk<BM>, RowWalk<BM, kHalfBand>> walk;
    walk.init(a);
    // the n-th tile of this workgroup or the first behind it; false: none
    auto tile_from = [&](int &n, LinearTile &t) {
        if constexpr (GRAD) {
            for (;; ++n) {
                const int found = walk.tile(a, n, BN, t);
                if (found != 0) return found > 0;
            }
        } else {
            return walk.tile(a, n, BN, t);
        }
    };

    // ---- loader: the slab whose units are being requested
    uint32_t off[8];             // this lane's byte offsets from xb / wb: two load instructions of A0, B0, B1, A1
    const char *xb = nullptr, *wb = nullptr;   // the slab's operands
    int l_n = 0, l_left = 0, l_last = 64, l_stage = 0;   // l_left: slabs of its tile from it on; l_last: terms of the last one
    bool l_done = false;
    const size_t adv_x = 2 * (XT ? (size_t)64 * a.ldx : 64), adv_w = 2 * (WT ? (size_t)64 * a.ldw : 64);
    auto thread_lane = [&]() {   // derived afresh, so that nothing computed from it stays in registers
        int l = threadIdx.x & 63;
        asm volatile("" : "+v"(l));
        return l;
    };
    // row (or k-row) and piece that a lane fetches in load instruction `inst` of a unit of U rows / columns
    auto place = [](auto transposed, int U, int l, int inst, int &r, int &piece) __attribute__((always_inline)) {
        if constexpr (!decltype(transposed)::value) {
            r = inst * 8 + (l >> 3);
            piece = (l & 7) ^ ((r >> 1) & 7);
        } else {
            const int P = U / 8, q = inst * 64 + l;
            r = q / P;
            const int rot = P == 16 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
            piece = (q - r * P - rot) & (P - 1);
        }
    };
    auto set_sources = [&](const LinearTile &t) __attribute__((always_inline)) {
        l_left = (t.kv + 63) / 64, l_last = t.kv - 64 * (l_left - 1);
        xb = static_cast<const char *>(a.x) + 2 * (GRAD ? (size_t)t.from * a.ldx : (size_t)t.first * a.ldx + t.from);
        wb = static_cast<const char *>(a.w) + 2 * ((GRAD ? 0 : (size_t)t.e * a.sw) + (WT ? (size_t)t.from * a.ldw : t.from));
        const int l = thread_lane();
        for_constants<4>([&](auto type) {
            constexpr int T = decltype(type)::value;
            constexpr bool IS_X = T == A0 || T == A1, TR = IS_X ? XT : WT;
            constexpr int H = T == A1 || T == B1 ? 1 : 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int r, piece;
                place(std::bool_constant<TR>{}, kExt[T], l, wave + i * NW, r, piece);
                const int at = TR ? piece * 8 : r;                                         // row or column inside the unit
                const int in_tile = IS_X ? H * UA + at : (at / 32) * 64 + H * 32 + at % 32;
                const uint32_t ld = IS_X ? a.ldx : a.ldw;
                if constexpr (TR) {
                    const int first = IS_X ? t.first : t.col0, ext = IS_X ? a.Mrows : a.Nout;
                    off[2 * T + i] = 2 * ((uint32_t)r * ld + min(first + in_tile, ext - 8));
                } else if constexpr (IS_X) {
                    off[2 * T + i] = 2 * ((uint32_t)min(in_tile, t.rows - 1) * ld + piece * 8);
                } else {
                    off[2 * T + i] = 2 * ((uint32_t)min(t.col0 + in_tile, a.Nout - 1) * ld + piece * 8);
                }
            }
        });
    };
    // WHOLE: the slab has 64 terms
    auto load_unit = [&](auto type, auto whole) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        constexpr bool IS_X = T == A0 || T == A1, TR = IS_X ? XT : WT;
        const char *base = IS_X ? xb : wb;
        asm volatile("" : "+s"(base));   // scalar base + 32-bit offset, not a 64-bit sum for each lane
        lds_char *const to = lds + l_stage + kOff[T] + wave * 1024;
        if (decltype(whole)::value || l_left > 1 || l_last == 64) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                __builtin_amdgcn_global_load_lds(SMILE_GPTR(base + off[2 * T + i]), SMILE_LPTR(to + i * NW * 1024), 16, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int r, piece;
                place(std::bool_constant<TR>{}, kExt[T], thread_lane(), wave + i * NW, r, piece);
                const char *p = (TR ? r : piece * 8) < l_last ? base + off[2 * T + i] : reinterpret_cast<const char *>(kZeroPiece);
                __builtin_amdgcn_global_load_lds(SMILE_GPTR(p), SMILE_LPTR(to + i * NW * 1024), 16, 0, 0);
            }
        }
    };
    // the next tile with terms, from number l_n on
    auto next_source = [&]() {
        LinearTile t;
        for (;; ++l_n) {
            if (!tile_from(l_n, t)) return false;
            if (!GRAD || t.kv > 0) break;
        }
        set_sources(t);
        return true;
    };
    auto advance = [&]() {
        l_stage ^= STAGE;
        if (l_done) return;
        if (--l_left > 0) {
            xb += adv_x, wb += adv_w;
            return;
        }
        ++l_n;
        if (!next_source()) l_done = true, l_left = 1;   // (the last slab again: addresses that exist)
    };
#define SMILE_IC(v) std::integral_constant<int, (v)>{}
    const bool any = next_source();
    const std::false_type maybe{};   // a slab that may have fewer than 64 terms
    if (any) {
        load_unit(SMILE_IC(A0), maybe), load_unit(SMILE_IC(B0), maybe), load_unit(SMILE_IC(B1), maybe), load_unit(SMILE_IC(A1), maybe);
        advance();
        load_unit(SMILE_IC(A0), maybe), load_unit(SMILE_IC(B0), maybe), load_unit(SMILE_IC(B1), maybe);
        wait_vmcnt<kAhead>();
        __builtin_amdgcn_s_barrier();
        if (STAGGER && wm == 1) __builtin_amdgcn_s_barrier();
    }

    // ---- fragments
    const int frow = lane & 31, fhi = lane >> 5;
    const int tj = (lane >> 2) & 3, tk0 = 8 * fhi + tj, tcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    vec8 fa[QA][4], fb0[4], fb1[4];
    f32x16 acc[2][TM];
    auto read_unit = [&](auto type, const lds_char *stage) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        constexpr bool IS_X = T == A0 || T == A1, TR = IS_X ? XT : WT;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int q = 0; q < (IS_X ? QA : 1); ++q) {
                const int first = IS_X ? wm * QA * 32 + q * 32 : wn * 32;
                vec8 v;
                if constexpr (!TR) {
                    v = *(const __attribute__((address_space(3))) vec8 *)(stage + kOff[T] + (first + frow) * 128 + (((2 * kk + fhi) ^ ((frow >> 1) & 7)) * 16));
                } else {
                    constexpr int P = kExt[T] / 8, PITCH = P * 16;
                    const int col = first + tcol, rot = P == 16 ? 4 * tj : 4 * ((tj >> 1) & 1);
                    read_transposed<4 * PITCH>(v, stage + kOff[T] + (tk0 + 16 * kk) * PITCH + (((col >> 3) + rot) & (P - 1)) * 16 + (col & 4) * 2);
                }
                if constexpr (IS_X) fa[q][kk] = v;
                else if constexpr (T == B0) fb0[kk] = v;
                else fb1[kk] = v;
            }
    };
    int c_stage = 0;
    bool upper = true;     // the tile has rows in A1
    // After an epilogue: `fresh` slabs have begun since (2: no longer counted), and `stores` of its store instructions, if their number is known, lie between the
    // loads that are waited for and those behind them.
    int fresh = 2, stores = 0;
    auto wait_next = [&]() __attribute__((always_inline)) {
        if (stores == 0) wait_vmcnt<kAhead>();
        else if (stores == 4 * TM) wait_vmcnt<kAhead + 4 * TM>();
        else wait_vmcnt<kAhead + 8 * TM>();
    };
    // Phase P of a slab.  `steady`: nothing of an epilogue is counted, and the slab requested is a whole one of the tile that was requested before: one branch for
    // all that may be otherwise, since branches cost more than what they save (128 x 128 tiles, gradient of the weights of 2048 rows 1024 -> 4096: 31.7 -> 24.2 us).
    auto phase = [&](auto number, bool steady) __attribute__((always_inline)) {
        constexpr int P = decltype(number)::value;
        // the stage read and the stage filled do not overlap
        auto fetch = [&](const lds_char *__restrict stage) __attribute__((always_inline)) {
            if constexpr (P == 0) {
                read_unit(SMILE_IC(A0), stage);
                read_unit(SMILE_IC(B0), stage), read_unit(SMILE_IC(B1), stage);
            } else {
                read_unit(SMILE_IC(A1), stage);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (__builtin_expect(steady, 1)) {
                if constexpr (P == 0) {
                    load_unit(SMILE_IC(A1), std::true_type{});
                } else {
                    xb += adv_x, wb += adv_w, l_stage ^= STAGE;
                    load_unit(SMILE_IC(A0), std::true_type{}), load_unit(SMILE_IC(B0), std::true_type{}), load_unit(SMILE_IC(B1), std::true_type{});
                }
                wait_vmcnt<kAhead>();
            } else if constexpr (P == 0) {
                if (fresh != 0) {   // (else requested, and waited for, in front of the epilogue)
                    load_unit(SMILE_IC(A1), maybe);
                    wait_next();
                }
            } else {
                advance();
                load_unit(SMILE_IC(A0), maybe), load_unit(SMILE_IC(B0), maybe), load_unit(SMILE_IC(B1), maybe);
                if (fresh > 0) stores = 0;
                wait_next();
            }
        };
        __builtin_amdgcn_sched_barrier(0);
        fetch(lds + c_stage);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): what was read here may be overwritten from the next phase on
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        if (P == 0 || __builtin_expect(upper, 1))   // nothing to multiply where the tile's rows all lie in A0
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int q = 0; q < QA; ++q) acc[i][P * QA + q] = Half<E>::mfma_32x32x16(i ? fb1[kk] : fb0[kk], fa[q][kk], acc[i][P * QA + q]);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (STAGGER && P == 0) {
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // The barrier behind a tile's last phase is what the later half owes until its epilogue is done: had it to meet the other half's next one in front of it, the two
    // epilogues would follow each other (16384 rows 1024 -> 4096 with GELU: 160 -> 150 us; 64 groups 417 -> 395, 4096 -> 1024 without 303 -> 293).
    bool owed = false;
    auto pay = [&]() __attribute__((always_inline)) {
        if (STAGGER && owed) __builtin_amdgcn_s_barrier();
        owed = false;
    };

    lds_char *const stg = lds + 2 * STAGE + wave * 4096;
    for (int n = 0;; ++n) {
        LinearTile t;
        if (!tile_from(n, t)) break;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
        upper = t.rows > UA;
        if (t.kv > 0) pay();
        int steady = 0;   // slabs to come that are
        for (int n_slabs = (t.kv + 63) / 64; n_slabs > 0; --n_slabs) {
            if (steady == 0 && fresh == 2 && !l_done) {   // (the slab requested in a slab's second phase is the one behind that of the first)
                steady = max(0, min(n_slabs, l_left - (l_last == 64 ? 1 : 2)));
                l_left -= steady;
            }
            const bool is_steady = steady > 0;
            phase(SMILE_IC(0), is_steady), phase(SMILE_IC(1), is_steady);
            if constexpr (STAGGER) {
                owed = n_slabs == 1 && wm == 1;
                if (!owed) __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
            }
            steady = max(steady - 1, 0);
            fresh = min(fresh + 1, 2);
            c_stage ^= STAGE;
        }
        // Loads and stores are counted in their order.  What the next slab reads is waited for here, and the slab behind it requested whole, before this tile's
        // stores queue up: with their number known, nothing waits for them until two slabs later.
        if (any) {
            wait_vmcnt<6>();
            if (fresh != 0) load_unit(SMILE_IC(A1), maybe);
        }
        fresh = 0, stores = 0;
        const bool full = t.rows >= BM && t.col0 + BN <= a.Nout;

        // ---- epilogue, private to a wave.  Accumulator element v of a lane is (column 8 (v / 4) + 4 (lane / 32) + v % 4, row lane % 32) of its 32 x 32 block:
        // rounded, staged as [32 rows][64 columns] in the wave's own 4 KB (piece p of a row at p ^ ((row >> 1) & 7)), stored in lines of 128 bytes.
        const int ol = thread_lane(), orow = ol & 31, ohi = ol >> 5, col0 = t.col0 + wn * 64;
        if (col0 >= a.Nout) continue;
        auto staged_at = [&](int row, int piece) { return stg + row * 128 + ((piece ^ ((row >> 1) & 7)) * 16); };
        if (WT && a.partial) {
            float *P = a.partial + (size_t)t.part * a.sy;
            for_constants<2 * TM>([&](auto block) {
                constexpr int i = decltype(block)::value % 2, j = decltype(block)::value / 2;
                const int row0 = (j / QA) * UA + wm * QA * 32 + (j % QA) * 32;
                if (row0 >= t.rows) return;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(__attribute__((address_space(3))) f32x4 *)(staged_at(orow, 2 * q + ohi)) =
                        f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                asm volatile("" ::: "memory");
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int lrow = it * 8 + (ol >> 3), p = ol & 7, row = row0 + lrow, col = col0 + i * 32 + p * 4;
                    const f32x4 v = *(const __attribute__((address_space(3))) f32x4 *)(staged_at(lrow, p));
                    if (row < t.rows && col < a.Nout) *reinterpret_cast<f32x4 *>(P + (size_t)(t.first + row) * a.Nout + col) = v;
                }
                asm volatile("" ::: "memory");
            });
            continue;   // (the stores are few beside the sum: not counted)
        }
        vec4 bias[2][4];
        if (!GRAD && a.bias) {
            const E *b = static_cast<const E *>(a.bias) + (size_t)t.e * a.Nout;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) bias[i][q] = *reinterpret_cast<const vec4 *>(b + min(col0 + i * 32 + 8 * q + 4 * ohi, a.Nout - 4));
            // here, so that the next tile's first reads need not wait for what a tile without rows left unused
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(bias[i][q]));
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) bias[i][q] = vec4{(E)0.f, (E)0.f, (E)0.f, (E)0.f};
        }
        E *const Y = static_cast<E *>(a.y) + (GRAD ? (size_t)t.e * a.sy : 0);
        for_constants<TM>([&](auto jj) {
            constexpr int j = decltype(jj)::value;
            const int row0 = (j / QA) * UA + wm * QA * 32 + (j % QA) * 32;
            if (row0 >= t.rows) return;
            auto each_piece = [&](auto f) __attribute__((always_inline)) {   // f(lrow, piece, element in y, valid)
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int lrow = it * 8 + (ol >> 3), p = ol & 7, row = row0 + lrow, col = col0 + p * 8;
                    f(it, lrow, p, (size_t)(t.first + row) * a.Nout + col, row < t.rows && col < a.Nout);
                }
            };
            // f(i, q, the four values) of every group of four neighbouring columns of this lane's row
            auto each_four = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f32x4 v;
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = WT ? acc[i][j][4 * q + k] : acc[i][j][4 * q + k] + (float)bias[i][q][k];
                        f(i, q, v, (__attribute__((address_space(3))) vec4 *)(staged_at(orow, i * 4 + q) + ohi * 8));
                    }
            };
            // past the L2, which the operands need more (64 groups of 512 rows, 1024 -> 4096: 342 -> 338 us, with GELU 460 -> 449)
            auto store_staged = [&](E *to) __attribute__((always_inline)) {
                asm volatile("" ::: "memory");
                u32x4 v[4];
                each_piece([&](int it, int lrow, int p, size_t, bool) __attribute__((always_inline)) {
                    v[it] = *(const __attribute__((address_space(3))) u32x4 *)(staged_at(lrow, p));
                });
                if (full) each_piece([&](int it, int, int, size_t at, bool) __attribute__((always_inline)) { __builtin_nontemporal_store(v[it], reinterpret_cast<u32x4 *>(to + at)); });
                else
                    each_piece([&](int it, int, int, size_t at, bool valid) __attribute__((always_inline)) {
                        if (valid) __builtin_nontemporal_store(v[it], reinterpret_cast<u32x4 *>(to + at));
                    });
                asm volatile("" ::: "memory");
            };
            u32x4 res[4];
            if (!GRAD && a.residual)
                each_piece([&](int it, int, int, size_t at, bool valid) __attribute__((always_inline)) {
                    res[it] = u32x4{0u, 0u, 0u, 0u};
                    if (valid) res[it] = *reinterpret_cast<const u32x4 *>(static_cast<const E *>(a.residual) + at);
                });
            if (!GRAD && a.pre) {
                each_four([&](int, int, f32x4 v, auto at) __attribute__((always_inline)) { *at = vec4{(E)v[0], (E)v[1], (E)v[2], (E)v[3]}; });
                store_staged(static_cast<E *>(a.pre));
            }
            if (!GRAD && a.residual) {
                each_piece([&](int it, int lrow, int p, size_t, bool) __attribute__((always_inline)) {
                    *(__attribute__((address_space(3))) u32x4 *)(staged_at(lrow, p)) = res[it];
                });
                asm volatile("" ::: "memory");
            }
            // one branch for all of a block, not one for each four values, which keeps their chains apart (16384 rows 1024 -> 4096 with GELU: 164 -> 157 us; 64 groups 424 -> 411)
            auto finish = [&](auto added) __attribute__((always_inline)) {
                each_four([&](int, int, f32x4 v, auto at) __attribute__((always_inline)) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = linear_act<false>(ACT, v[k]);
                    if constexpr (decltype(added)::value) {
                        const vec4 r = *at;
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] += (float)r[k];
                    }
                    *at = vec4{(E)v[0], (E)v[1], (E)v[2], (E)v[3]};
                });
            };
            if (!GRAD && a.residual) finish(std::true_type{});
            else finish(std::false_type{});
            store_staged(Y);
        });
        if (full) stores = TM * (!GRAD && a.pre ? 8 : 4);
    }
    pay();
    if (any) {
        wait_vmcnt<0>();   // nothing of this workgroup reaches its LDS any more
        if (STAGGER && wm == 0) __builtin_amdgcn_s_barrier();
    }
}

#undef SMILE_IC

template <typename E, int WM, int WN, int QA, bool GRAD, bool WT, int ACT>
hipError_t launch_half(LinearGemm g, const Tuning &tune, hipStream_t s)
{
    constexpr int BM = 64 * QA * WM, BN = 64 * WN, PER_CU = WM * WN == 8 ? 1 : 2;
    g.col_tiles = (g.Nout + BN - 1) / BN, g.row_tiles = (g.Mrows + BM - 1) / BM;
    const long long most = g.parts * (GRAD ? (long long)g.row_tiles : (g.rows + BM - 1) / BM + (long long)std::min(g.N, g.rows) - 1) * g.col_tiles;
    if (most >= 1ll << 31) return hipErrorInvalidValue;
    const int grid = (int)std::min((most + 7) / 8 * 8, (long long)workgroup_slots(tune, PER_CU));
    SMILE_LAUNCH((linear_half_kernel<E, WM, WN, QA, GRAD, WT, ACT>), dim3(grid), dim3(WM * WN * 64), 0, s, g);
    return hipGetLastError();
}

}  // namespace

}  // namespace smile
