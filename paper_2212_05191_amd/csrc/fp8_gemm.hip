// Grouped product of 8-bit rows with 8-bit weights:  p[e][r][o] = sum_k x[e][r][k] w[e][o][k] + bias, with the activation, its derivative at a
// kept pre-activation, and 8-bit outputs in the epilogue.
//
// Two kernels.  fp8_gemm_ring.hpp has the one for many rows.  fp8_gemm_rows_kernel, for few rows a group: what counts is the weights' way from HBM and the latency of a tile, so a tile is 32 rows x 32 WN
// columns, the contraction is split over WK waves, and every wave reads both operands straight into the registers of its matrix
// instructions, four blocks of 128 ahead: a lane holds row (or column) lane % 32 and the half lane / 32 of its 128 bytes.  The order of
// the k inside a block does not matter as long as both operands have the same.  The waves' sums meet in LDS in a fixed order, and the
// epilogue works on runs of eight columns, sixteen lanes to a block of the 8-bit outputs.
#include "fp8_gemm_ring.hpp"

namespace smile {

namespace {

// Eight neighbouring elements in the storage type `dtype`, which is the same for the whole launch
__device__ __forceinline__ void load8(int dtype, const void *base, size_t at, float *v)
{
    if (dtype == SMILE_DTYPE_BF16) Piece<SMILE_DTYPE_BF16>::widen(Piece<SMILE_DTYPE_BF16>::load(base, at), v);
    else if (dtype == SMILE_DTYPE_F16) Piece<SMILE_DTYPE_F16>::widen(Piece<SMILE_DTYPE_F16>::load(base, at), v);
    else Piece<SMILE_DTYPE_F32>::widen(Piece<SMILE_DTYPE_F32>::load(base, at), v);
}
__device__ __forceinline__ void store8(int dtype, void *base, size_t at, const float *v)
{
    if (dtype == SMILE_DTYPE_BF16) Piece<SMILE_DTYPE_BF16>::store(base, at, Piece<SMILE_DTYPE_BF16>::narrow(v));
    else if (dtype == SMILE_DTYPE_F16) Piece<SMILE_DTYPE_F16>::store(base, at, Piece<SMILE_DTYPE_F16>::narrow(v));
    else Piece<SMILE_DTYPE_F32>::store(base, at, Piece<SMILE_DTYPE_F32>::narrow(v));
}
__device__ __forceinline__ void activate8(int act, float *v)
{
    if (act == 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = fp8_activate<1>(v[k]);
    } else if (act == 3) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = fp8_activate<3>(v[k]);
    }
}

// The epilogue of eight columns col .. col + 7 of row r of group e; ROWS8: sixteen lanes of a DPP row hold a whole block of 128 columns.
// Columns beyond Nout are zero codes and no elements.
template <bool ROWS8>
__device__ __forceinline__ void finish8(const Fp8Gemm &a, int e, int r, int col, float *v)
{
    const size_t row = (size_t)e * a.C + r;
    const int NB = (a.Nout + kFp8Block - 1) / kFp8Block;
    const size_t code = row * ((size_t)NB * kFp8Block) + col, scale = ((size_t)e * NB + col / kFp8Block) * a.Cs + r;
    const bool in = col < a.Nout;
    if (!in) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.f;
    } else if (a.bias) {
        float b[8];
        load8(a.dtype, a.bias, (size_t)e * a.Nout + col, b);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += b[k];
    }
    if constexpr (ROWS8) {
        if (a.p8) {
            u32x2 c;
            const uint32_t byte = pack_block(v, c);
            *reinterpret_cast<u32x2 *>(a.p8 + code) = c;
            if (col % kFp8Block == 0) a.ps[scale] = (uint8_t)byte;
        }
        if (a.g8) {
            const u32x2 c = *reinterpret_cast<const u32x2 *>(a.g8 + code);
            const float s = scale_value(a.gs[scale]);
            float g[8];
            unpack4(c[0], s, g);
            unpack4(c[1], s, g + 4);
            if (a.act == 1) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= fp8_slope<1>(g[k]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= fp8_slope<3>(g[k]);
            }
        } else {
            activate8(a.act, v);
        }
        if (a.y8) {
            u32x2 c;
            const uint32_t byte = pack_block(v, c);
            *reinterpret_cast<u32x2 *>(a.y8 + code) = c;
            if (col % kFp8Block == 0) a.ys[scale] = (uint8_t)byte;
        }
    } else {
        activate8(a.act, v);
    }
    if (a.y && in) store8(a.dtype, a.y, row * a.Nout + col, v);
}

// WN waves side by side, 32 columns each; WK waves share the contraction
template <int WN, int WK, bool ROWS8>
__global__ __launch_bounds__(64 * WN * WK) void fp8_gemm_rows_kernel(Fp8Gemm a)
{
    constexpr int BN = 32 * WN, PITCH = BN + 4, THREADS = 64 * WN * WK, AHEAD = 4;
    static_assert(!ROWS8 || BN == kFp8Block, "a tile is one block of the 8-bit outputs");
    __shared__ __attribute__((aligned(16))) float sums[WK * 32 * PITCH];
    int tile = blockIdx.x;
    const int rt = tile % a.row_tiles;
    tile /= a.row_tiles;
    const int ct = tile % a.col_tiles, e = tile / a.col_tiles;
    const int valid = rows_of(a.rows, e, a.C);
    if (rt * 32 >= valid) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wn = wave % WN, wk = wave / WN;
    const int half = lane >> 5, K = a.KB * kFp8Block;
    const int row = min(rt * 32 + (lane & 31), valid - 1), col = min(ct * BN + wn * 32 + (lane & 31), a.Nout - 1);   // beyond: the last one again
    const uint8_t *x = a.x + ((size_t)e * a.C + row) * K + half * 64, *w = a.w + ((size_t)e * a.Nout + col) * K + half * 64;
    const uint8_t *xs = a.xs + (size_t)e * a.KB * a.Cs + row, *ws = a.ws + (size_t)e * a.KB * a.Ws + col / kFp8Block;
    struct Block {
        u32x4 x[4], w[4];
        uint8_t xs, ws;
    } block[AHEAD];
    const auto request = [&](Block &b, int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) b.w[i] = *reinterpret_cast<const u32x4 *>(w + (size_t)kb * kFp8Block + 16 * i);
#pragma unroll
        for (int i = 0; i < 4; ++i) b.x[i] = *reinterpret_cast<const u32x4 *>(x + (size_t)kb * kFp8Block + 16 * i);
        b.ws = ws[(size_t)kb * a.Ws], b.xs = xs[(size_t)kb * a.Cs];
    };
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
    const int kb0 = a.KB * wk / WK, kb1 = a.KB * (wk + 1) / WK;
    for_constants<AHEAD>([&](auto i) {
        if (kb0 + decltype(i)::value < kb1) request(block[decltype(i)::value], kb0 + decltype(i)::value);
    });
    for (int kb = kb0; kb < kb1; kb += AHEAD) {
        for_constants<AHEAD>([&](auto i) {
            constexpr int I = decltype(i)::value;
            if (kb + I >= kb1) return;
            Block &b = block[I];
            acc = mfma_scaled(set_high(set_low(b.w[0]), b.w[1]), set_high(set_low(b.x[0]), b.x[1]), acc, b.ws, b.xs);
            acc = mfma_scaled(set_high(set_low(b.w[2]), b.w[3]), set_high(set_low(b.x[2]), b.x[3]), acc, b.ws, b.xs);
            if (kb + I + AHEAD < kb1) request(b, kb + I + AHEAD);
        });
    }
    // element v of a lane: column 8 (v / 4) + 4 half + v % 4 of row lane % 32
    float *mine = sums + (wk * 32 + (lane & 31)) * PITCH + wn * 32 + 4 * half;
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4 *>(mine + 8 * q) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    for (int p = threadIdx.x; p < 32 * BN / 8; p += THREADS) {
        const int lr = p / (BN / 8), lc = p % (BN / 8) * 8, r = rt * 32 + lr, c = ct * BN + lc;
        if (r >= valid || (!ROWS8 && c >= a.Nout)) continue;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WK; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += sums[(k * 32 + lr) * PITCH + lc + j];
        finish8<ROWS8>(a, e, r, c, v);
    }
}

template <int WN, int WK, bool ROWS8>
hipError_t launch_rows(Fp8Gemm a, hipStream_t s)
{
    a.row_tiles = (a.C + 31) / 32;
    a.col_tiles = (a.Nout + 32 * WN - 1) / (32 * WN);
    const long long tiles = (long long)a.N * a.row_tiles * a.col_tiles;   // (few, by the rule below)
    SMILE_LAUNCH((fp8_gemm_rows_kernel<WN, WK, ROWS8>), dim3((unsigned)tiles), dim3(64 * WN * WK), 0, s, a);
    return hipGetLastError();
}

template <int KIND>
hipError_t launch_act(const Fp8Gemm &g, const Tuning &tune, hipStream_t s)
{
    if (g.act == 1) return launch_fp8_ring<1, 2, KIND, 1>(g, tune, s);
    if (g.act == 3) return launch_fp8_ring<1, 2, KIND, 3>(g, tune, s);
    return launch_fp8_ring<1, 2, KIND, 0>(g, tune, s);
}

}  // namespace

// Which kernel and tile.  us of a kernel, 32-row tiles first:
//   * y alone: 32 x 32 tiles with the contraction split over four waves while they are at most two a CU.  1 group x 16 rows, 1024 -> 4096 (128 tiles) 4.8 and
//     7.6, 128 rows (512) 7.1 and 8.1; 4096 -> 1024 9.5 and 15.8; 16 x 16, 3072 -> 768 (384) 12.8 and 13.0; beyond, 16 x 48 (768) 20.5 and
//     13.0, 16 x 1, 768 -> 3072 (1536) 11.9 and 9.8, 8 x 128, 256 -> 1024 (1024) 6.5 and 5.5.
//   * 8-bit rows, whose 128 columns a workgroup of eight waves needs: contractions of four blocks or less and at most one tile a CU.  4 x 16,
//     512 -> 1024 6.8 and 7.6, 8 x 128, 256 -> 1024 6.0 and 7.7; but 1 x 16, 1024 -> 4096 9.8 and 9.0, 16 x 1, 768 -> 3072 13.0 and 11.8.
//   * else 128 x 128, two on a CU; 128 x 256, which moves a quarter less through L2, for long contractions without an epilogue that the other workgroup
//     would hide, where there are four rounds of such tiles: 8192 x 8192 x 8192 498 -> 462, 128 groups x 256 rows, 3072 -> 768 119 -> 113; 64 x
//     256, 4096 -> 1024 (three rounds) 98 -> 104, 16384 x 1024 -> 4096 81 -> 92.
int pick_fp8_kernel(int cus, int N, int C, int KB, int Nout, bool rows8, int act)
{
    const auto tiles = [&](int rows, int columns) { return (long long)N * ((C + rows - 1) / rows) * ((Nout + columns - 1) / columns); };
    if (rows8) return KB <= 4 && tiles(32, 128) <= cus ? kFp8FewRowsCodes : kFp8Ring128;
    if (tiles(32, 32) <= 2 * cus) return kFp8FewRowsY;
    return act == 0 && KB >= 16 && tiles(128, 256) >= 4 * cus ? kFp8Ring256 : kFp8Ring128;
}

hipError_t launch_fp8_gemm(const Fp8Gemm &g, const Tuning &tune, hipStream_t s)
{
    const bool rows8 = g.y8 || g.p8 || g.g8;
    switch (pick_fp8_kernel(tune.cus, g.N, g.C, g.KB, g.Nout, rows8, g.act)) {
    case kFp8FewRowsY: return launch_rows<1, 4, false>(g, s);
    case kFp8FewRowsCodes: return launch_rows<4, 2, true>(g, s);
    case kFp8Ring256: return launch_fp8_ring<2, 1, kFp8Y, 0>(g, tune, s);
    default: break;
    }
    if (g.g8) return g.act == 1 ? launch_fp8_ring<1, 2, kFp8Slope, 1>(g, tune, s) : launch_fp8_ring<1, 2, kFp8Slope, 3>(g, tune, s);
    return rows8 ? launch_act<kFp8Rows>(g, tune, s) : launch_act<kFp8Y>(g, tune, s);
}

}  // namespace smile
