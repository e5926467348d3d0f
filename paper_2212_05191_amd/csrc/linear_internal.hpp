// The products of smile_linear and of its gradients, as their launchers take them.
#pragma once

#include "smile_internal.hpp"

namespace smile {

// One product, y(i, j) = sum_k X(i, k) W(j, k) per group e.
//   rows (forward, gradient of x): X is the group's rows of x [rows][ldx], W = w[e] [Nout][K], or [K][Nout] where the kernel takes it transposed
//   weights' gradient: X(i, r) = x[r][i], W(j, r) = w[r][j], summed over the group's rows r; y[e] is [Mrows][Nout]
struct LinearGemm {
    const void *x, *w;
    const void *bias, *residual;   // [N][Nout], [rows][Nout]
    void *y, *pre;
    const int32_t *start;          // [N+1] or null: one group of all rows
    float *partial;                // gradients whose sums are cut into parts: of the weights [parts][Mrows][Nout], of the rows [parts][rows][Nout]; else null
    int N, rows;
    int Mrows, Nout, K;
    int ldx, ldw;                  // elements
    long long sw, sy;              // elements of a group in w; of a group of dw, or of a part
    int row_tiles, col_tiles;      // (row_tiles: weights' gradient)
    int chunk, parts;              // terms of a part of the sum (0: whole sums), and the parts: of all groups (weights' gradient), of a row (rows' gradient)
    int act;                       // 0 none, 1 ReLU, 2 GELU
};

enum LinearKind { kLinearForward, kLinearRowGrad, kLinearWeightGrad };
// Tiles of the 16-bit kernel: 256 x 256 alone on a CU, 128 x 128 two on a CU
enum HalfTile { kHalf256, kHalf128 };
// what the choice of a tile and the cuts of the gradients' sums go by: their workspace is asked for on the host alone
constexpr int kLinearCus = 256;
HalfTile forward_half_tile(const LinearGemm &g);
double linear_half_time(HalfTile tile, LinearKind kind, double tiles, double slabs, bool gelu);   // estimated, us
hipError_t launch_linear_half(int dtype, const LinearGemm &g, LinearKind kind, HalfTile tile, const Tuning &tune, hipStream_t s);

// The forward product of few rows (linear_few.hip), and whether it is the faster one
hipError_t launch_linear_few(int dtype, const LinearGemm &g, const Tuning &tune, hipStream_t s);
bool linear_few_applies(const LinearGemm &g);

}  // namespace smile
