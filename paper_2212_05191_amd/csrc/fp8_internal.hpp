// Launchers of the 8-bit operators.  Shapes were validated by the entry points (fp8_api.hip); 8-bit rows and weights are laid out as
// include/smile.h says.
#pragma once

#include "smile_internal.hpp"

namespace smile {

struct RmsNormIo {
    const void *x, *residual, *weight;
    void *sum, *y;
    uint8_t *y8, *y8_scale;
    float *rstd;
    int T, d;
    float eps;
};
hipError_t launch_rms_norm(int dtype, const RmsNormIo &io, hipStream_t s);

struct RmsNormGradIo {
    const void *dy, *dsum, *s, *weight;
    const float *rstd;
    void *ds;
    float *dweight, *partial;
    int T, d;
};
size_t rms_norm_backward_workspace(int T, int d);
hipError_t launch_rms_norm_backward(int dtype, const RmsNormGradIo &io, hipStream_t s);

// 8-bit rows [N][C][K] from or to `dtype`
struct RowsIo {
    int N, C, K;
    const int32_t *rows;
};
hipError_t launch_fp8_pack_rows(int dtype, const RowsIo &io, const void *src, uint8_t *codes, uint8_t *scales, hipStream_t s);
hipError_t launch_fp8_unpack_rows(int dtype, const RowsIo &io, const uint8_t *codes, const uint8_t *scales, void *dst, hipStream_t s);
hipError_t launch_fp8_pack_weights(int dtype, int N, int Nout, int K, const void *w, uint8_t *codes, uint8_t *scales, uint8_t *codes_t,
                                   uint8_t *scales_t, hipStream_t s);
hipError_t launch_fp8_dispatch(const smile_layer_desc &d, const uint8_t *x8, const uint8_t *x_scale, const int32_t *group_idx,
                               const int32_t *local_idx, const int32_t *slot, uint8_t *xe8, uint8_t *xe_scale, hipStream_t s);

// The argument block of the product's kernels
struct Fp8Gemm {
    const uint8_t *x, *xs, *w, *ws;
    const void *bias;
    const int32_t *rows;
    void *y;
    uint8_t *y8, *ys, *p8, *ps;      // result and pre-activation as 8-bit rows
    const uint8_t *g8, *gs;          // pre-activation whose derivative multiplies the result
    int N, C, Nout, KB;              // KB: blocks of 128 along the contraction
    int Cs, Ws;                      // bytes of a line of scales: rows, blocks of columns
    int dtype, act;                  // act: 0 none, 1 ReLU, 3 GELU
    int row_tiles, col_tiles;
};
enum Fp8Kernel { kFp8FewRowsY, kFp8FewRowsCodes, kFp8Ring128, kFp8Ring256 };   // 32 x 32 tiles, 32 x 128; 128 x 128, 128 x 256
int pick_fp8_kernel(int cus, int N, int C, int KB, int Nout, bool rows8, int act);   // rows8: 8-bit rows are written or read in the epilogue
hipError_t launch_fp8_gemm(const Fp8Gemm &g, const Tuning &tune, hipStream_t s);
hipError_t launch_fp8_near_zero(const Fp8Gemm &g, hipStream_t s);   // after a product with p8: its codes next to zero from exact sums

// Weight gradients from 8-bit rows without a widened copy
struct Fp8WeightGrad {
    const uint16_t *dy;              // [N][C][Nout] bfloat16
    const uint8_t *x, *xs;           // 8-bit rows [N][C][K]
    const int32_t *rows;
    uint16_t *dw;                    // [N][Nout][K]
    int N, C, Nout, K, KB, Cs;
    int o_tiles, k_tiles, tiles, chunk;
};
bool fp8_weight_grad_applies(int dtype, int N, int C, int Nout, int K, const Tuning &tune);
hipError_t launch_fp8_weight_grad(Fp8WeightGrad a, hipStream_t s);

}  // namespace smile
