// The 16-bit products of linear_half.hpp: their variants and the choice of a tile.
#include <algorithm>
#include <cmath>

#include "linear_half.hpp"
#include "linear_internal.hpp"

namespace smile {

namespace {

template <typename E, int WM, int WN, int QA>
hipError_t launch_shape(const LinearGemm &g, LinearKind kind, const Tuning &tune, hipStream_t s)
{
    if (kind == kLinearWeightGrad) return launch_half<E, WM, WN, QA, true, true, 0>(g, tune, s);
    if (kind == kLinearRowGrad) return launch_half<E, WM, WN, QA, false, true, 0>(g, tune, s);
    if (g.act == 0) return launch_half<E, WM, WN, QA, false, false, 0>(g, tune, s);
    if (g.act == 1) return launch_half<E, WM, WN, QA, false, false, 1>(g, tune, s);
    return launch_half<E, WM, WN, QA, false, false, 2>(g, tune, s);
}

template <typename E>
hipError_t launch_typed(const LinearGemm &g, LinearKind kind, HalfTile tile, const Tuning &tune, hipStream_t s)
{
    if (tile == kHalf256) return launch_shape<E, 2, 4, 2>(g, kind, tune, s);
    return launch_shape<E, 2, 2, 1>(g, kind, tune, s);
}

}  // namespace

// 256 x 256 outputs alone on a CU move half of the bytes from L2 that 128 x 128 do, but the epilogue waits for nobody and nobody multiplies meanwhile, and there
// are a quarter as many tiles to spread.  Time of `tiles` tiles of `slabs` slabs, us: rounds of the chip, each slabs x time of a slab (shorter while CUs are idle) + what a
// tile costs beside it; from two rounds on workgroups are out of step and share the last one.  Measured, bfloat16, 256 and 128 (in brackets the model):
//   forward, 16384 rows 1024 -> 4096: 125 / 156 (124 / 159), with GELU 146 / 170 (145 / 175); 256 -> 4096: 57 / 64 (52 / 63), 75 / 83 (73 / 79)
//   64 groups of 512 rows, 1024 -> 4096: 363 / 431 (303 / 351), GELU 376 / 421 (355 / 387), 512 -> 1024 GELU: 70 / 59 (68 / 68); 16 groups, 768 -> 2304: 45 / 46 (53 / 47)
//   gradient of x, 4096 rows, 4096 terms, 4096 columns: 108 / 130 (107 / 136), 1024 columns of 2048 rows: 69 / 44 (72 / 46)
//   gradient of the weights, 16384 x 4096 of 1024 rows: 124 / 146 (123 / 153); 2048 x 1024 of 4096 rows: 70 / 43 (72 / 46)
double linear_half_time(HalfTile tile, LinearKind kind, double tiles, double slabs, bool gelu)
{
    auto shared = [](double n) { return n <= 2.0 ? std::ceil(n) : std::min(std::ceil(n), n + 0.25); };
    const double n = tiles / (tile == kHalf256 ? kLinearCus : 2 * kLinearCus), full = std::min(n, 1.0);
    if (tile == kHalf256) {
        const double beside = kind == kLinearWeightGrad ? 5.4 : kind == kLinearRowGrad ? 5.5 : gelu ? 11.0 : 5.8;
        return 5.0 + shared(n) * ((0.92 + 0.58 * full * full) * slabs + beside);
    }
    const double beside = kind == kLinearWeightGrad ? 2.5 : kind == kLinearRowGrad ? 2.5 : gelu ? 5.2 : 3.2;
    // (up to half of the slots: one workgroup on a CU)
    return 5.0 + shared(n) * ((n <= 0.5 ? 0.59 + 0.41 * n * n : 1.0) * slabs + (n <= 1.0 ? 0.5 : 1.0) * beside);
}

// Groups of unknown rows are taken as even, with half a tile more each
HalfTile forward_half_tile(const LinearGemm &g)
{
    auto time = [&](HalfTile tile) {
        const int size = tile == kHalf256 ? 256 : 128;
        const double cols = (g.Nout + size - 1) / size, per = (double)g.rows / g.N;
        const double tiles = g.N == 1 ? std::ceil(per / size) : std::min((double)g.rows, g.N * std::max(1.0, per / size + 0.5));
        return linear_half_time(tile, kLinearForward, tiles * cols, (g.K + 63) / 64, g.act == 2);
    };
    return time(kHalf256) <= time(kHalf128) ? kHalf256 : kHalf128;
}

hipError_t launch_linear_half(int dtype, const LinearGemm &g, LinearKind kind, HalfTile tile, const Tuning &tune, hipStream_t s)
{
    if (dtype == SMILE_DTYPE_BF16) return launch_typed<__bf16>(g, kind, tile, tune, s);
    return launch_typed<_Float16>(g, kind, tile, tune, s);
}

}  // namespace smile
