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
// are a quarter as many tiles to spread.  Time of `tiles` tiles of `slabs` slabs, us: rounds of the chip, each slabs x time of a slab + what a tile costs beside it; from
// three rounds on workgroups are out of step and share the last one.  Its figures, and what they stand for (bfloat16; measured, 256 and 128, in brackets the model):
//   forward, 16384 rows 4096 -> 1024: 143 / 155 (135 / 147); 64 groups of 512 rows, 1024 -> 4096: 391 / 398 (399 / 407), with GELU 470 / 435 (497 / 461)
//   gradient of x, 16384 rows 4096 -> 1024: 171 / 200 (168 / 187); of the weights, 64 groups: 395 / 460 (380 / 441)
//   4096 rows 1024 -> 1024 (64 and 256 tiles): 30 / 19 (43 / 19); 16 groups of 512 rows 768 -> 2304 with GELU: 66 / 50 (85 / 67)
double linear_half_time(HalfTile tile, double tiles, double slabs, bool gelu)
{
    auto shared = [](double n) { return n <= 3.0 ? std::ceil(n) : n + 0.25; };
    if (tile == kHalf256) return 5.0 + shared(tiles / kLinearCus) * (1.9 * slabs + (gelu ? 17.5 : 8.0));
    const double n = tiles / (2 * kLinearCus), beside = gelu ? 8.0 : 5.0;
    return 5.0 + (n <= 0.5 ? 0.68 * slabs + 0.6 * beside : shared(n) * (1.06 * slabs + beside));
}

// Groups of unknown rows are taken as even, with half a tile more each
HalfTile pick_half_tile(LinearKind kind, const LinearGemm &g)
{
    auto time = [&](HalfTile tile) {
        const int size = tile == kHalf256 ? 256 : 128;
        const double cols = (g.Nout + size - 1) / size, per = (double)g.rows / g.N;
        if (kind == kLinearWeightGrad) return linear_half_time(tile, (double)g.parts * ((g.Mrows + size - 1) / size) * cols, std::ceil((double)g.rows / g.parts / 64), false);
        const double tiles = g.N == 1 ? std::ceil(per / size) : std::min((double)g.rows, g.N * std::max(1.0, per / size + 0.5));
        return linear_half_time(tile, g.parts * tiles * cols, std::ceil((double)g.K / g.parts / 64), g.act == 2);
    };
    return time(kHalf256) <= time(kHalf128) ? kHalf256 : kHalf128;
}

hipError_t launch_linear_half(int dtype, const LinearGemm &g, LinearKind kind, HalfTile tile, const Tuning &tune, hipStream_t s)
{
    if (dtype == SMILE_DTYPE_BF16) return launch_typed<__bf16>(g, kind, tile, tune, s);
    return launch_typed<_Float16>(g, kind, tile, tune, s);
}

}  // namespace smile
