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

// Time of `tiles` tiles in rounds of the chip, a round of 256 x 256 tiles being 1 (and of 128 x 128 tiles `weight`, a little more than half of that if half of
// the slots are empty); from three rounds on workgroups are out of step and share the last one.
double rounds(double tiles, int slots, double weight, double half)
{
    const double n = tiles / slots;
    if (n > 3.0) return weight * (n + 0.25);
    const double whole = std::floor(n), rest = n - whole;
    return weight * whole + (rest <= 0.0 ? 0.0 : rest <= 0.5 ? half : weight);
}

}  // namespace

// 256 x 256 outputs alone on a CU move half of the bytes from L2 that 128 x 128 do, but the epilogue waits for nobody and nobody multiplies meanwhile, and there
// are a quarter as many tiles to spread.  Measured, us, 256 and 128 (bfloat16, two cards, of which the second runs at a lower clock):
//   forward, 16384 rows 4096 -> 1024: 119 / 135 and 143 / 155; 64 groups of 512 rows, 1024 -> 4096: 337 / 363, 391 / 398; with GELU 420 / 402 and 467 / 435
//   gradient of x, 16384 rows 4096 -> 1024: 150 / 167, 170 / 200; of the weights, 64 groups: 387 / 451, 398 / 460
//   4096 rows 1024 -> 1024 (64 and 256 tiles): 30 / 15; 16 groups of 512 rows 768 -> 2304 with GELU: 66 / 44
// so that a round of two 128 x 128 tiles on each CU counts as 0.56 of one of 256 x 256, with GELU as 0.48.  Groups of unknown rows are taken as even, with half a
// tile more each.
HalfTile pick_half_tile(LinearKind kind, int N, int rows, int Mrows, int Nout, int act)
{
    auto tiles = [&](int size) {
        const double cols = (Nout + size - 1) / size, per = (double)rows / N;
        if (kind == kLinearWeightGrad) return (double)N * ((Mrows + size - 1) / size) * cols;
        return N == 1 ? std::ceil(per / size) * cols : (per < 1.0 ? rows : N * std::max(1.0, per / size + 0.5)) * cols;
    };
    const double big = tiles(256), small = tiles(128), weight = act == 2 ? 0.48 : 0.56;
    if (kind == kLinearWeightGrad && N * (long long)rows > 0) {   // few tiles: the sums are cut until the chip is full
        if (big < kLinearCus && small < 2 * kLinearCus) return rows >= 8192 && big >= 16 ? kHalf256 : kHalf128;
    }
    return rounds(big, kLinearCus, 1.0, 1.0) <= rounds(small, 2 * kLinearCus, weight, 0.7 * weight) ? kHalf256 : kHalf128;
}

hipError_t launch_linear_half(int dtype, const LinearGemm &g, LinearKind kind, HalfTile tile, const Tuning &tune, hipStream_t s)
{
    if (dtype == SMILE_DTYPE_BF16) return launch_typed<__bf16>(g, kind, tile, tune, s);
    return launch_typed<_Float16>(g, kind, tile, tune, s);
}

}  // namespace smile
