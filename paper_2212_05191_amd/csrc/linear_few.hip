// The products of linear_few.hpp: how many rows at a time.
#include <algorithm>

#include "linear_few.hpp"

namespace smile {

namespace {

// Rows of a group that the kernel goes by: of several groups, whose rows the host does not know, a half more than the average
int few_rows(const LinearGemm &g) { return g.N == 1 ? g.rows : (int)((g.rows * 3ll / 2 + g.N - 1) / g.N); }

// row tiles of `size` rows, a half more than they have a group
double row_tiles(const LinearGemm &g, int size)
{
    const double per = (double)g.rows / g.N;
    return g.N == 1 ? (g.rows + size - 1) / size : std::min((double)g.rows, g.N * std::max(1.0, per / size + 0.5));
}

template <typename E>
hipError_t launch_typed(const LinearGemm &g, int rows, const Tuning &tune, hipStream_t s)
{
    if (rows <= 16) return launch_few<E, 1>(g, tune, s);
    if (rows <= 32) return launch_few<E, 2>(g, tune, s);
    return launch_few<E, 4>(g, tune, s);
}

}  // namespace

// Estimated times, us.  Measured with bfloat16 and GELU in a graph, this kernel and the tiles of 128 x 128: 1024 -> 4096, 1 row 3.8 / 13.7, 16 4.5 / 13.8, 32 5.5 / 14.0,
// 64 7.5 / 13.9, 128 11.9 / 17.0, 256 21.4 / 17.2, 512 40 / 17.6; 4096 -> 1024, 16 rows 9.6 / 38, 64 20.2 / 38, 256 21.3 / 45, 512 38.5 / 45; 256 -> 256, 256 rows 4.0 / 9.7;
// 64 groups 1024 -> 4096, 16 rows in all 21.3 / 21.8, 128 97 / 90, 1024 225 / 104 (the weights' bytes 26, 103, 103); 16 groups 768 -> 2304, 1024 rows 53 / 20; 8 groups
// 256 -> 512, 2000 rows 11.5 / 9.1.  Here a workgroup's time goes with its rows and terms,
// and the workgroups share the CUs; there a slab costs 0.6 us as long as the tiles do not fill the chip.
bool linear_few_applies(const LinearGemm &g)
{
    const int rows = few_rows(g), size = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    const double k = g.K / 1024.0, cost = size == 16 ? 1.6 : size == 32 ? 2.5 : 4.3;
    const double here = row_tiles(g, size) * ((g.Nout + 15) / 16) / kLinearCus, tiles = row_tiles(g, 128) * ((g.Nout + 127) / 128) / (1.5 * kLinearCus);
    return 3.2 + cost * (k + 0.1) * std::max(1.0, here) < 6.0 + 9.6 * k * std::max(1.0, tiles);
}

hipError_t launch_linear_few(int dtype, const LinearGemm &g, const Tuning &tune, hipStream_t s)
{
    const int rows = few_rows(g);
    return dtype == SMILE_DTYPE_BF16 ? launch_typed<__bf16>(g, rows, tune, s) : launch_typed<_Float16>(g, rows, tune, s);
}

}  // namespace smile
