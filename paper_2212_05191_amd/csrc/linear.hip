// Products of sorted or dense rows with bias, activation and residual, and their gradients: the choice of kernels, and the kernels beside the products.
#include "linear_f32.hpp"
#include "sorted_internal.hpp"

#include <algorithm>
#include <type_traits>

namespace smile {

namespace {

// rows of a part of the bias gradient's sums: 16384 rows of 1024 values take 12.4 us by 128, 9.2 by 64, 8.0 by 32, their sums 4.0, 4.4 and 7.7 more
constexpr int kGradRows = 64;

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// ---- g = dy act'(pre) in the storage type, and its sums over the rows of each part, before that rounding.  Both products take it as an operand of the 16-bit matrix
// instructions, so that it is rounded like dy and pre themselves: dx and dw then have two roundings instead of one (half precision, 15 groups: 2.9e-4 from 64 bits, with g in fp32
// 2.1e-4), and in half precision a g above 65504 is infinite.  Parts: rows cut at the multiples of
// kGradRows and at the groups' ends, numbered as in GradWalk.  A workgroup takes 256 columns of a part, 8 a thread, a row in eight.  Bound: HBM (dy and pre
// read, g written).
struct GradRows {
    const void *dy, *pre;
    const int32_t *start;
    void *g;                   // or null
    float *sums;               // [parts][F] or null
    int N, rows, F, act;
};

template <typename E>
__global__ __launch_bounds__(256) void linear_grad_rows_kernel(GradRows a)
{
    __shared__ float part[8][256 + 4];
    int e = 0, above = a.N;
    const int id = blockIdx.x;
    while (above - e > 1) {
        const int mid = (e + above) / 2;
        if (min(max(a.start[mid], 0), a.rows) / kGradRows + mid <= id) e = mid;
        else above = mid;
    }
    int lo, hi;
    group_rows(a.start, a.rows, e, lo, hi);
    const long long begin = (long long)(id - e) * kGradRows;
    lo = (int)max((long long)lo, begin), hi = (int)min((long long)hi, begin + kGradRows);
    if (lo >= hi) return;
    const int col = blockIdx.y * 256 + (threadIdx.x & 31) * 8, sub = threadIdx.x >> 5;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    if (col < a.F)
#pragma unroll 4
        for (int r = lo + sub; r < hi; r += 8) {
            const size_t at = (size_t)r * a.F + col;
            Eight<E> d, p;
            d.load(static_cast<const E *>(a.dy) + at);
            if (a.act) {
                p.load(static_cast<const E *>(a.pre) + at);
#pragma unroll
                for (int i = 0; i < 8; ++i) d.v[i] *= linear_act_grad<sizeof(E) == 4>(a.act, p.v[i]);
                if (a.g) d.store(static_cast<E *>(a.g) + at);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += d.v[i];
        }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[sub][(threadIdx.x & 31) * 8 + i] = sum[i];
    __syncthreads();
    const int c = blockIdx.y * 256 + threadIdx.x;
    if (c >= a.F) return;
    float s = part[0][threadIdx.x];
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i][threadIdx.x];
    a.sums[(size_t)id * a.F + c] = s;
}

// dbias[e][c] = sum of the parts of group e, in 64 bits and in their order (four threads a column, then theirs)
template <typename E>
__global__ __launch_bounds__(256) void linear_bias_sum_kernel(const float *sums, const int32_t *start, E *dbias, int rows, int F)
{
    __shared__ double part[4][64];
    const int e = blockIdx.y, c = blockIdx.x * 64 + (threadIdx.x & 63), sub = threadIdx.x >> 6;
    int lo, hi;
    group_rows(start, rows, e, lo, hi);
    double s = 0.0;
    if (lo < hi && c < F) {
        const int first = lo / kGradRows, last = (hi - 1) / kGradRows;
#pragma unroll 8
        for (int b = first + sub; b <= last; b += 4) s += (double)sums[(size_t)(b + e) * F + c];
    }
    part[sub][threadIdx.x & 63] = s;
    __syncthreads();
    if (sub == 0 && c < F) dbias[(size_t)e * F + c] = (E)(float)((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]));
}

// dw[e] = sum of the parts of group e, in fp32 in their order.  Bound: HBM (the parts are read once).
template <typename E>
__global__ __launch_bounds__(256) void linear_part_sum_kernel(const float *partial, const int32_t *start, E *dw, int rows, int chunk, long long size)
{
    const int e = blockIdx.y;
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= size) return;
    int lo, hi;
    group_rows(start, rows, e, lo, hi);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (lo < hi)
#pragma unroll 4
        for (int b = lo / chunk; b <= (hi - 1) / chunk; ++b) s += *reinterpret_cast<const f32x4 *>(partial + (size_t)(b + e) * size + at);
    store4(dw + (size_t)e * size + at, s);
}

// dx[r] = sum of the parts of row r, in fp32 in their order
template <typename E>
__global__ __launch_bounds__(256) void linear_row_sum_kernel(const float *partial, const int32_t *start, E *dx, int N, int rows, int K, int parts)
{
    int lo = 0, hi = rows;
    if (start) lo = min(max(start[0], 0), rows), hi = min(max(start[N], 0), rows);
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4, size = (long long)rows * K;
    if (at < (long long)lo * K || at >= (long long)hi * K) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) s += *reinterpret_cast<const f32x4 *>(partial + p * size + at);
    store4(dx + at, s);
}

// How the gradients' sums are cut into parts, where their tiles leave the chip idle: the tile and the number of parts with the least estimated time, of which a part
// costs a launch and its bytes, written and read in fp32 (at 9 TB/s: they mostly stay in the caches).  The parts of both gradients share a piece of the workspace.
struct GradPlan {
    int chunk, parts;         // weights: rows of a part (0: whole groups), parts of all groups
    int x_chunk, x_parts;     // rows: terms of a part, parts
    HalfTile tile, x_tile;    // of the weights' gradient and the rows', 16-bit types
    size_t sums_at, partial_at, total;
};
constexpr int kMostParts = 16;
double parts_time(int parts, double elements) { return parts > 1 ? 4.0 + parts * elements * 8.0 / 9e6 : 0.0; }

GradPlan grad_plan(const smile_linear_backward_args &a)
{
    GradPlan p{};
    const bool half = a.dtype != SMILE_DTYPE_F32;
    // An fp32 tile of 64 x 64 outputs, four of them on a CU, is counted as half a tile of 128 x 128 in 16 bits with half again as many slabs.  That is less than it takes: a slab of 64
    // terms 0.9 us alone on a CU and 1.5 on a full chip, measured 1.2 to 1.6 (16 rows 1024 -> 4096) and 4.4 (4096^3 in 1120 us, 122 of the library's 154 TFLOP/s).  Large sums are
    // rightly left whole and few tiles rightly cut; in between the estimate chooses wrongly (gradient of the weights: 2 groups, 1500 rows, 520 x 1032 whole 58 us, in five parts 32;
    // 8 groups, 8000 rows, 256 x 512 in 23 parts 48 us, whole 33).
    auto time = [&](LinearKind kind, int size, double tiles, double slabs) {
        return half ? linear_half_time(size == 256 ? kHalf256 : kHalf128, kind, tiles, slabs, false) : linear_half_time(kHalf128, kind, tiles / 2, 1.5 * slabs, false);
    };
    auto tiles_of = [](int n, int size) { return (n + size - 1) / size; };
    p.parts = a.N, p.tile = p.x_tile = kHalf128;
    if (a.dw) {
        const double elements = (double)a.N * a.F * a.K;
        double best = 1e30;
        int cuts = 1;
        for (const int size : {half ? 128 : kF32Tile, 256}) {
            if (!half && size == 256) break;
            for (int n = 1; n <= kMostParts && (n == 1 || (long long)a.N * n * 256 <= a.rows); ++n) {
                const double per_group = std::ceil((double)a.rows / a.N / n / 64);
                const double t = time(kLinearWeightGrad, size, (double)a.N * n * tiles_of(a.F, size) * tiles_of(a.K, size), per_group) + parts_time(n, elements);
                if (t < best) best = t, cuts = n, p.tile = size == 256 ? kHalf256 : kHalf128;
            }
        }
        if (cuts > 1) {
            p.chunk = (int)std::max(64ll, ((long long)a.rows / a.N / cuts + 63) / 64 * 64);
            p.parts = tiles_of(a.rows, p.chunk) + a.N - 1;
        }
    }
    p.x_parts = 1;
    if (a.dx) {
        const int slabs = tiles_of(a.F, 64);
        const double per = (double)a.rows / a.N;
        double best = 1e30;
        int cuts = 1;
        for (const int size : {half ? 128 : kF32Tile, 256}) {
            if (!half && size == 256) break;
            const double tiles = (a.N == 1 ? std::ceil(per / size) : std::min((double)a.rows, a.N * std::max(1.0, per / size + 0.5))) * tiles_of(a.K, size);
            for (int n = 1; n <= kMostParts && (n == 1 || 4 * n <= slabs); ++n) {
                const double t = time(kLinearRowGrad, size, tiles * n, tiles_of(slabs, n)) + parts_time(n, (double)a.rows * a.K);
                if (t < best) best = t, cuts = n, p.x_tile = size == 256 ? kHalf256 : kHalf128;
            }
        }
        if (cuts > 1) {
            p.x_chunk = tiles_of(slabs, cuts) * 64;
            p.x_parts = tiles_of(a.F, p.x_chunk);
        }
    }
    const bool own_g = a.act != SMILE_ACT_NONE && (a.dx || a.dw);
    p.sums_at = round256(own_g ? (size_t)a.rows * a.F * elem_size(a.dtype) : 0);
    p.partial_at = p.sums_at + round256(a.dbias ? ((size_t)(a.rows + kGradRows - 1) / kGradRows + a.N - 1) * a.F * sizeof(float) : 0);
    p.total = p.partial_at + round256(std::max(p.chunk ? (size_t)p.parts * a.F * a.K * sizeof(float) : 0, p.x_parts > 1 ? (size_t)p.x_parts * a.rows * a.K * sizeof(float) : 0));
    return p;
}

int act_of(int act) { return act == SMILE_ACT_NONE ? 0 : act == SMILE_ACT_RELU ? 1 : 2; }

template <typename E, bool GRAD, bool WT>
hipError_t launch_f32(LinearGemm g, const Tuning &tune, hipStream_t s)
{
    g.col_tiles = (g.Nout + kF32Tile - 1) / kF32Tile, g.row_tiles = (g.Mrows + kF32Tile - 1) / kF32Tile;
    const long long most = g.parts * (GRAD ? (long long)g.row_tiles : (g.rows + kF32Tile - 1) / kF32Tile + (long long)std::min(g.N, g.rows) - 1) * g.col_tiles;
    if (most >= 1ll << 31) return hipErrorInvalidValue;
    const int grid = (int)std::min((most + 7) / 8 * 8, (long long)workgroup_slots(tune, 4));
    SMILE_LAUNCH((linear_f32_kernel<E, GRAD, WT>), dim3(grid), dim3(256), 0, s, g);
    return hipGetLastError();
}

template <typename E, bool GRAD, bool WT>
hipError_t launch_product(const LinearGemm &g, const Tuning &tune, hipStream_t s, HalfTile tile = kHalf128)
{
    if constexpr (sizeof(E) == 4) return launch_f32<E, GRAD, WT>(g, tune, s);
    else {
        const int dtype = std::is_same_v<E, __bf16> ? SMILE_DTYPE_BF16 : SMILE_DTYPE_F16;
        if (WT) return launch_linear_half(dtype, g, GRAD ? kLinearWeightGrad : kLinearRowGrad, tile, tune, s);   // (the gradients' tiles go with their parts)
        return linear_few_applies(g) ? launch_linear_few(dtype, g, tune, s) : launch_linear_half(dtype, g, kLinearForward, forward_half_tile(g), tune, s);
    }
}

template <typename E>
hipError_t forward(const smile_linear_args &a, const Tuning &tune, hipStream_t s)
{
    LinearGemm g{};
    g.x = a.x, g.w = a.w, g.bias = a.bias, g.residual = a.residual, g.y = a.y, g.pre = a.pre, g.start = a.start;
    g.N = a.N, g.rows = a.rows, g.Nout = a.F, g.K = a.K, g.ldx = a.K, g.ldw = a.K, g.sw = (long long)a.F * a.K, g.act = act_of(a.act), g.parts = 1;
    return launch_product<E, false, false>(g, tune, s);
}

template <typename E>
hipError_t backward(const smile_linear_backward_args &a, const Tuning &tune, void *workspace, hipStream_t s)
{
    const GradPlan p = grad_plan(a);
    char *ws = static_cast<char *>(workspace);
    const int act = act_of(a.act);
    const void *g = a.dy;
    if ((act && (a.dx || a.dw)) || a.dbias) {
        GradRows r{a.dy, a.pre, a.start, nullptr, a.dbias ? reinterpret_cast<float *>(ws + p.sums_at) : nullptr, a.N, a.rows, a.F, act};
        if (act && (a.dx || a.dw)) g = r.g = ws;
        const int parts = (a.rows + kGradRows - 1) / kGradRows + a.N - 1;
        SMILE_LAUNCH(linear_grad_rows_kernel<E>, dim3(parts, (a.F + 255) / 256), dim3(256), 0, s, r);
        if (a.dbias)
            SMILE_LAUNCH(linear_bias_sum_kernel<E>, dim3((a.F + 63) / 64, a.N), dim3(256), 0, s, (const float *)r.sums, a.start, static_cast<E *>(a.dbias), a.rows, a.F);
    }
    if (a.dx) {
        LinearGemm m{};
        m.x = g, m.w = a.w, m.y = a.dx, m.start = a.start, m.N = a.N, m.rows = a.rows, m.Nout = a.K, m.K = a.F, m.ldx = a.F, m.ldw = a.K;
        m.sw = (long long)a.F * a.K, m.sy = (long long)a.rows * a.K, m.chunk = p.x_chunk, m.parts = p.x_parts;
        if (p.x_parts > 1) m.partial = reinterpret_cast<float *>(ws + p.partial_at);
        const hipError_t err = launch_product<E, false, true>(m, tune, s, p.x_tile);
        if (err != hipSuccess) return err;
        if (p.x_parts > 1)
            SMILE_LAUNCH(linear_row_sum_kernel<E>, dim3((unsigned)((m.sy + 1023) / 1024)), dim3(256), 0, s, (const float *)m.partial, a.start, static_cast<E *>(a.dx), a.N, a.rows,
                         a.K, p.x_parts);
    }
    if (a.dw) {
        LinearGemm m{};
        m.x = g, m.w = a.x, m.y = a.dw, m.start = a.start, m.N = a.N, m.rows = a.rows, m.Mrows = a.F, m.Nout = a.K, m.ldx = a.F, m.ldw = a.K;
        m.sy = (long long)a.F * a.K, m.chunk = p.chunk, m.parts = p.parts;
        if (p.chunk) m.partial = reinterpret_cast<float *>(ws + p.partial_at);
        const hipError_t err = launch_product<E, true, true>(m, tune, s, p.tile);
        if (err != hipSuccess) return err;
        if (p.chunk)
            SMILE_LAUNCH(linear_part_sum_kernel<E>, dim3((unsigned)((m.sy + 1023) / 1024), a.N), dim3(256), 0, s, (const float *)m.partial, a.start, static_cast<E *>(a.dw),
                         a.rows, p.chunk, m.sy);
    }
    return hipGetLastError();
}

}  // namespace

size_t linear_backward_workspace(const smile_linear_backward_args &a) { return grad_plan(a).total; }

hipError_t launch_linear(const smile_linear_args &a, const Tuning &tune, hipStream_t s)
{
    if (a.dtype == SMILE_DTYPE_F32) return forward<float>(a, tune, s);
    return a.dtype == SMILE_DTYPE_BF16 ? forward<__bf16>(a, tune, s) : forward<_Float16>(a, tune, s);
}

hipError_t launch_linear_backward(const smile_linear_backward_args &a, const Tuning &tune, void *workspace, hipStream_t s)
{
    if (a.dtype == SMILE_DTYPE_F32) return backward<float>(a, tune, workspace, s);
    return a.dtype == SMILE_DTYPE_BF16 ? backward<__bf16>(a, tune, workspace, s) : backward<_Float16>(a, tune, workspace, s);
}

}  // namespace smile
