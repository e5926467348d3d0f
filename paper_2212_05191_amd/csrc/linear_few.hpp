// Products of a few rows a group in 16 bits: the weights are read once, straight into registers, for up to 16 RB rows at a time.
//
// A workgroup of eight waves computes 16 columns; the waves take chunks of 64 terms in turns, and their sums are added through LDS in their order.  A lane reads 32
// neighbouring bytes of a weight row (four lanes a line of 128) and the same of each row of x, two operands of v_mfma_f32_16x16x32: the order of the
// terms inside a chunk does not matter, as long as both operands have the same.  Everything of kAhead chunks is requested before the first is used.
// Bound: the weights' bytes where there are enough of them (64 groups), else the latency of a chain: rows, loads, sum of eight waves, store.
#pragma once

#include "linear_walk.hpp"

namespace smile {

namespace {

template <typename E, int RB, int ACT>
__global__ __launch_bounds__(512) void linear_few_kernel(LinearGemm a)
{
    typedef typename Half<E>::vec8 vec8;
    constexpr int BM = 16 * RB, BN = 16, WAVES = 8, kAhead = RB == 4 ? 2 : 4;
    __shared__ float part[WAVES][BM][BN + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    RowWalk<BM, 1> walk;
    walk.init(a);
    const int chunks = (a.K + 63) / 64;
    for (int n = 0;; ++n) {
        LinearTile t;
        if (!walk.tile(a, n, BN, t)) return;
        const E *w = static_cast<const E *>(a.w) + (size_t)t.e * a.sw + (size_t)min(t.col0 + r, a.Nout - 1) * a.ldw + g * 16;
        const E *x[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) x[b] = static_cast<const E *>(a.x) + (size_t)(t.first + min(b * 16 + r, t.rows - 1)) * a.ldx + g * 16;
        mfma_f32x4 acc[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[b] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
        for (int c0 = wave; c0 < chunks; c0 += WAVES * kAhead) {
            u32x4 wf[kAhead][2], xf[kAhead][RB][2];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = (c0 + u * WAVES) * 64 + h * 8;
                    const bool some = k + g * 16 < a.K;      // K is a multiple of 8: a piece exists or not
                    wf[u][h] = u32x4{0u, 0u, 0u, 0u};
                    if (some) wf[u][h] = *reinterpret_cast<const u32x4 *>(w + k);
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        xf[u][b][h] = u32x4{0u, 0u, 0u, 0u};
                        if (some) xf[u][b][h] = *reinterpret_cast<const u32x4 *>(x[b] + k);
                    }
                }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int b = 0; b < RB; ++b)
                        acc[b] = Half<E>::mfma_16x16x32(__builtin_bit_cast(vec8, wf[u][h]), __builtin_bit_cast(vec8, xf[u][b][h]), acc[b]);
        }
        // element v of a lane: column 4 (lane / 16) + v, row lane % 16
        __syncthreads();   // (the sums of the tile before have been read)
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) part[wave][b * 16 + r][4 * g + v] = acc[b][v];
        __syncthreads();
        for (int id = threadIdx.x; id < BM * 8; id += 512) {
            const int row = id >> 3, c = (id & 7) * 2, col = t.col0 + c;
            if (row >= t.rows || col >= a.Nout) continue;
            float v[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[i] = part[0][row][c + i];
#pragma unroll
                for (int o = 1; o < WAVES; ++o) v[i] += part[o][row][c + i];
            }
            const size_t at = (size_t)(t.first + row) * a.Nout + col;
            auto pair = [](const void *p, size_t i) { return *reinterpret_cast<const uint32_t *>(static_cast<const E *>(p) + i); };
            auto store = [](void *p, size_t i, uint32_t w) { *reinterpret_cast<uint32_t *>(static_cast<E *>(p) + i) = w; };
            if (a.bias) {
                const uint32_t w2 = pair(a.bias, (size_t)t.e * a.Nout + col);
                v[0] += Half<E>::lo(w2), v[1] += Half<E>::hi(w2);
            }
            if (a.pre) store(a.pre, at, Half<E>::pack(v[0], v[1]));
            v[0] = linear_act<false>(ACT, v[0]), v[1] = linear_act<false>(ACT, v[1]);
            if (a.residual) {
                const uint32_t w2 = pair(a.residual, at);
                v[0] += Half<E>::lo(w2), v[1] += Half<E>::hi(w2);
            }
            store(a.y, at, Half<E>::pack(v[0], v[1]));
        }
    }
}

template <typename E, int RB>
hipError_t launch_few(LinearGemm g, const Tuning &tune, hipStream_t s)
{
    constexpr int BM = 16 * RB;
    g.col_tiles = (g.Nout + 15) / 16;
    const long long most = ((g.rows + BM - 1) / BM + (long long)std::min(g.N, g.rows) - 1) * g.col_tiles;
    if (most >= 1ll << 31) return hipErrorInvalidValue;
    const dim3 grid((unsigned)std::min((most + 7) / 8 * 8, (long long)workgroup_slots(tune, 4)));
    if (g.act == 0) SMILE_LAUNCH((linear_few_kernel<E, RB, 0>), grid, dim3(512), 0, s, g);
    else if (g.act == 1) SMILE_LAUNCH((linear_few_kernel<E, RB, 1>), grid, dim3(512), 0, s, g);
    else SMILE_LAUNCH((linear_few_kernel<E, RB, 2>), grid, dim3(512), 0, s, g);
    return hipGetLastError();
}

}  // namespace

}  // namespace smile
