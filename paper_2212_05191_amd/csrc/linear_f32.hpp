// Products over sorted rows on v_mfma_f32_32x32x2_f32: fp32 operands, products and sums.
//
// 64 x 64 outputs a workgroup of four waves (32 x 32 each), slabs of 32 terms: a thread loads eight elements of either operand for the next slab
// while this one is multiplied from LDS (two buffers, one barrier a slab).  A normal operand lies there as [row][32 k], rows 36 words apart, so that the
// 16-byte reads of 16 rows meet all banks; a transposed one as [k][64], k-rows 72 words apart, so that the halves of a wave (k and k + 4) do.  What is
// beyond a matrix or a group's rows is zero in both operands.
#pragma once

#include "linear_walk.hpp"

namespace smile {

namespace {

template <typename E>
struct Eight {   // eight neighbouring elements as fp32
    float v[8];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    __device__ __forceinline__ void load(const E *p)
    {
        if constexpr (sizeof(E) == 4) {
            const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
        } else {
            const u32x4 a = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = Half<E>::lo(a[i]), v[2 * i + 1] = Half<E>::hi(a[i]);
        }
    }
    __device__ __forceinline__ void store(E *p) const
    {
        if constexpr (sizeof(E) == 4) {
            reinterpret_cast<f32x4 *>(p)[0] = f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4 *>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
            *reinterpret_cast<u32x4 *>(p) = u32x4{Half<E>::pack(v[0], v[1]), Half<E>::pack(v[2], v[3]), Half<E>::pack(v[4], v[5]), Half<E>::pack(v[6], v[7])};
        }
    }
};

// four neighbouring elements
template <typename E>
__device__ __forceinline__ f32x4 load4(const E *p)
{
    typedef __attribute__((__vector_size__(4 * sizeof(E)))) E vec4;
    const vec4 a = *reinterpret_cast<const vec4 *>(p);
    return f32x4{(float)a[0], (float)a[1], (float)a[2], (float)a[3]};
}
template <typename E>
__device__ __forceinline__ void store4(E *p, f32x4 v)
{
    typedef __attribute__((__vector_size__(4 * sizeof(E)))) E vec4;
    *reinterpret_cast<vec4 *>(p) = vec4{(E)v[0], (E)v[1], (E)v[2], (E)v[3]};
}

constexpr int kF32Tile = 64, kF32Slab = 32, kF32Band = 8;

// GRAD: the weights' gradient (both operands transposed); WT: w transposed
template <typename E, bool GRAD, bool WT>
__global__ __launch_bounds__(256) void linear_f32_kernel(LinearGemm a)
{
    static_assert(!GRAD || WT, "the weights' gradient takes both operands transposed");
    constexpr int B = kF32Tile, BK = kF32Slab, NPITCH = BK + 4, TPITCH = B + 8;
    constexpr int OPERAND = NPITCH * B > TPITCH * BK ? NPITCH * B : TPITCH * BK;
    __shared__ __attribute__((aligned(16))) float lds[2][2][OPERAND];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const int frow = lane & 31, h = lane >> 5;

    std::conditional_t<GRAD, GradWalk<B>, RowWalk<B, kF32Band>> walk;
    walk.init(a);
    int buf = 0;
    for (int n = 0;; ++n) {
        LinearTile t;
        if constexpr (GRAD) {
            const int found = walk.tile(a, n, B, t);
            if (found < 0) return;
            if (found == 0) continue;
        } else {
            if (!walk.tile(a, n, B, t)) return;
        }
        const E *X = static_cast<const E *>(a.x) + (GRAD ? (size_t)t.from * a.ldx : (size_t)t.first * a.ldx + t.from);
        const E *W = static_cast<const E *>(a.w) + (GRAD ? 0 : (size_t)t.e * a.sw) + (WT ? (size_t)t.from * a.ldw : t.from);
        Eight<E> xr, wr;
        // this thread's elements of the slab from term k0 on: of an operand whose rows begin at `first` and number `ext`
        auto fetch = [&](Eight<E> &r, const E *p, auto transposed, int ld, int first, int ext, int k0) {
            r.zero();
            if constexpr (decltype(transposed)::value) {
                const int k = k0 + (tid >> 3), col = first + (tid & 7) * 8;
                if (k < t.kv && col < ext) r.load(p + (size_t)k * ld + col);
            } else {
                const int row = first + (tid >> 2), k = k0 + (tid & 3) * 8;
                if (k < t.kv && row < ext) r.load(p + (size_t)row * ld + k);
            }
        };
        auto fetch_slab = [&](int k0) {
            if constexpr (GRAD) fetch(xr, X, std::true_type{}, a.ldx, t.first, a.Mrows, k0);
            else fetch(xr, X, std::false_type{}, a.ldx, 0, t.rows, k0);
            fetch(wr, W, std::bool_constant<WT>{}, a.ldw, t.col0, a.Nout, k0);
        };
        auto put = [&](float *to, const Eight<E> &r, auto transposed) {
            float *p = decltype(transposed)::value ? to + (tid >> 3) * TPITCH + (tid & 7) * 8 : to + (tid >> 2) * NPITCH + (tid & 3) * 8;
            reinterpret_cast<f32x4 *>(p)[0] = f32x4{r.v[0], r.v[1], r.v[2], r.v[3]}, reinterpret_cast<f32x4 *>(p)[1] = f32x4{r.v[4], r.v[5], r.v[6], r.v[7]};
        };
        f32x16 acc;
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[v] = 0.f;
        const int slabs = (t.kv + BK - 1) / BK;
        if (slabs) fetch_slab(0);
        for (int s = 0; s < slabs; ++s, buf ^= 1) {
            put(lds[buf][0], xr, std::bool_constant<GRAD>{});
            put(lds[buf][1], wr, std::bool_constant<WT>{});
            __syncthreads();
            if (s + 1 < slabs) fetch_slab((s + 1) * BK);
            auto read = [&](const float *from, auto transposed, int first, int p) {   // terms 8 p + 4 h + i of row / column first + frow
                if constexpr (decltype(transposed)::value) {
                    const float *q = from + (8 * p + 4 * h) * TPITCH + first + frow;
                    return f32x4{q[0], q[TPITCH], q[2 * TPITCH], q[3 * TPITCH]};
                } else {
                    return *reinterpret_cast<const f32x4 *>(from + (first + frow) * NPITCH + 8 * p + 4 * h);
                }
            };
#pragma unroll
            for (int p = 0; p < BK / 8; ++p) {
                const f32x4 xf = read(lds[buf][0], std::bool_constant<GRAD>{}, wm * 32, p), wf = read(lds[buf][1], std::bool_constant<WT>{}, wn * 32, p);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(wf[q], xf[q], acc, 0, 0, 0);
            }
        }
        // element v of a lane: column 8 (v / 4) + 4 h + v % 4, row lane % 32 of the wave's block
        const int row = wm * 32 + frow;
        if (row >= t.rows) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = t.col0 + wn * 32 + 8 * q + 4 * h;
            if (col >= a.Nout) continue;
            f32x4 f = {acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
            const size_t at = (size_t)(t.first + row) * a.Nout + col;
            if (WT && a.partial) {
                *reinterpret_cast<f32x4 *>(a.partial + (size_t)t.part * a.sy + at) = f;
            } else if constexpr (GRAD) {
                store4(static_cast<E *>(a.y) + (size_t)t.e * a.sy + at, f);
            } else {
                if (a.bias) f += load4(static_cast<const E *>(a.bias) + (size_t)t.e * a.Nout + col);
                if (a.pre) store4(static_cast<E *>(a.pre) + at, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = linear_act<sizeof(E) == 4>(a.act, f[i]);
                if (a.residual) f += load4(static_cast<const E *>(a.residual) + at);
                store4(static_cast<E *>(a.y) + at, f);
            }
        }
    }
}

}  // namespace

}  // namespace smile
