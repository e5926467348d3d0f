// Root-mean-square norm with the residual's addition, 16-bit (or fp32) and 8-bit outputs, and its gradients.
//
//   s = x + residual (rounded),  rstd = (mean s^2 + eps)^-1/2,  y = s rstd w
//   u = s rstd, g = w dy:  ds = dsum + rstd (g - u mean(g u)),  dw = sum over rows of dy u
//
// Bound: HBM.  Forward reads x and residual and writes s, y and the codes, nine bytes an element with 16-bit storage; backward reads dy, dsum
// and s and writes ds.  A row stays in the registers of LPR lanes between its two uses, eight neighbouring elements (16 bytes of 16-bit
// storage) at a time, so that each tensor is touched once.  Sixteen such lanes are a block of the 8-bit output, whose
// largest magnitude is found by four DPP steps.  A group of lanes takes consecutive rows, requests the next one
// before it works on this one, and keeps its part of w, and of dw, in registers over all of them.  The sum over rows for dw is one
// fp32 vector per workgroup, added up by a second launch in a fixed order.
#include "fp8_device.hpp"
#include "fp8_internal.hpp"

namespace smile {

namespace {

constexpr int kThreads = 256;

// sum over the LPR lanes of a row, in all of them; LPR == kThreads: over the workgroup, through `lds`
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float *lds)
{
#pragma unroll
    for (int off = 1; off < (LPR < 64 ? LPR : 64); off <<= 1) v += __shfl_xor(v, off, 64);
    if constexpr (LPR > 64) {
        __syncthreads();   // the row before is done with lds
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < LPR / 64; ++w) v += lds[w];
    }
    return v;
}

// LPR lanes a row, NP pieces of eight columns a lane: piece i of lane `sub` is columns 8 (i LPR + sub) ..
template <int DT, int LPR, int NP>
__global__ __launch_bounds__(kThreads) void rms_norm_kernel(RmsNormIo io, int rows_per_group)
{
    typedef Piece<DT> P;
    __shared__ float lds[kThreads / 64];
    const int sub = threadIdx.x % LPR, d = io.d, T = io.T;
    const int first = (blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR) * rows_per_group;
    const int last = min(first + rows_per_group, T);
    const int pitch = (d + kFp8Block - 1) / kFp8Block * kFp8Block, line = (T + 15) / 16 * 16;
    bool in[NP];
    float w[NP][8];
    typename P::Raw rx[NP], rr[NP];
    const auto request = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!in[i]) continue;
            const size_t at = (size_t)t * d + (i * LPR + sub) * 8;
            rx[i] = P::load(io.x, at);
            if (io.residual) rr[i] = P::load(io.residual, at);
        }
    };
#pragma unroll
    for (int i = 0; i < NP; ++i) in[i] = (i * LPR + sub) * 8 < d;
    // (a workgroup of one row per LPR lanes walks its rows together, as row_sum may need all of it)
    if (first < T) request(first);
#pragma unroll
    for (int i = 0; i < NP; ++i)
        if (in[i]) P::widen(P::load(io.weight, (i * LPR + sub) * 8), w[i]);
    const float inv_d = 1.0f / (float)d;
    for (int t = first; t < last; ++t) {
        float v[NP][8];
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
            if (!in[i]) continue;
            P::widen(rx[i], v[i]);
            if (io.residual) {
                float r[8];
                P::widen(rr[i], r);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[i][k] += r[k];
                const typename P::Raw s = P::narrow(v[i]);   // the stream is kept rounded, and its norm is that of what is kept
                P::widen(s, v[i]);
                if (io.sum) P::store(io.sum, (size_t)t * d + (i * LPR + sub) * 8, s);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sq = fmaf(v[i][k], v[i][k], sq);
        }
        if (t + 1 < last) request(t + 1);
        const float rstd = 1.0f / sqrtf(row_sum<LPR>(sq, lds) * inv_d + io.eps);
        if (io.rstd && sub == 0) io.rstd[t] = rstd;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int col = (i * LPR + sub) * 8;
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = in[i] ? v[i][k] * rstd * w[i][k] : 0.f;
            if (io.y && in[i]) P::store(io.y, (size_t)t * d + col, P::narrow(y));
            if (io.y8 && col < pitch) {   // whole blocks: the sixteen lanes of one agree
                u32x2 codes;
                const uint32_t byte = pack_block(y, codes);
                *reinterpret_cast<u32x2 *>(io.y8 + (size_t)t * pitch + col) = codes;
                if (sub % 16 == 0) io.y8_scale[(size_t)(col / kFp8Block) * line + t] = (uint8_t)byte;
            }
        }
    }
}

template <int DT, int LPR, int NP>
__global__ __launch_bounds__(kThreads) void rms_norm_backward_kernel(RmsNormGradIo io, int rows_per_group)
{
    typedef Piece<DT> P;
    constexpr int GROUPS = kThreads / LPR;
    __shared__ float lds[kThreads / 64];
    __shared__ float dw_lds[GROUPS > 1 ? GROUPS * NP * LPR * 8 : 1];
    const int sub = threadIdx.x % LPR, group = threadIdx.x / LPR, d = io.d, T = io.T;
    const int first = (blockIdx.x * GROUPS + group) * rows_per_group;
    const int last = min(first + rows_per_group, T);
    bool in[NP];
    float w[NP][8], dw[NP][8];
    typename P::Raw ry[NP], rs[NP], ra[NP];
    float next_rstd = 0.f;
    const auto request = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!in[i]) continue;
            const size_t at = (size_t)t * d + (i * LPR + sub) * 8;
            ry[i] = P::load(io.dy, at);
            rs[i] = P::load(io.s, at);
            if (io.dsum) ra[i] = P::load(io.dsum, at);
        }
        next_rstd = io.rstd[t];
    };
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        in[i] = (i * LPR + sub) * 8 < d;
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[i][k] = 0.f;
    }
    if (first < T) request(first);
#pragma unroll
    for (int i = 0; i < NP; ++i)
        if (in[i]) P::widen(P::load(io.weight, (i * LPR + sub) * 8), w[i]);
    const float inv_d = 1.0f / (float)d;
    for (int t = first; t < last; ++t) {
        const float rstd = next_rstd;
        float g[NP][8], u[NP][8], a[NP][8];
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!in[i]) continue;
            float y[8];
            P::widen(ry[i], y);
            P::widen(rs[i], u[i]);
            if (io.dsum) P::widen(ra[i], a[i]);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                u[i][k] *= rstd;
                g[i][k] = y[k] * w[i][k];
                dot = fmaf(g[i][k], u[i][k], dot);
                dw[i][k] = fmaf(y[k], u[i][k], dw[i][k]);
            }
        }
        if (t + 1 < last) request(t + 1);
        const float c = row_sum<LPR>(dot, lds) * inv_d;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (!in[i]) continue;
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = fmaf(rstd, fmaf(-u[i][k], c, g[i][k]), io.dsum ? a[i][k] : 0.f);
            P::store(io.ds, (size_t)t * d + (i * LPR + sub) * 8, P::narrow(o));
        }
    }
    // the workgroup's part of dw: its groups in order
    float *part = io.partial + (size_t)blockIdx.x * d;
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) dw_lds[(group * NP * LPR + i * LPR + sub) * 8 + k] = dw[i][k];
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += kThreads) {
            float v = 0.f;
            for (int q = 0; q < GROUPS; ++q) v += dw_lds[q * NP * LPR * 8 + c];
            part[c] = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if (in[i])
                Piece<SMILE_DTYPE_F32>::store(part, (i * LPR + sub) * 8, Piece<SMILE_DTYPE_F32>::narrow(dw[i]));
    }
}

// dweight[c] = sum of the workgroups' parts, 16 columns a workgroup: thread (c, q) adds parts q, q + 64, ... in order, eight loads in flight, then the
// 64 are added in order, in 64 bits (a column has up to some thousand parts of either sign).
__global__ __launch_bounds__(1024) void rms_norm_dweight_kernel(const float *__restrict__ part, float *__restrict__ dweight, int parts, int d)
{
    __shared__ double lds[64][17];
    const int lc = threadIdx.x % 16, c = blockIdx.x * 16 + lc, q = threadIdx.x / 16;
    double v = 0.;
    if (c < d) {
        int p = q;
        for (; p + 7 * 64 < parts; p += 8 * 64) {
            float a[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = part[(size_t)(p + i * 64) * d + c];
#pragma unroll
            for (int i = 0; i < 8; ++i) v += (double)a[i];
        }
        for (; p < parts; p += 64) v += (double)part[(size_t)p * d + c];
    }
    lds[q][lc] = v;
    __syncthreads();
    if (q < 8) {
        v = 0.;
#pragma unroll
        for (int k = 0; k < 8; ++k) v += lds[q * 8 + k][lc];
    }
    __syncthreads();
    if (q < 8) lds[q][lc] = v;
    __syncthreads();
    if (q == 0 && c < d) {
#pragma unroll
        for (int k = 1; k < 8; ++k) v += lds[k][lc];
        dweight[c] = (float)v;
    }
}

// Workgroups at most, each of consecutive rows: four a CU forward, three backward, whose number is that of the parts of dw.  That many are resident with
// one or two pieces a lane in 16 bits (88 and 140 registers), which they were measured with.  Of four pieces (1032 to 2048 and 4104 to 8192 columns: 138 and 250
// registers) three and two are, of eight two and one; fp32 backward: two of two pieces, one beyond.  Those run in more than one round.
// Part of a row is in accumulation registers in backward beyond 8192 columns, in fp32 beyond 1024, where 16384 columns spill too.  us, 65536 x 1024 bf16, y alone: 768 116, 1024 103, 1280 111, 2048 108 (a copy of its bytes: 104); y8 alone 105, 92, 100, 98
// (91); backward 512 114, 768 113, 1024 113, 4096 118 (104); 16384 x 1024: 28.3, 25.9, 27.3, 36.4 (26.0); 5003 x 960 fp16 12.4, 11.9, 11.9, 15.2 (7.4).
// Wide rows as they are (y and sum; backward; a copy of either's bytes): bf16 8192 x 1600 21, 27 (20), 65536 x 1600 230, 177 (163), 65536 x 2048 256, 224 (208),
// 16384 x 4096 108, 116 (104), 16384 x 8192 261, 242 (208), 4096 x 16384 122, 143 (104); fp32 65536 x 1024 219, 217 (208), 65536 x 1600 383, 335 (325),
// 16384 x 4096 213, 226 (208), 4096 x 16384 224, 314 (208).
constexpr int kForwardBlocks = 1024, kGradBlocks = 768;

struct NormShape {
    int lanes, pieces;
};
// Lanes for a row and pieces for a lane.  Rows up to 2048 columns stay within a wave, so that nothing waits for another wave; fewer rows
// than the chip has waves, and wider ones, take the workgroup.
NormShape norm_shape(int T, int d)
{
    const int pieces = (d + 7) / 8;
    int lanes = pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
    if (pieces > 256 || (pieces > 64 && T <= 1024)) lanes = kThreads;
    int np = 1;
    while (np * lanes < pieces) np *= 2;
    return {lanes, np};
}

template <int DT, int LPR, int NP>
hipError_t launch_shape(const RmsNormIo *f, const RmsNormGradIo *g, hipStream_t s)
{
    constexpr int GROUPS = kThreads / LPR;
    const int T = f ? f->T : g->T;
    const int blocks = min_int((T + GROUPS - 1) / GROUPS, f ? kForwardBlocks : kGradBlocks);
    const int per = (T + blocks * GROUPS - 1) / (blocks * GROUPS);
    const int grid = (T + GROUPS * per - 1) / (GROUPS * per);
    if (f) {
        SMILE_LAUNCH((rms_norm_kernel<DT, LPR, NP>), dim3(grid), dim3(kThreads), 0, s, *f, per);
    } else {
        SMILE_LAUNCH((rms_norm_backward_kernel<DT, LPR, NP>), dim3(grid), dim3(kThreads), 0, s, *g, per);
        SMILE_LAUNCH(rms_norm_dweight_kernel, dim3((g->d + 15) / 16), dim3(1024), 0, s, (const float *)g->partial, g->dweight, grid, g->d);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t launch_typed(const RmsNormIo *f, const RmsNormGradIo *g, hipStream_t s)
{
    const NormShape n = f ? norm_shape(f->T, f->d) : norm_shape(g->T, g->d);
    if (n.lanes == 16) return launch_shape<DT, 16, 1>(f, g, s);
    if (n.lanes == 32) return launch_shape<DT, 32, 1>(f, g, s);
    if (n.lanes == 64) {
        if (n.pieces == 1) return launch_shape<DT, 64, 1>(f, g, s);
        if (n.pieces == 2) return launch_shape<DT, 64, 2>(f, g, s);
        return launch_shape<DT, 64, 4>(f, g, s);
    }
    if (n.pieces == 1) return launch_shape<DT, kThreads, 1>(f, g, s);
    if (n.pieces == 2) return launch_shape<DT, kThreads, 2>(f, g, s);
    if (n.pieces == 4) return launch_shape<DT, kThreads, 4>(f, g, s);
    return launch_shape<DT, kThreads, 8>(f, g, s);   // 16384 columns, the limit
}

hipError_t launch_any(int dtype, const RmsNormIo *f, const RmsNormGradIo *g, hipStream_t s)
{
    if (dtype == SMILE_DTYPE_BF16) return launch_typed<SMILE_DTYPE_BF16>(f, g, s);
    if (dtype == SMILE_DTYPE_F16) return launch_typed<SMILE_DTYPE_F16>(f, g, s);
    return launch_typed<SMILE_DTYPE_F32>(f, g, s);
}

}  // namespace

hipError_t launch_rms_norm(int dtype, const RmsNormIo &io, hipStream_t s) { return launch_any(dtype, &io, nullptr, s); }

size_t rms_norm_backward_workspace(int T, int d) { return (size_t)min_int(T, kGradBlocks) * d * sizeof(float); }

hipError_t launch_rms_norm_backward(int dtype, const RmsNormGradIo &io, hipStream_t s) { return launch_any(dtype, nullptr, &io, s); }

}  // namespace smile
