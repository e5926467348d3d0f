// 8-bit rows and weights: packing, unpacking, and the dispatch of packed token rows.
//
// All of it streams through HBM once.  Sixteen lanes hold a block of 128 values, eight each, and find its largest magnitude with four DPP
// steps; a workgroup takes sixteen consecutive rows, so that the scale bytes of a block column, which lie row by row, leave it side by side.
#include "fp8_device.hpp"
#include "fp8_internal.hpp"
#include "permute_device.hpp"

namespace smile {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerBlock = kThreads / 16, kBlocksPerLane = 4;   // rows of a workgroup; blocks of 128 columns in flight per lane

template <int DT>
__global__ __launch_bounds__(kThreads) void fp8_pack_rows_kernel(const void *src, const int32_t *rows, uint8_t *codes, uint8_t *scales, int C,
                                                                 int K, int KB, int line)
{
    typedef Piece<DT> P;
    const int e = blockIdx.z, r = blockIdx.x * kRowsPerBlock + threadIdx.x / 16, sub = threadIdx.x % 16;
    if (r >= rows_of(rows, e, C)) return;
    const int kb0 = blockIdx.y * kBlocksPerLane;
    const size_t row = (size_t)e * C + r;
    typename P::Raw raw[kBlocksPerLane];
#pragma unroll
    for (int i = 0; i < kBlocksPerLane; ++i) {
        const int col = (kb0 + i) * kFp8Block + sub * 8;
        if (col < K) raw[i] = P::load(src, row * K + col);
    }
#pragma unroll
    for (int i = 0; i < kBlocksPerLane; ++i) {
        const int kb = kb0 + i, col = kb * kFp8Block + sub * 8;
        if (kb >= KB) break;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (col < K) P::widen(raw[i], v);
        u32x2 c;
        const uint32_t byte = pack_block(v, c);
        *reinterpret_cast<u32x2 *>(codes + row * (KB * kFp8Block) + col) = c;
        if (sub == 0) scales[((size_t)e * KB + kb) * line + r] = (uint8_t)byte;
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void fp8_unpack_rows_kernel(const uint8_t *codes, const uint8_t *scales, const int32_t *rows, void *dst, int C,
                                                                   int K, int KB, int line)
{
    typedef Piece<DT> P;
    const int e = blockIdx.z, r = blockIdx.x * kRowsPerBlock + threadIdx.x / 16, sub = threadIdx.x % 16;
    if (r >= rows_of(rows, e, C)) return;
    const int kb0 = blockIdx.y * kBlocksPerLane;
    const size_t row = (size_t)e * C + r;
    u32x2 c[kBlocksPerLane];
    uint8_t b[kBlocksPerLane];
#pragma unroll
    for (int i = 0; i < kBlocksPerLane; ++i) {
        const int kb = kb0 + i, col = kb * kFp8Block + sub * 8;
        if (col >= K) break;
        c[i] = *reinterpret_cast<const u32x2 *>(codes + row * (KB * kFp8Block) + col);
        b[i] = scales[((size_t)e * KB + kb) * line + r];
    }
#pragma unroll
    for (int i = 0; i < kBlocksPerLane; ++i) {
        const int col = (kb0 + i) * kFp8Block + sub * 8;
        if (col >= K) break;
        float v[8];
        const float s = scale_value(b[i]);
        unpack4(c[i][0], s, v);
        unpack4(c[i][1], s, v + 4);
        if constexpr (DT == SMILE_DTYPE_F16) {   // a finite value stays one: 65504 is kept as 65536
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = fabsf(v[k]) > 65504.f ? copysignf(65504.f, v[k]) : v[k];
        }
        P::store(dst, row * K + col, P::narrow(v));
    }
}

// One 128 x 128 block of a weight matrix a workgroup: 16 lanes a row, rows g, g + 16, ... in eight steps that are all in flight.  The transposed
// form goes through LDS: a thread collects 16 codes of a column.
template <int DT, bool TRANSPOSED>
__global__ __launch_bounds__(kThreads) void fp8_pack_weights_kernel(const void *w, uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t,
                                                                    int Nout, int K)
{
    typedef Piece<DT> P;
    constexpr int PITCH = kFp8Block + 8;
    __shared__ uint32_t largest_of[kThreads / 64];
    __shared__ __attribute__((aligned(16))) uint8_t tile[TRANSPOSED ? kFp8Block * PITCH : 16];
    const int kb = blockIdx.x, nb = blockIdx.y, e = blockIdx.z, KB = gridDim.x, NB = gridDim.y;
    const int g = threadIdx.x / 16, sub = threadIdx.x % 16, col = kb * kFp8Block + sub * 8;
    typename P::Raw raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int o = nb * kFp8Block + i * 16 + g;
        if (o < Nout && col < K) raw[i] = P::load(w, ((size_t)e * Nout + o) * K + col);
    }
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (nb * kFp8Block + i * 16 + g >= Nout || col >= K) continue;
        float v[8];
        P::widen(raw[i], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) largest = max(largest, magnitude_key(v[k]));
    }
    largest = max_of_16(largest);
    largest = max(largest, (uint32_t)__shfl_xor((int)largest, 16, 64));
    largest = max(largest, (uint32_t)__shfl_xor((int)largest, 32, 64));
    if ((threadIdx.x & 63) == 0) largest_of[threadIdx.x >> 6] = largest;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) largest = max(largest, largest_of[i]);
    const uint32_t byte = scale_byte(magnitude_of(largest));
    const float r = scale_value(byte);
    const int lines = (NB + 15) / 16 * 16, lines_t = (KB + 15) / 16 * 16;
    if (threadIdx.x == 0) {
        scales[((size_t)e * KB + kb) * lines + nb] = (uint8_t)byte;
        if (TRANSPOSED) scales_t[((size_t)e * NB + nb) * lines_t + kb] = (uint8_t)byte;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int lo = i * 16 + g, o = nb * kFp8Block + lo;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (o < Nout && col < K) P::widen(raw[i], v);
        u32x2 c;
        c[0] = pack4(v[0], v[1], v[2], v[3], r), c[1] = pack4(v[4], v[5], v[6], v[7], r);
        if (o < Nout) *reinterpret_cast<u32x2 *>(codes + ((size_t)e * Nout + o) * ((size_t)KB * kFp8Block) + col) = c;
        if (TRANSPOSED) *reinterpret_cast<u32x2 *>(tile + lo * PITCH + sub * 8) = c;
    }
    if constexpr (TRANSPOSED) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // eight lanes a row of the transposed form: 128 bytes
            const int q = i * kThreads + threadIdx.x, lk = q / 8, part = q % 8, k = kb * kFp8Block + lk;
            if (k >= K) continue;
            u32x4 out;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t word = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) word |= (uint32_t)tile[(part * 16 + j * 4 + b) * PITCH + lk] << (8 * b);
                out[j] = word;
            }
            *reinterpret_cast<u32x4 *>(codes_t + ((size_t)e * K + k) * ((size_t)NB * kFp8Block) + nb * kFp8Block + part * 16) = out;
        }
    }
}

// The row move of dispatch_kernel for packed rows: ppr pieces of codes, KB scale bytes
template <int LPR>
__global__ __launch_bounds__(kThreads) void fp8_dispatch_kernel(const u32x4 *__restrict__ x8, const uint8_t *__restrict__ xs,
                                                                const int32_t *__restrict__ group_idx, const int32_t *__restrict__ local_idx,
                                                                const int32_t *__restrict__ slot, u32x4 *__restrict__ xe8, uint8_t *__restrict__ xes,
                                                                int T, int ppr, int m, int C, int line_t, int line_c)
{
    const int t = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR, sub = threadIdx.x % LPR;
    if (t >= T) return;
    const int sl = slot[t];
    if (sl < 0 || sl >= C) return;
    const size_t e = group_idx[t] * m + local_idx[t], KB = ppr / 8;
    move_row<LPR>(x8 + (size_t)t * ppr, xe8 + (e * C + sl) * ppr, ppr, sub, [](u32x4 v) { return v; });
    for (int kb = sub; kb < (int)KB; kb += LPR) xes[(e * KB + kb) * line_c + sl] = xs[(size_t)kb * line_t + t];
}

template <int DT>
hipError_t pack_weights_typed(int N, int Nout, int K, const void *w, uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t, hipStream_t s)
{
    const dim3 grid(fp8_blocks(K), fp8_blocks(Nout), N), block(kThreads);
    if (codes_t) SMILE_LAUNCH((fp8_pack_weights_kernel<DT, true>), grid, block, 0, s, w, codes, scales, codes_t, scales_t, Nout, K);
    else SMILE_LAUNCH((fp8_pack_weights_kernel<DT, false>), grid, block, 0, s, w, codes, scales, codes_t, scales_t, Nout, K);
    return hipGetLastError();
}

// (16 rows, kBlocksPerLane blocks, group) workgroups
dim3 rows_grid(const RowsIo &io)
{
    return dim3((io.C + kRowsPerBlock - 1) / kRowsPerBlock, (fp8_blocks(io.K) + kBlocksPerLane - 1) / kBlocksPerLane, io.N);
}

}  // namespace

hipError_t launch_fp8_pack_rows(int dtype, const RowsIo &io, const void *src, uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    const dim3 grid = rows_grid(io), block(kThreads);
    const int KB = fp8_blocks(io.K), line = fp8_scale_pitch(io.C);
    if (dtype == SMILE_DTYPE_BF16) SMILE_LAUNCH((fp8_pack_rows_kernel<SMILE_DTYPE_BF16>), grid, block, 0, s, src, io.rows, codes, scales, io.C, io.K, KB, line);
    else if (dtype == SMILE_DTYPE_F16) SMILE_LAUNCH((fp8_pack_rows_kernel<SMILE_DTYPE_F16>), grid, block, 0, s, src, io.rows, codes, scales, io.C, io.K, KB, line);
    else SMILE_LAUNCH((fp8_pack_rows_kernel<SMILE_DTYPE_F32>), grid, block, 0, s, src, io.rows, codes, scales, io.C, io.K, KB, line);
    return hipGetLastError();
}

hipError_t launch_fp8_unpack_rows(int dtype, const RowsIo &io, const uint8_t *codes, const uint8_t *scales, void *dst, hipStream_t s)
{
    const dim3 grid = rows_grid(io), block(kThreads);
    const int KB = fp8_blocks(io.K), line = fp8_scale_pitch(io.C);
    if (dtype == SMILE_DTYPE_BF16) SMILE_LAUNCH((fp8_unpack_rows_kernel<SMILE_DTYPE_BF16>), grid, block, 0, s, codes, scales, io.rows, dst, io.C, io.K, KB, line);
    else if (dtype == SMILE_DTYPE_F16) SMILE_LAUNCH((fp8_unpack_rows_kernel<SMILE_DTYPE_F16>), grid, block, 0, s, codes, scales, io.rows, dst, io.C, io.K, KB, line);
    else SMILE_LAUNCH((fp8_unpack_rows_kernel<SMILE_DTYPE_F32>), grid, block, 0, s, codes, scales, io.rows, dst, io.C, io.K, KB, line);
    return hipGetLastError();
}

hipError_t launch_fp8_pack_weights(int dtype, int N, int Nout, int K, const void *w, uint8_t *codes, uint8_t *scales, uint8_t *codes_t,
                                   uint8_t *scales_t, hipStream_t s)
{
    if (dtype == SMILE_DTYPE_BF16) return pack_weights_typed<SMILE_DTYPE_BF16>(N, Nout, K, w, codes, scales, codes_t, scales_t, s);
    if (dtype == SMILE_DTYPE_F16) return pack_weights_typed<SMILE_DTYPE_F16>(N, Nout, K, w, codes, scales, codes_t, scales_t, s);
    return pack_weights_typed<SMILE_DTYPE_F32>(N, Nout, K, w, codes, scales, codes_t, scales_t, s);
}

hipError_t launch_fp8_dispatch(const smile_layer_desc &d, const uint8_t *x8, const uint8_t *x_scale, const int32_t *group_idx,
                               const int32_t *local_idx, const int32_t *slot, uint8_t *xe8, uint8_t *xe_scale, hipStream_t s)
{
    const int ppr = fp8_pitch(d.d_model) / 16, lpr = lanes_per_row(ppr);
    const u32x4 *src = reinterpret_cast<const u32x4 *>(x8);
    u32x4 *dst = reinterpret_cast<u32x4 *>(xe8);
    const int line_t = fp8_scale_pitch(d.T), line_c = fp8_scale_pitch(d.capacity);
    const dim3 grid((unsigned)(((long long)d.T + kThreads / lpr - 1) / (kThreads / lpr))), block(kThreads);
    if (lpr == 8) SMILE_LAUNCH(fp8_dispatch_kernel<8>, grid, block, 0, s, src, x_scale, group_idx, local_idx, slot, dst, xe_scale, d.T, ppr, d.m_local, d.capacity, line_t, line_c);
    else if (lpr == 16) SMILE_LAUNCH(fp8_dispatch_kernel<16>, grid, block, 0, s, src, x_scale, group_idx, local_idx, slot, dst, xe_scale, d.T, ppr, d.m_local, d.capacity, line_t, line_c);
    else SMILE_LAUNCH(fp8_dispatch_kernel<32>, grid, block, 0, s, src, x_scale, group_idx, local_idx, slot, dst, xe_scale, d.T, ppr, d.m_local, d.capacity, line_t, line_c);
    return hipGetLastError();
}

}  // namespace smile
