// Pre-activations kept in 8 bits for ReLU's backward pass: the codes next to zero, computed again.
//
// Of such a row only the side of zero is read: the derivative is one where the code is positive, else zero.  The matrix cores leave an error of some 1.5e-5
// of a row's typical sum (fp8_gemm.hip), which moves about four elements in a million over that border, and each of them gives
// or takes a whole term of the gradients: with few rows in a group that is a good part of a weight's gradient.  So every code whose magnitude is below
// 2^-5, where the largest is up to 448 (exponent field 0 or 1: three in ten thousand of normally distributed sums, several times the error) is replaced by the code of the sum in 64 bits, where
// the products of codes and their sums are exact for all that matters.  (The error goes by the terms.  Of 25 million sums of 768 none was left on the wrong side
// where they cancel to a tenth of what their terms would give at random, half of one in a million at a twentieth, a tenth of one with channels 30 times the others.)
//
// One wave reads 1024 codes of a row, 16 a lane, and takes the near ones in turn, all lanes along the contraction.  What bounds it are the
// waves that meet several: 3 us each, the latency of two rows and of the sum.  16 groups of 512 rows, 3072 columns, K = 768: 14 us after the
// product's 40; 16 of 32 rows 4.6.  Four rows a wave at a time: the same, and 7.7 us for the small one.
// Sums that are zero exactly count as near ones, since a zero code does not tell them from small ones: columns of zero weights beside others in a block
// of 128 cost a sum each for every row (blocks of zeros alone are passed over).  The whole call, 16 groups of 512 rows: 47 us without such
// columns, 94 with one in each block, 2914 with every other one; 64 groups of 320 rows, 1024 -> 4096: 192, 336, 9563.
#include "fp8_device.hpp"
#include "fp8_internal.hpp"

namespace smile {

namespace {

constexpr int kChunk = 1024;      // codes of a wave
constexpr int kNearBlocks = 2048; // workgroups of four waves: what the chip holds

template <int DT>
__global__ __launch_bounds__(256) void fp8_near_zero_kernel(Fp8Gemm a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, chunk = blockIdx.y;
    const int pitch = (a.Nout + kFp8Block - 1) / kFp8Block * kFp8Block, blocks = pitch / kFp8Block, xpitch = a.KB * kFp8Block;
    const int first = chunk * kChunk + lane * 16;   // of this lane's columns
    const int rows = a.N * a.C;                     // at most 2^27
    for (int row = blockIdx.x * 4 + wave; row < rows; row += gridDim.x * 4) {
        const int e = row / a.C, r = row - e * a.C;
        if (r >= rows_of(a.rows, e, a.C)) continue;
        uint32_t near = 0, byte = 1;
        if (first < pitch) {
            const u32x4 codes = *reinterpret_cast<const u32x4 *>(a.p8 + (size_t)row * pitch + first);
            byte = a.ps[((size_t)e * blocks + first / kFp8Block) * a.Cs + r];
#pragma unroll
            for (int k = 0; k < 16; ++k) near |= (codes[k / 4] >> 8 * (k % 4) & 0x70u) == 0 && first + k < a.Nout ? 1u << k : 0u;
            if (byte <= 1) near = 0;   // a block of zeros, or of what its own scale cannot hold
        }
        for (uint64_t lanes = __ballot(near != 0); lanes; lanes = __ballot(near != 0)) {
            const int owner = __ffsll((unsigned long long)lanes) - 1;
            const int col = chunk * kChunk + owner * 16 + __ffs(__builtin_amdgcn_readlane((int)near, owner)) - 1;
            const uint8_t *x = a.x + (size_t)row * xpitch, *w = a.w + ((size_t)e * a.Nout + col) * xpitch;
            const uint8_t *xs = a.xs + (size_t)e * a.KB * a.Cs + r, *ws = a.ws + (size_t)e * a.KB * a.Ws + col / kFp8Block;
            double sum = 0.0;
            for (int k = lane * 16; k < xpitch; k += kChunk) {
                const u32x4 xc = *reinterpret_cast<const u32x4 *>(x + k), wc = *reinterpret_cast<const u32x4 *>(w + k);
                const int scale = xs[(size_t)(k / kFp8Block) * a.Cs] + ws[(size_t)(k / kFp8Block) * a.Ws] - 254;
                double part = 0.0;
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    float xv[4], wv[4];
                    unpack4(xc[p], 1.f, xv), unpack4(wc[p], 1.f, wv);
#pragma unroll
                    for (int v = 0; v < 4; ++v) part += (double)(xv[v] * wv[v]);
                }
                sum += ldexp(part, scale);
            }
#pragma unroll
            for (int off = 32; off; off /= 2) sum += __shfl_xor(sum, off);
            if (a.bias) sum += (double)(float)static_cast<const typename Piece<DT>::E *>(a.bias)[(size_t)e * a.Nout + col];
            if (lane == owner) {
                a.p8[(size_t)row * pitch + col] = (uint8_t)pack4((float)sum, 0.f, 0.f, 0.f, scale_value(byte));
                near &= near - 1;
            }
        }
    }
}

}  // namespace

hipError_t launch_fp8_near_zero(const Fp8Gemm &a, hipStream_t s)
{
    const int chunks = (a.Nout + kChunk - 1) / kChunk;
    const int groups = (a.N * a.C + 3) / 4;   // N C <= 2^27
    const dim3 grid(std::min(groups, std::max(1, kNearBlocks / chunks)), chunks);
    if (a.dtype == SMILE_DTYPE_F32) SMILE_LAUNCH((fp8_near_zero_kernel<SMILE_DTYPE_F32>), grid, dim3(256), 0, s, a);
    else if (a.dtype == SMILE_DTYPE_F16) SMILE_LAUNCH((fp8_near_zero_kernel<SMILE_DTYPE_F16>), grid, dim3(256), 0, s, a);
    else SMILE_LAUNCH((fp8_near_zero_kernel<SMILE_DTYPE_BF16>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace smile
