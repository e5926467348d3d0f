// Weight gradient from an operand kept in 8 bits: dw[e][o][k] = sum_r dy[e][r][o] x[e][r][k], dy and dw in bfloat16, x as 8-bit rows.
//
// The scales vary along the contraction, which is over rows, so the 8-bit matrix instructions cannot take them; but a code times its
// scale is a bfloat16, exactly, and the conversion instruction multiplies it in: the operand goes through L2 and LDS in 8 bits and becomes 16 bits in
// registers.  Both operands have the contraction index as their slow index and are read by the transposing LDS reads: four rows at a time of
// dy (ds_read_b64_tr_b16, see gemm_transposed.hip), eight of x (ds_read_b64_tr_b8: of the sixteen 8-byte pieces that the lanes of a group
// address, pieces 2 r and 2 r + 1 are row r, and lane i gets byte i of the eight rows).
//
// A workgroup computes 128 (o) x 256 (k): wave w takes 64 k, so that no code is converted twice, of a single block of 128.  Rows come in slabs of 32
// through four LDS stages, three of them in flight, at one barrier a slab; two workgroups share a CU and hide each other's first slabs and
// epilogue.  Rows beyond the group's count are zeros: the buffer resources end there.
//
// What bounds it: the write of dw (64 groups, 1024 x 4096: 537 MB, 104 us) and the matrix instructions (256 rows each: 114 us at the rate of a large
// product).  Measured 204 us, with one slab of rows only 94 us, without the write 172 us; widening the operand to
// memory and the 16-bit gradient kernels take 238 us in all.  Ordinary stores instead of nontemporal ones: 244 us.  A persistent grid: 223 us.
//
// Operand tiles in LDS: dy [32 rows][16 pieces], the pieces of row r rotated by 4 (r & 3); x [32 rows][16 pieces], rotated by 2 (r & 7): the eight rows of
// a transposing read then cover all banks.
#include "fp8_device.hpp"
#include "fp8_internal.hpp"

namespace smile {

namespace {

constexpr int kTileO = 128, kTileK = 256;   // of the workgroup

__global__ __launch_bounds__(256, 2) void fp8_weight_grad_kernel(Fp8WeightGrad a)
{
#ifdef __HIP_DEVICE_COMPILE__   // (the host has no type for a buffer resource)
    constexpr int kSlab = 32, kStages = 4;   // rows of a slab
    constexpr int DY = kSlab * kTileO * 2, X = kSlab * kTileK, STAGE = DY + X + 4 * 256, SROW = 64 * 2 + 16, LOADS = 5;
    __shared__ __attribute__((aligned(16))) char stages[kStages * STAGE];
    static_assert(2 * sizeof(stages) <= kLdsPerCu && 4 * 32 * SROW <= sizeof(stages), "LDS");
    lds_char *const lds = (lds_char *)stages;
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
    typedef typename Half<__bf16>::vec8 vec8;

    // consecutive tiles of an expert on one XCD
    const int ticket = blockIdx.x % 8 * a.chunk + blockIdx.x / 8;
    if (ticket >= a.tiles) return;
    const int per = a.o_tiles * a.k_tiles, e = ticket / per, kt = ticket % per / a.o_tiles, ot = ticket % a.o_tiles;
    const int o0 = ot * kTileO, k0 = kt * kTileK, pitch = a.KB * kFp8Block, valid = rows_of(a.rows, e, a.C), S = (valid + kSlab - 1) / kSlab;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hi = lane >> 5;

    // ---- loader: two instructions of dy, two of x, one of this wave's scales
    uint32_t dy_off[2], x_off[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int q = (wave + 4 * i) * 64 + lane, r = q / 16;
        dy_off[i] = (uint32_t)r * a.Nout * 2 + ((q - 4 * (r & 3)) & 15) * 16;
        x_off[i] = (uint32_t)r * pitch + ((q - 2 * (r & 7)) & 15) * 16;
    }
    const int block = min(kt * 2 + wave / 2, a.KB - 1);
    const auto resource = [](const void *p, long long bytes) __attribute__((always_inline)) {
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), up = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
        const uint32_t size = __builtin_amdgcn_readfirstlane(bytes <= 0 ? 0u : bytes < 0xffffffffll ? (uint32_t)bytes : 0xffffffffu);
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(((uint64_t)up << 32) | lo), 0, (int)size, 0x00027000);
    };
    const auto request = [&](int s) __attribute__((always_inline)) {
        lds_char *const to = lds + (s & (kStages - 1)) * STAGE;
        const size_t row = (size_t)e * a.C + (size_t)s * kSlab;
        const long long left = (long long)valid - (long long)s * kSlab;   // rows of this slab and all later ones
        const auto dy = resource(a.dy + row * a.Nout + o0, (left * a.Nout - o0) * 2);
        const auto x = resource(a.x + row * pitch + k0, left * pitch - k0);
        const auto xs = resource(a.xs + ((size_t)e * a.KB + block) * a.Cs + (size_t)s * kSlab, (long long)a.Cs - (long long)s * kSlab);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(dy, SMILE_LPTR(to + (wave + 4 * i) * 1024), 16, dy_off[i], 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(x, SMILE_LPTR(to + DY + (wave + 4 * i) * 1024), 16, x_off[i], 0, 0, 0);
        }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(xs, SMILE_LPTR(to + DY + X + wave * 256), 4, (lane & 7) * 4, 0, 0, 0);
    };

    f32x16 acc[2][4];   // [32 k][32 o]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // fragment addressing (see above): row and column of this lane's piece
    const int tj = (lane >> 2) & 3, tcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int xr = 8 * hi + (lane & 15) / 2, xpiece = wave * 4 + ((lane >> 4) & 1);
    const auto multiply = [&](const lds_char *__restrict stage) __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < kSlab / 16; ++kk) {
            vec8 dy[4], x[2];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = j * 32 + tcol;
                read_transposed<4 * 256>(dy[j], stage + (16 * kk + 8 * hi + tj) * 256 + (((col >> 3) + 4 * tj) & 15) * 16 + (col & 4) * 2);
            }
            const u32x2 bytes = *(const lds_u32x2 *)(stage + DY + X + wave * 256 + 16 * kk + 8 * hi);   // scales of the eight rows
            float scale[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) scale[r] = scale_value(min(max(bytes[r / 4] >> 8 * (r % 4) & 255u, 1u), 254u));   // (rows beyond the last: anything)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                typedef int i32x2 __attribute__((ext_vector_type(2)));
                const int piece = (xpiece + 2 * i + 2 * (xr & 7)) & 15;
                const i32x2 codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)(stage + DY + (16 * kk + xr) * 256 + piece * 16 + 8 * (lane & 1)));
                uint32_t w[4];
                // two codes a conversion with one scale: each pair twice, one half of each
                for_constants<4>([&](auto pair) {
                    constexpr int p = decltype(pair)::value;
                    const uint32_t even = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)codes[p / 2], scale[2 * p], p % 2 == 1));
                    const uint32_t odd = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)codes[p / 2], scale[2 * p + 1], p % 2 == 1));
                    w[p] = (even & 0xffffu) | (odd & 0xffff0000u);
                });
                x[i] = __builtin_bit_cast(vec8, u32x4{w[0], w[1], w[2], w[3]});
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = Half<__bf16>::mfma_32x32x16(x[i], dy[j], acc[i][j]);
        }
    };
    // (slabs beyond the last are requested too, as zeros, so that the counts stay the same)
    for_constants<kStages - 1>([&](auto s) { request(decltype(s)::value); });
    for (int s = 0; s < S; ++s) {
        wait_vmcnt<(kStages - 2) * LOADS>();
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): this wave's reads of the stage to be filled
        __builtin_amdgcn_s_barrier();
        request(s + kStages - 1);
        multiply(lds + (s & (kStages - 1)) * STAGE);
    }
    wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();

    // ---- epilogue: element v of a lane is (k 8 (v / 4) + 4 (lane / 32) + v % 4, o lane % 32) of its block; 32 o x 64 k pass through the wave's own
    // piece of LDS and leave as runs of 128 bytes, past the L2: nothing reads them soon
    lds_char *const stg = lds + wave * 32 * SROW;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (o0 + j * 32 >= a.Nout) break;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16 &c = acc[i][j];
                *(lds_u32x2 *)(stg + (lane & 31) * SROW + (i * 32 + 8 * q + 4 * hi) * 2) =
                    u32x2{Half<__bf16>::pack(c[4 * q], c[4 * q + 1]), Half<__bf16>::pack(c[4 * q + 2], c[4 * q + 3])};
            }
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int lo = it * 8 + lane / 8, o = o0 + j * 32 + lo, k = k0 + wave * 64 + lane % 8 * 8;
            const u32x4 v = *(const lds_u32x4 *)(stg + lo * SROW + lane % 8 * 16);
            if (o < a.Nout && k < a.K) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(a.dw + ((size_t)e * a.Nout + o) * a.K + k));
        }
    }
#endif
}

}  // namespace

// The rows of a tile go through one workgroup, one slab after another (0.6 us each), while the 16-bit kernels take smaller tiles or split the rows,
// after a widening that takes at least 8 us.  Measured, this kernel against that (us): 67 tiles of 97 rows 6.8 : 9.4, 128 of 500 15 : 21, 256 of
// 1000 27 : 32, 288 of 1000 34.8 : 34.8, 2600 of 2000 340 : 377; the other way 8 tiles of 500 13.6 : 10.5, 144 of 1000 27 : 25, 216 of 1500 36 : 37,
// 256 of 2000 52 : 47, 256 of 4000 88 : 81, 128 of 8192 164 : 90.
bool fp8_weight_grad_applies(int dtype, int N, int C, int Nout, int K, const Tuning &tune)
{
    const long long tiles = (long long)N * ((Nout + kTileO - 1) / kTileO) * ((K + kTileK - 1) / kTileK);
    return dtype == SMILE_DTYPE_BF16 && (C <= 4 * tiles || tiles >= 2 * tune.cus) && tiles < 1ll << 23;
}

hipError_t launch_fp8_weight_grad(Fp8WeightGrad a, hipStream_t s)
{
    a.o_tiles = (a.Nout + kTileO - 1) / kTileO, a.k_tiles = (a.K + kTileK - 1) / kTileK;
    a.tiles = a.N * a.o_tiles * a.k_tiles, a.chunk = (a.tiles + 7) / 8;
    SMILE_LAUNCH(fp8_weight_grad_kernel, dim3(8 * a.chunk), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace smile
