// Weight gradient from an operand kept in 8 bits: dw[e][o][k] = sum_r dy[e][r][o] x[e][r][k], dy and dw in bfloat16, x as 8-bit rows.
//
// The scales vary along the contraction, which is over rows, so the 8-bit matrix instructions cannot take them; but a code times its
// scale is a bfloat16, exactly, and the conversion instruction multiplies it in: the operand goes through L2 and LDS in 8 bits and becomes 16 bits in
// registers.  Both operands have the contraction index as their slow index and are read by the transposing LDS reads, four rows at a time
// (ds_read_b64_tr_b16, see gemm_transposed.hip), the codes in pairs of columns: the conversion takes a pair with one scale, and two byte
// permutations sort two rows' pairs into the even and the odd column, which are operands of two matrix instructions.
//
// A workgroup computes 128 (o) x 256 (k): wave w takes 64 k, so that no code is converted twice, of a single block of 128.  Rows come in slabs of 32
// through three LDS stages, two of them in flight, at one barrier a slab; three workgroups share a CU and hide each other's first slabs and
// epilogue (168 registers: 128 of sums, and the order of the reads held to two operands at a time).  Rows beyond the
// group's count are zeros: the buffer resources end there.
//
// What bounds it: the write of dw (64 groups, 1024 x 4096: 537 MB, 104 us) and the matrix instructions (256 rows each: 114 us at the rate of a large
// product).  Measured 173 us; two workgroups with four stages 192, codes converted column by column 195, scales taken out of their word by more
// than one shift 179 (and sums over 6000 rows, 8 x 1600 x 6400, 1019, 1001, 939 where it is 894 now, 1.10 PFLOP/s); ordinary instead of nontemporal stores
// 40 us more; a persistent grid 20 us more.  Widening the operand to memory and the 16-bit gradient kernels take 238 us in all.
//
// Operand tiles in LDS: 32 rows of 16 pieces of 16 bytes, the pieces of row r rotated by 4 (r & 3): the four rows of a transposing read cover all banks.
#include "fp8_device.hpp"
#include "fp8_internal.hpp"

namespace smile {

namespace {

constexpr int kTileO = 128, kTileK = 256;   // of the workgroup

__global__ __launch_bounds__(256, 3) void fp8_weight_grad_kernel(Fp8WeightGrad a)
{
#ifdef __HIP_DEVICE_COMPILE__   // (the host has no type for a buffer resource)
    constexpr int kSlab = 32, kStages = 3;   // rows of a slab
    constexpr int DY = kSlab * kTileO * 2, X = kSlab * kTileK, STAGE = DY + X + 4 * 256, SROW = 64 * 2 + 16, LOADS = 5;
    __shared__ __attribute__((aligned(16))) char stages[kStages * STAGE];
    static_assert(3 * sizeof(stages) <= kLdsPerCu && 4 * 32 * SROW <= sizeof(stages), "LDS");
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
    const int lr = (wave * 64 + lane) / 16, lp = (lane - 4 * (lr & 3)) & 15;   // row and piece; the second instruction: sixteen rows on
    const uint32_t dy_off = (uint32_t)lr * a.Nout * 2 + lp * 16, x_off = (uint32_t)lr * pitch + lp * 16;
    const int block = min(kt * 2 + wave / 2, a.KB - 1);
    const auto resource = [](const void *p, long long bytes) __attribute__((always_inline)) {
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), up = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
        const uint32_t size = __builtin_amdgcn_readfirstlane(bytes <= 0 ? 0u : bytes < 0xffffffffll ? (uint32_t)bytes : 0xffffffffu);
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(((uint64_t)up << 32) | lo), 0, (int)size, 0x00027000);
    };
    const auto request = [&](int s, lds_char *to) __attribute__((always_inline)) {
        const size_t row = (size_t)e * a.C + (size_t)s * kSlab;
        const long long left = (long long)valid - (long long)s * kSlab;   // rows of this slab and all later ones
        const auto dy = resource(a.dy + row * a.Nout + o0, (left * a.Nout - o0) * 2);
        const auto x = resource(a.x + row * pitch + k0, left * pitch - k0);
        const auto xs = resource(a.xs + ((size_t)e * a.KB + block) * a.Cs + (size_t)s * kSlab, (long long)a.Cs - (long long)s * kSlab);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(dy, SMILE_LPTR(to + (wave + 4 * i) * 1024), 16, dy_off + 32u * i * a.Nout, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(x, SMILE_LPTR(to + DY + (wave + 4 * i) * 1024), 16, x_off + 16u * i * pitch, 0, 0, 0);
        }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(xs, SMILE_LPTR(to + DY + X + wave * 256), 4, (lane & 7) * 4, 0, 0, 0);
    };

    f32x16 acc[2][4];   // [even k, odd k][32 o]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // fragment addressing (see above): row and column of this lane's piece
    const int tj = (lane >> 2) & 3, tcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int piece0 = (8 * hi + tj) * 256 + (tcol >> 3) * 16 + (tcol & 4) * 2;
    const auto multiply = [&](const lds_char *__restrict stage) __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < kSlab / 16; ++kk) {
            vec8 x[2];
            {
                const u32x2 bytes = *(const lds_u32x2 *)(stage + DY + X + wave * 256 + 16 * kk + 8 * hi);   // scales of the eight rows
                vec8 pairs;
                read_transposed<4 * 256>(pairs, stage + DY + 16 * kk * 256 + piece0 + ((wave + tj) & 3) * 64);
                const u32x4 codes = __builtin_bit_cast(u32x4, pairs);
                u32x4 even, odd;   // columns
                for_constants<4>([&](auto pair) {
                    constexpr int p = decltype(pair)::value;
                    // (the conversion reads a scale's exponent alone: what else of the word is shifted along does not matter)
                    const auto scale = [&](int r) __attribute__((always_inline)) { return __uint_as_float(r % 4 < 3 ? bytes[r / 4] << (23 - 8 * (r % 4)) : bytes[r / 4] >> 1); };
                    const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[p], scale(2 * p), false));
                    const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[p], scale(2 * p + 1), true));
                    even[p] = __builtin_amdgcn_perm(b, a, 0x05040100u), odd[p] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                });
                x[0] = __builtin_bit_cast(vec8, even), x[1] = __builtin_bit_cast(vec8, odd);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
                vec8 dy[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) read_transposed<4 * 256>(dy[j], stage + 16 * kk * 256 + piece0 + ((2 * jj + j + tj) & 3) * 64);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) acc[i][2 * jj + j] = Half<__bf16>::mfma_32x32x16(x[i], dy[j], acc[i][2 * jj + j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // (slabs beyond the last are requested too, as zeros, so that the counts stay the same)
    for_constants<kStages - 1>([&](auto s) { request(decltype(s)::value, lds + decltype(s)::value * STAGE); });
    lds_char *at = lds, *fill = lds + (kStages - 1) * STAGE;
    for (int s = 0; s < S; ++s) {
        wait_vmcnt<(kStages - 2) * LOADS>();
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): this wave's reads of the stage to be filled
        __builtin_amdgcn_s_barrier();
        request(s + kStages - 1, fill);
        // the scales of rows beyond the last are anything: beside codes of zero, one that counts as NaN would not do
        if (s == S - 1 && lane < kSlab && lane >= valid - s * kSlab) *(at + DY + X + wave * 256 + lane) = 127;
        multiply(at);
        fill = at, at = at == lds + (kStages - 1) * STAGE ? lds : at + STAGE;
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
        for (int q = 0; q < 4; ++q) {
            const f32x16 &c = acc[0][j], &d = acc[1][j];
            u32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = Half<__bf16>::pack(c[4 * q + k], d[4 * q + k]);
            *(lds_u32x4 *)(stg + (lane & 31) * SROW + (16 * q + 8 * hi) * 2) = v;
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
// after a widening that takes at least 8 us.  Measured, this kernel against that (us): 67 tiles of 97 rows 7 : 9, 128 of 500 16 : 21, 288 of 1000
// 33 : 35, 576 of 512 42 : 62, 8192 of 256 173 : 238; the other way 8 tiles of 500 14.6 : 10.9, 144 of 1000 27 : 26, 256 of 2000 50 : 47, 256 of
// 4000 89 : 83, 128 of 8192 164 : 90.  From two tiles a CU on, long rows too: 1024 tiles of 3000 rows 193 : 262, of 6000 366 : 500, 1300 of 8192 655 : 730,
// 1440 of 2048 177 : 268, 1536 of 4096 380 : 565.
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
