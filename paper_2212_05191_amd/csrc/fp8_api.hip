// C-ABI entry points of the 8-bit operators: argument checks, all of them on the host before anything is enqueued.
#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>

#include "api_checks.hpp"
#include "fp8_device.hpp"
#include "fp8_internal.hpp"

namespace smile {

namespace {

constexpr int kWidest = 32768, kWidestNorm = 16384;
constexpr long long kMostRows = 1ll << 27;          // (32 lanes a row, 2^32 threads a launch)
constexpr double kMostElements = 1099511627776.0;   // 2^40

bool known(int dtype) { return dtype == SMILE_DTYPE_F32 || dtype == SMILE_DTYPE_BF16 || dtype == SMILE_DTYPE_F16; }

// N groups of C rows of `width` columns
smile_status check_rows(int N, int C, int width, int dtype)
{
    if (!known(dtype)) return SMILE_UNSUPPORTED;
    if (N < 1 || C < 1 || width < 8 || width % 8 || width > kWidest || N > 4096) return SMILE_BAD_SHAPE;
    if ((long long)N * C > kMostRows || (double)N * C * fp8_pitch(width) >= kMostElements) return SMILE_BAD_SHAPE;
    if ((long long)fp8_blocks(width) * fp8_scale_pitch(C) >= 1ll << 31) return SMILE_BAD_SHAPE;   // the scales of a group, in 32 bits
    return SMILE_OK;
}

smile_status check_norm(int T, int d, int dtype)
{
    const smile_status st = check_rows(1, T, d, dtype);
    return st != SMILE_OK ? st : d > kWidestNorm ? SMILE_BAD_SHAPE : SMILE_OK;
}

// The compute units of the current device, asked for once per device
Tuning device_tuning()
{
    constexpr int kDevices = 64;
    static std::atomic<int> known_cus[kDevices];
    Tuning t;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kDevices) {
        (void)hipGetLastError();
        return t;
    }
    int cus = known_cus[dev].load(std::memory_order_relaxed);
    if (cus == 0) {
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) {
            (void)hipGetLastError();
            return t;
        }
        known_cus[dev].store(cus, std::memory_order_relaxed);
    }
    t.cus = cus;
    return t;
}

size_t weight_grad_workspace(int N, int C, int K, int dtype) { return align_up((size_t)N * C * K * elem_size(dtype), 256); }

}  // namespace

}  // namespace smile

using namespace smile;

extern "C" {

int32_t smile_fp8_pitch(int32_t K) { return K < 1 || K > INT_MAX - kFp8Block ? -1 : fp8_pitch(K); }

int32_t smile_fp8_scale_pitch(int32_t rows) { return rows < 1 || rows > INT_MAX - 16 ? -1 : fp8_scale_pitch(rows); }

smile_status smile_rms_norm(int32_t T, int32_t d, int32_t dtype, const void *x, const void *residual, const void *weight,
                            float eps, void *sum, void *y, void *y8, void *y8_scale, float *rstd, void *stream)
{
    if (bad(x) || bad_opt(residual) || bad(weight) || bad_opt(sum) || bad_opt(y) || bad_opt(y8) || bad_opt(y8_scale) || bad_opt(rstd))
        return SMILE_INVALID_ARG;
    if ((y8 == nullptr) != (y8_scale == nullptr) || (!y && !y8) || (sum && !residual)) return SMILE_INVALID_ARG;
    const smile_status st = check_norm(T, d, dtype);
    if (st != SMILE_OK) return st;
    if (!(eps > 0.f) || !std::isfinite(eps)) return SMILE_BAD_SHAPE;
    return from_hip(launch_rms_norm(dtype, RmsNormIo{x, residual, weight, sum, y, static_cast<uint8_t *>(y8), static_cast<uint8_t *>(y8_scale), rstd, T, d, eps},
                                    static_cast<hipStream_t>(stream)));
}

smile_status smile_rms_norm_backward_workspace_bytes(int32_t T, int32_t d, size_t *bytes)
{
    if (!bytes) return SMILE_INVALID_ARG;
    const smile_status st = check_norm(T, d, SMILE_DTYPE_F32);
    if (st != SMILE_OK) return st;
    *bytes = rms_norm_backward_workspace(T, d);
    return SMILE_OK;
}

smile_status smile_rms_norm_backward(int32_t T, int32_t d, int32_t dtype, const void *dy, const void *dsum, const void *s,
                                     const void *weight, const float *rstd, void *ds, float *dweight, void *workspace,
                                     size_t workspace_bytes, void *stream)
{
    if (bad(dy) || bad_opt(dsum) || bad(s) || bad(weight) || bad(rstd) || bad(ds) || bad(dweight) || !workspace) return SMILE_INVALID_ARG;
    const smile_status st = check_norm(T, d, dtype);
    if (st != SMILE_OK) return st;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < rms_norm_backward_workspace(T, d)) return SMILE_WORKSPACE;
    return from_hip(launch_rms_norm_backward(dtype, RmsNormGradIo{dy, dsum, s, weight, rstd, ds, dweight, static_cast<float *>(workspace), T, d},
                                             static_cast<hipStream_t>(stream)));
}

smile_status smile_fp8_pack_rows(int32_t N, int32_t C, int32_t K, int32_t dtype, const void *src, const int32_t *rows,
                                 void *codes, void *scales, void *stream)
{
    if (bad(src) || bad_opt(rows) || bad(codes) || bad(scales)) return SMILE_INVALID_ARG;
    const smile_status st = check_rows(N, C, K, dtype);
    if (st != SMILE_OK) return st;
    return from_hip(launch_fp8_pack_rows(dtype, RowsIo{N, C, K, rows}, src, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales),
                                         static_cast<hipStream_t>(stream)));
}

smile_status smile_fp8_unpack_rows(int32_t N, int32_t C, int32_t K, int32_t dtype, const void *codes, const void *scales,
                                   const int32_t *rows, void *dst, void *stream)
{
    if (bad(codes) || bad(scales) || bad_opt(rows) || bad(dst)) return SMILE_INVALID_ARG;
    const smile_status st = check_rows(N, C, K, dtype);
    if (st != SMILE_OK) return st;
    return from_hip(launch_fp8_unpack_rows(dtype, RowsIo{N, C, K, rows}, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), dst,
                                           static_cast<hipStream_t>(stream)));
}

smile_status smile_fp8_pack_weights(int32_t N, int32_t Nout, int32_t K, int32_t dtype, const void *w, void *codes, void *scales,
                                    void *codes_t, void *scales_t, void *stream)
{
    if (bad(w) || bad(codes) || bad(scales) || bad_opt(codes_t) || bad_opt(scales_t) || (codes_t == nullptr) != (scales_t == nullptr))
        return SMILE_INVALID_ARG;
    smile_status st = check_rows(N, Nout, K, dtype);
    if (st == SMILE_OK) st = check_rows(N, K, Nout, dtype);
    if (st != SMILE_OK) return st;
    return from_hip(launch_fp8_pack_weights(dtype, N, Nout, K, w, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales),
                                            static_cast<uint8_t *>(codes_t), static_cast<uint8_t *>(scales_t), static_cast<hipStream_t>(stream)));
}

smile_status smile_fp8_dispatch(smile_ctx *ctx, const void *x8, const void *x_scale, const int32_t *group_idx,
                                const int32_t *local_idx, const int32_t *slot, void *xe8, void *xe_scale, void *stream)
{
    if (!ctx || bad(x8) || bad(x_scale) || bad(group_idx) || bad(local_idx) || bad(slot) || bad(xe8) || bad(xe_scale)) return SMILE_INVALID_ARG;
    const smile_layer_desc &d = ctx->desc;
    smile_status st = check_rows(1, d.T, d.d_model, d.dtype);
    if (st == SMILE_OK) st = check_rows(d.n_groups * d.m_local, d.capacity, d.d_model, d.dtype);
    if (st != SMILE_OK) return st;
    return from_hip(launch_fp8_dispatch(d, static_cast<const uint8_t *>(x8), static_cast<const uint8_t *>(x_scale), group_idx, local_idx, slot,
                                        static_cast<uint8_t *>(xe8), static_cast<uint8_t *>(xe_scale), static_cast<hipStream_t>(stream)));
}

smile_status smile_fp8_gemm(const smile_fp8_gemm_args *p, void *stream)
{
    if (!p) return SMILE_INVALID_ARG;
    const smile_fp8_gemm_args &a = *p;
    if (bad(a.x8) || bad(a.x_scale) || bad(a.w8) || bad(a.w_scale) || bad_opt(a.bias) || bad_opt(a.rows) || bad_opt(a.y) || bad_opt(a.y8) ||
        bad_opt(a.y_scale) || bad_opt(a.pre8) || bad_opt(a.pre_scale) || bad_opt(a.grad8) || bad_opt(a.grad_scale))
        return SMILE_INVALID_ARG;
    if ((a.y8 == nullptr) != (a.y_scale == nullptr) || (a.pre8 == nullptr) != (a.pre_scale == nullptr) ||
        (a.grad8 == nullptr) != (a.grad_scale == nullptr) || (!a.y && !a.y8) || (a.grad8 && (a.bias || a.pre8)))
        return SMILE_INVALID_ARG;
    if (a.act != SMILE_ACT_NONE && a.act != SMILE_ACT_RELU && a.act != SMILE_ACT_GELU) return SMILE_UNSUPPORTED;
    if (a.grad8 && a.act == SMILE_ACT_NONE) return SMILE_UNSUPPORTED;
    smile_status st = check_rows(a.N, a.C, a.K, a.dtype);
    if (st == SMILE_OK) st = check_rows(a.N, a.C, a.Nout, a.dtype);
    if (st == SMILE_OK) st = check_rows(a.N, a.Nout, a.K, a.dtype);
    if (st != SMILE_OK) return st;
    Fp8Gemm g{};
    g.x = static_cast<const uint8_t *>(a.x8), g.xs = static_cast<const uint8_t *>(a.x_scale);
    g.w = static_cast<const uint8_t *>(a.w8), g.ws = static_cast<const uint8_t *>(a.w_scale);
    g.bias = a.bias, g.rows = a.rows, g.y = a.y;
    g.y8 = static_cast<uint8_t *>(a.y8), g.ys = static_cast<uint8_t *>(a.y_scale);
    g.p8 = static_cast<uint8_t *>(a.pre8), g.ps = static_cast<uint8_t *>(a.pre_scale);
    g.g8 = static_cast<const uint8_t *>(a.grad8), g.gs = static_cast<const uint8_t *>(a.grad_scale);
    g.N = a.N, g.C = a.C, g.Nout = a.Nout, g.KB = fp8_blocks(a.K);
    g.Cs = fp8_scale_pitch(a.C), g.Ws = fp8_scale_pitch(fp8_blocks(a.Nout));
    g.dtype = a.dtype, g.act = a.act == SMILE_ACT_NONE ? 0 : a.act == SMILE_ACT_RELU ? 1 : 3;
    hipError_t err = launch_fp8_gemm(g, device_tuning(), static_cast<hipStream_t>(stream));
    if (err == hipSuccess && g.p8 && g.act == 1) err = launch_fp8_near_zero(g, static_cast<hipStream_t>(stream));
    return from_hip(err);
}

smile_status smile_fp8_weight_grad_workspace_bytes(int32_t N, int32_t C, int32_t K, int32_t dtype, size_t *bytes)
{
    if (!bytes) return SMILE_INVALID_ARG;
    const smile_status st = check_rows(N, C, K, dtype);
    if (st != SMILE_OK) return st;
    *bytes = weight_grad_workspace(N, C, K, dtype);
    return SMILE_OK;
}

smile_status smile_fp8_weight_grad(int32_t N, int32_t C, int32_t Nout, int32_t K, int32_t dtype, const void *dy, const void *x8,
                                   const void *x_scale, const int32_t *rows, void *dw, void *workspace, size_t workspace_bytes,
                                   void *stream)
{
    if (bad(dy) || bad(x8) || bad(x_scale) || bad_opt(rows) || bad(dw) || !workspace) return SMILE_INVALID_ARG;
    smile_status st = check_rows(N, C, K, dtype);
    if (st == SMILE_OK) st = check_rows(N, C, Nout, dtype);
    if (st == SMILE_OK) st = check_rows(N, Nout, K, dtype);
    if (st == SMILE_OK && is_half(dtype) && (K % 64 || Nout % 64)) st = SMILE_BAD_SHAPE;
    if (st != SMILE_OK) return st;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < weight_grad_workspace(N, C, K, dtype)) return SMILE_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Tuning tune = device_tuning();
    if (fp8_weight_grad_applies(dtype, N, C, Nout, K, tune)) {
        Fp8WeightGrad g{};
        g.dy = static_cast<const uint16_t *>(dy), g.x = static_cast<const uint8_t *>(x8), g.xs = static_cast<const uint8_t *>(x_scale);
        g.rows = rows, g.dw = static_cast<uint16_t *>(dw), g.N = N, g.C = C, g.Nout = Nout, g.K = K, g.KB = fp8_blocks(K), g.Cs = fp8_scale_pitch(C);
        return from_hip(launch_fp8_weight_grad(g, s));
    }
    // Half precision, which does not hold every product of a code and a scale, fp32, and few tiles: the operand is widened and multiplied by the gradient
    // kernels of the expert FFN.
    hipError_t err = launch_fp8_unpack_rows(dtype, RowsIo{N, C, K, rows}, static_cast<const uint8_t *>(x8), static_cast<const uint8_t *>(x_scale), workspace, s);
    if (err != hipSuccess) return from_hip(err);
    // Row counts that the device knows alone: the rules of the gradient kernels, which go by the rows expected, are given four fifths of the buffers
    // (capacity factor 1.25).  Half precision, 64 groups of 256 rows, 1024 x 4096: buffers of 320 252 -> 241 us; of 256 and of 512 rows the same either way (226,
    // 267), as are 16 groups of 512 rows in 512 or 640, 15 of 334 in 417 and 128 of 20 in 26.
    const int tokens = rows ? (int)std::max(1ll, (long long)N * C * 4 / 5) : 0;
    const long long sx = (long long)C * Nout, sw = (long long)C * K, sy = (long long)Nout * K;
    if (is_half(dtype)) {
        TransposedGemm g{};
        g.x = dy, g.w = workspace, g.y = dw, g.k_valid = rows, g.N = N, g.Mrows = Nout, g.Nout = K, g.K = C, g.ldx = Nout, g.ldw = K;
        g.sx = sx, g.sw = sw, g.sy = sy, g.x_transposed = g.w_transposed = true, g.tune = tune, g.tokens = tokens;
        return from_hip(launch_grouped_gemm_t(dtype, g, s));
    }
    F32Gemm g{};
    g.x = dy, g.w = workspace, g.y = dw, g.k_valid = rows, g.N = N, g.Mrows = Nout, g.Nout = K, g.K = C, g.ldx = Nout, g.ldw = K;
    g.sx = sx, g.sw = sw, g.sy = sy, g.x_transposed = g.w_transposed = true, g.tune = tune;
    return from_hip(launch_grouped_gemm_f32(g, s));
}

}  // extern "C"
