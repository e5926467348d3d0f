// AdamW over many tensors in one launch, states in 32 bits or in 8; and the values of 8-bit states.
//
// The tensors are cut into chunks of 2048 elements, eight a thread; a list of (tensor, chunk) made on the host lets one launch walk all of them, small
// tensors and large.  A block of 128 elements, which shares a scale in 8-bit states, is 16 neighbouring lanes.  Bound: HBM: each element's parameter,
// master, gradient and moments are read and written once (22 bytes an element with 8-bit states and a 32-bit master of a bfloat16 parameter: 14 of them
// the master and the parameter, 4 the moments); everything a thread loads is requested before the first use.
#include "fp8_device.hpp"
#include "sorted_internal.hpp"

#include <algorithm>

namespace smile {

namespace {

constexpr int kThreads = 256, kEach = kAdamwChunk / kThreads;
static_assert(kEach == 8, "eight elements a thread");

// A 32-bit integer hash: xor-shifts and multiplications
__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}

// 1 - beta^t, t >= 1, in 64 bits
__device__ __forceinline__ double one_minus_power(double beta, uint32_t t)
{
    double p = 1.0;
    for (; t; t >>= 1) {
        if (t & 1) p *= beta;
        beta *= beta;
    }
    return 1.0 - p;
}

// the largest of the 16 lanes of a block
__device__ __forceinline__ float block_max(float v)
{
    auto step = [&](int other) { v = fmaxf(v, __int_as_float(other)); };
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, true));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, true));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true));
    step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true));
    return v;
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.402823466e38f; }

// ---- the first moment: e4m3 codes.  Between two codes of a value's binade lie 2^20 steps of fp32, of which the 16 random bits are the upper ones: adding
// them to the float's bits and cutting off 20 rounds up where the part cut off is at least 1 - R / 65536 of a code's step, and carries into the exponent.
__device__ __forceinline__ uint32_t m_code(float v, int e, uint32_t r)   // e: exponent of the block's power of two
{
    if (!finite(v)) return 0x7fu;
    const float u = __builtin_amdgcn_ldexpf(fabsf(v), -e);
    uint32_t c;
    if (u >= 0.015625f) {                                   // 2^-6, the least normal code
        c = ((__float_as_uint(u) + (r << 4)) >> 20) - ((127u - 7u) << 3);
    } else {
        const float a = u * 512.f, whole = floorf(a);       // steps of 2^-9
        c = (uint32_t)whole + (a - whole >= 1.f - (float)r * (1.f / 65536.f) ? 1u : 0u);
    }
    return c | (__float_as_uint(v) >> 31 << 7);
}
// exponent of the block's power of two: the least with which `largest` is at most 448 = 0.875 * 2^9
__device__ __forceinline__ int m_exponent(float largest)
{
    if (largest == 0.f) return -126;
    const float f = __builtin_amdgcn_frexp_mantf(largest);
    return max(__builtin_amdgcn_frexp_expf(largest) - 9 + (f > 0.875f ? 1 : 0), -126);
}

// ---- the second moment: codes of 5 exponent and 3 fraction bits, code 8 (x + 30) + f for (1 + f / 8) 2^x of the block's power of two
__device__ __forceinline__ uint32_t v_code(float v, int e, uint32_t r)
{
    if (!finite(v)) return 0xffu;
    if (v == 0.f) return 0u;
    const float u = __builtin_amdgcn_ldexpf(v, -e);         // below 2; what is so small that it loses bits here gets the least code
    const int c = (int)((__float_as_uint(u) + (r << 4)) >> 20) - ((127 - 30) << 3);
    return (uint32_t)max(c, 1);
}
__device__ __forceinline__ int v_exponent(float largest)
{
    return largest == 0.f ? -126 : max(__builtin_amdgcn_frexp_expf(largest) - 1, -126);
}
__device__ __forceinline__ float v_value(uint32_t c, int e)
{
    return c == 0 ? 0.f : __builtin_amdgcn_ldexpf(__uint_as_float((c + ((127u - 30u) << 3)) << 20), e);
}

__device__ __forceinline__ void m_values(uint2 codes, int e, float *m)
{
    unpack4(codes.x, 1.f, m), unpack4(codes.y, 1.f, m + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = __builtin_amdgcn_ldexpf(m[i], e);
}
__device__ __forceinline__ void v_values(uint2 codes, int e, float *v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = v_value(codes.x >> 8 * i & 255u, e), v[4 + i] = v_value(codes.y >> 8 * i & 255u, e);
}

// Eight neighbouring elements: all of them in 16-byte pieces, or the first `live`
template <int DT>
__device__ __forceinline__ void load8(const void *base, size_t at, int live, float *v)
{
    if (live >= 8) {
        Piece<DT>::widen(Piece<DT>::load(base, at), v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < live ? (float)static_cast<const typename Piece<DT>::E *>(base)[at + i] : 0.f;
    }
}
template <int DT>
__device__ __forceinline__ void store8(void *base, size_t at, int live, const float *v)
{
    if (live >= 8) {
        Piece<DT>::store(base, at, Piece<DT>::narrow(v));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < live) static_cast<typename Piece<DT>::E *>(base)[at + i] = (typename Piece<DT>::E)v[i];
    }
}

struct AdamwStep {
    int32_t *arrived;               // workgroups that have read the step number
    const AdamwTensor *tensors;
    const AdamwChunk *list;
    const float *lr;
    int32_t *step;
    long long chunks;
    double beta1, beta2;
    float beta1_f, beta2_f, rest1, rest2, eps;   // beta, 1 - beta
    uint32_t seed;
};

template <int DT, int GDT, bool EIGHT, bool MASTER>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwStep a)
{
    AdamwChunk c = a.list[blockIdx.x];
    const float lr = *a.lr;
    const uint32_t t = (uint32_t)*a.step + 1u;
    // All of the workgroup has read the step before thread 0 counts the workgroup, so the last one counted may write the next: one atomic a
    // workgroup, beside its data.
    asm volatile("" ::"v"(t) : "memory");
    __syncthreads();
    if (threadIdx.x == 0 && atomicAdd(a.arrived, 1) == (int)gridDim.x - 1) {
        atomicExch(a.arrived, 0);
        *a.step = (int32_t)t;
    }
    const float inv1 = (float)(1.0 / one_minus_power(a.beta1, t)), inv2 = (float)(1.0 / one_minus_power(a.beta2, t));
    const uint32_t key_step = mix(mix(a.seed) ^ t);
    for (long long n = blockIdx.x; n < a.chunks; n += gridDim.x) {
        if (n != blockIdx.x) c = a.list[n];
        const AdamwTensor &x = a.tensors[c.tensor];
        const size_t at = (size_t)c.chunk * kAdamwChunk + threadIdx.x * 8;
        const long long left = x.n - (long long)at;
        const int live = (int)min(left, 8ll);
        // (8-bit states: the lanes of a block that holds an element stay together, behind the tensor's end too)
        if (EIGHT ? (long long)at >= (x.n + 127) / 128 * 128 : live <= 0) continue;
        float g[8], p[8], m[8], v[8];
        const size_t block = at / 128;
        load8<GDT>(x.grad, at, live, g);
        if constexpr (MASTER) load8<SMILE_DTYPE_F32>(x.master, at, live, p);
        else load8<DT>(x.param, at, live, p);
        if constexpr (EIGHT) {
            const uint2 mc = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(x.m) + at);
            const uint2 vc = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(x.v) + at);
            m_values(mc, (int)x.m_scale[block] - 127, m);
            v_values(vc, (int)x.v_scale[block] - 127, v);
        } else {
            load8<SMILE_DTYPE_F32>(x.m, at, live, m);
            load8<SMILE_DTYPE_F32>(x.v, at, live, v);
        }
        const float decay = x.weight_decay;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = fmaf(a.beta1_f, m[i], a.rest1 * g[i]);
            v[i] = fmaf(a.beta2_f, v[i], a.rest2 * g[i] * g[i]);
            const float update = m[i] * inv1 * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[i] * inv2) + a.eps);
            p[i] -= lr * fmaf(decay, p[i], update);
        }
        store8<DT>(x.param, at, live, p);
        if constexpr (MASTER) store8<SMILE_DTYPE_F32>(x.master, at, live, p);
        if constexpr (!EIGHT) {
            store8<SMILE_DTYPE_F32>(x.m, at, live, m);
            store8<SMILE_DTYPE_F32>(x.v, at, live, v);
        } else {
            float top_m = 0.f, top_v = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= live) m[i] = v[i] = 0.f;
                if (finite(m[i])) top_m = fmaxf(top_m, fabsf(m[i]));
                if (finite(v[i])) top_v = fmaxf(top_v, v[i]);
            }
            const int em = m_exponent(block_max(top_m)), ev = v_exponent(block_max(top_v));
            const uint32_t key = mix(key_step ^ (uint32_t)c.tensor);
            uint32_t mc[2] = {0u, 0u}, vc[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t r = mix((uint32_t)at + i + key);
                mc[i / 4] |= m_code(m[i], em, r & 0xffffu) << 8 * (i % 4);
                vc[i / 4] |= v_code(v[i], ev, r >> 16) << 8 * (i % 4);
            }
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(x.m) + at) = uint2{mc[0], mc[1]};
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(x.v) + at) = uint2{vc[0], vc[1]};
            if ((threadIdx.x & 15) == 0) x.m_scale[block] = (uint8_t)(em + 127), x.v_scale[block] = (uint8_t)(ev + 127);
        }
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void adamw_unpack_kernel(long long n, const uint8_t *m, const uint8_t *m_scale, const uint8_t *v, const uint8_t *v_scale,
                                                                void *m_value, void *v_value)
{
    const long long stride = (long long)gridDim.x * kAdamwChunk;
    for (long long at = ((long long)blockIdx.x * kThreads + threadIdx.x) * 8; at < n; at += stride) {
        float f[8];
        m_values(*reinterpret_cast<const uint2 *>(m + at), (int)m_scale[at / 128] - 127, f);
        store8<DT>(m_value, at, 8, f);
        v_values(*reinterpret_cast<const uint2 *>(v + at), (int)v_scale[at / 128] - 127, f);
        store8<DT>(v_value, at, 8, f);
    }
}

template <int DT, int GDT>
hipError_t launch_typed(const smile_adamw_args &a, const AdamwStep &step, int grid, hipStream_t s)
{
    if constexpr (DT != SMILE_DTYPE_F32) {
        if (a.has_master) {
            if (a.state_bits == 8) SMILE_LAUNCH((adamw_kernel<DT, GDT, true, true>), dim3(grid), dim3(kThreads), 0, s, step);
            else SMILE_LAUNCH((adamw_kernel<DT, GDT, false, true>), dim3(grid), dim3(kThreads), 0, s, step);
            return hipGetLastError();
        }
    }
    if (a.state_bits == 8) SMILE_LAUNCH((adamw_kernel<DT, GDT, true, false>), dim3(grid), dim3(kThreads), 0, s, step);
    else SMILE_LAUNCH((adamw_kernel<DT, GDT, false, false>), dim3(grid), dim3(kThreads), 0, s, step);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(const smile_adamw_args &a, void *plan, const float *lr, int32_t *step, const Tuning &tune, hipStream_t s)
{
    char *base = static_cast<char *>(plan);
    AdamwStep st{};
    st.arrived = reinterpret_cast<int32_t *>(base);
    st.tensors = reinterpret_cast<const AdamwTensor *>(base + kAdamwTensorsAt);
    st.list = reinterpret_cast<const AdamwChunk *>(base + kAdamwTensorsAt + (size_t)a.tensors * sizeof(AdamwTensor));
    st.lr = lr, st.step = step, st.chunks = a.chunks, st.beta1 = a.beta1, st.beta2 = a.beta2, st.seed = (uint32_t)a.seed;
    st.beta1_f = (float)a.beta1, st.beta2_f = (float)a.beta2, st.rest1 = (float)(1.0 - a.beta1), st.rest2 = (float)(1.0 - a.beta2), st.eps = (float)a.eps;
    const int grid = (int)std::min((long long)a.chunks, (long long)workgroup_slots(tune, 8));
    constexpr int F = SMILE_DTYPE_F32, B = SMILE_DTYPE_BF16, H = SMILE_DTYPE_F16;
    if (a.dtype == F) return launch_typed<F, F>(a, st, grid, s);
    if (a.dtype == B) return a.grad_dtype == F ? launch_typed<B, F>(a, st, grid, s) : launch_typed<B, B>(a, st, grid, s);
    return a.grad_dtype == F ? launch_typed<H, F>(a, st, grid, s) : launch_typed<H, H>(a, st, grid, s);
}

hipError_t launch_adamw_unpack(int dtype, long long n, const uint8_t *m, const uint8_t *m_scale, const uint8_t *v, const uint8_t *v_scale, void *m_value,
                               void *v_value, hipStream_t s)
{
    const int grid = (int)std::min((n + kAdamwChunk - 1) / kAdamwChunk, 4096ll);
    if (dtype == SMILE_DTYPE_F32) SMILE_LAUNCH(adamw_unpack_kernel<SMILE_DTYPE_F32>, dim3(grid), dim3(kThreads), 0, s, n, m, m_scale, v, v_scale, m_value, v_value);
    else SMILE_LAUNCH(adamw_unpack_kernel<SMILE_DTYPE_BF16>, dim3(grid), dim3(kThreads), 0, s, n, m, m_scale, v, v_scale, m_value, v_value);
    return hipGetLastError();
}

}  // namespace smile
