// AdamW over many tensors in one launch, states in 32 bits or in 8; and the values of 8-bit states.
//
// The tensors are cut into chunks of 2048 elements, eight a thread; a list of (tensor, chunk) made on the host lets one launch walk all of them, small
// tensors and large.  A block of 128 elements, which shares a scale in 8-bit states, is 16 neighbouring lanes.  Bound: HBM: each element's master (or
// parameter), gradient and moments are read once, master, parameter and moments written once.  16 bytes an element with 8-bit states, a 32-bit master and a bfloat16
// gradient: 10 of them the master and the parameter, 4 the moments, 2 the gradient; 134 M elements 472 us, 4.6 TB/s.  32-bit states: 28 bytes, 810 us, 4.6 TB/s.  Everything a
// thread loads is requested before the first use.
#include "fp8_device.hpp"
#include "sorted_internal.hpp"

#include <algorithm>
#include <type_traits>

namespace smile {

namespace {

constexpr int kThreads = 256, kEach = kAdamwChunk / kThreads;
// Workgroups on a CU, all resident: a thread has one chunk's loads in flight, so their number is what covers the memory's latency.  134 M elements with 8-bit states and
// master weights, without and with the codes past the L2: five (88 registers) 554 / 532 us, six 514 / 490, seven (72 registers) 467 (472 since roots reach below the normal range), eight
// spill 535.
constexpr int kPerCu = 7;
static_assert(kEach == 8, "eight elements a thread");

// A 32-bit integer hash: xor-shifts and multiplications.  The shifts and both multipliers are those that Chris Wellons published in 2018, found by a search for the least
// bias: a table, so that whoever computes the bits elsewhere gets the same.
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
__device__ __forceinline__ uint32_t block_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));
}

constexpr uint32_t kInfinity = 0x7f800000u;   // magnitudes from here on are not finite

// ---- the first moment: e4m3 codes.  Between two codes of a value's binade lie 2^20 steps of fp32, of which the 16 random bits are the upper ones: adding
// them to the float's bits and cutting off 20 rounds up where the part cut off is at least 1 - R / 65536 of a code's step, and carries into the exponent.  Below 2^-6 the
// codes are 2^-9 apart: the same in units of 2^-25.  v finite.
__device__ __forceinline__ uint32_t m_code(float v, int e, uint32_t r)   // e: exponent of the block's power of two
{
    const float u = __builtin_amdgcn_ldexpf(fabsf(v), -e);
    const uint32_t normal = ((__float_as_uint(u) + (r << 4)) >> 20) - ((127u - 7u) << 3), small = ((uint32_t)(u * 33554432.f) + r) >> 16;
    return (u >= 0.015625f ? normal : small) | (__float_as_uint(v) >> 24 & 0x80u);
}
// exponent of the block's power of two: the least with which `largest` is at most 448 = 0.875 * 2^9
__device__ __forceinline__ int m_exponent(float largest)
{
    if (largest == 0.f) return -126;
    const float f = __builtin_amdgcn_frexp_mantf(largest);
    return max(__builtin_amdgcn_frexp_expf(largest) - 9 + (f > 0.875f ? 1 : 0), -126);
}

// ---- the second moment: codes of 5 exponent and 3 fraction bits, code 8 (x + 30) + f for (1 + f / 8) 2^x of the block's power of two, at most 248 (its
// double); 255 is infinity.  v finite.
__device__ __forceinline__ uint32_t v_code(float v, int e, uint32_t r)
{
    const float u = __builtin_amdgcn_ldexpf(v, -e);         // below 2; what is so small that it loses bits here gets the least code
    const int c = (int)((__float_as_uint(u) + (r << 4)) >> 20) - ((127 - 30) << 3);
    return v == 0.f ? 0u : (uint32_t)max(c, 1);
}
__device__ __forceinline__ int v_exponent(float largest)
{
    return largest == 0.f ? -126 : max(__builtin_amdgcn_frexp_expf(largest) - 1, -126);
}

// values of eight codes, before the block's power of two; and after
__device__ __forceinline__ void m_units(uint2 codes, float *m) { unpack4(codes.x, 1.f, m), unpack4(codes.y, 1.f, m + 4); }
// (infinity: the square of a finite gradient may be that, and its m is not.  Were v as small as its neighbours from the next step on, m would be divided by almost nothing.)
__device__ __forceinline__ float v_unit(uint32_t c) { return __uint_as_float(c - 1u < 248u ? (c + ((127u - 30u) << 3)) << 20 : c << 23); }   // 255 << 23: infinity
__device__ __forceinline__ void v_units(uint2 codes, float *v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = v_unit(codes.x >> 8 * i & 255u), v[4 + i] = v_unit(codes.y >> 8 * i & 255u);
}
__device__ __forceinline__ void scaled(float *v, int e)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_ldexpf(v[i], e);
}

// the first `live` of eight neighbouring elements, zeros behind them
template <int DT>
__device__ __forceinline__ void load_some(const void *base, size_t at, int live, float *v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < live ? (float)static_cast<const typename Piece<DT>::E *>(base)[at + i] : 0.f;
}
template <int DT>
__device__ __forceinline__ void store8(void *base, size_t at, int live, const float *v)
{
    if (live >= 8) {
        // not read again by this launch: past the L2 (134 M elements, 8-bit states: 568 -> 545 us)
        const auto r = Piece<DT>::narrow(v);
        u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<typename Piece<DT>::E *>(base) + at);
        __builtin_nontemporal_store(r.a, p);
        if constexpr (DT == SMILE_DTYPE_F32) __builtin_nontemporal_store(r.b, p + 1);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < live) static_cast<typename Piece<DT>::E *>(base)[at + i] = (typename Piece<DT>::E)v[i];
    }
}

__device__ __forceinline__ void store_codes(void *base, size_t at, const uint32_t (&c)[2])
{
    __builtin_nontemporal_store((uint64_t)c[1] << 32 | c[0], reinterpret_cast<uint64_t *>(static_cast<uint8_t *>(base) + at));
}

// The root's instruction takes what lies below the normal range as 0: such values are scaled by 2^64 on the way.
__device__ __forceinline__ float root(float x)
{
    const bool small = x < 1.17549435e-38f;
    const float r = __builtin_amdgcn_sqrtf(__builtin_amdgcn_ldexpf(x, small ? 64 : 0));
    return small ? r * 2.32830644e-10f : r;
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

// The moments' next values, every product and sum rounded by itself in the order that the formulas have: a state in 8 bits is rounded at random, and what decides it
// should not depend on how a compiler contracts them.
__device__ __forceinline__ void moments(const AdamwStep &a, float g, float &m, float &v)
{
#pragma clang fp contract(off)
    m = a.beta1_f * m + a.rest1 * g;
    v = fmaxf(a.beta2_f * v, 0.f) + a.rest2 * g * g;   // (0 times infinity, of a v that overflowed, is NaN, and the larger of NaN and 0 is 0)
}

template <int DT, int GDT, bool EIGHT, bool MASTER>
__global__ __launch_bounds__(kThreads, kPerCu) void adamw_kernel(AdamwStep a)
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
    const uint32_t key_step = mix(mix(a.seed) ^ t);
    // one chunk's loads are in flight while the one before is computed and stored
    struct Raw {
        typename Piece<GDT>::Raw g;
        typename Piece<MASTER ? SMILE_DTYPE_F32 : DT>::Raw p;
        typename std::conditional_t<EIGHT, uint2, typename Piece<SMILE_DTYPE_F32>::Raw> m, v;
        uint8_t m_scale, v_scale;
    };
    auto fetch = [&](AdamwChunk c, Raw &r) {
        const AdamwTensor &x = a.tensors[c.tensor];
        const size_t at = (size_t)c.chunk * kAdamwChunk + threadIdx.x * 8;
        if ((long long)at + 8 <= x.n) {
            r.g = Piece<GDT>::load(x.grad, at);
            r.p = Piece<MASTER ? SMILE_DTYPE_F32 : DT>::load(MASTER ? x.master : x.param, at);
            if constexpr (!EIGHT) r.m = Piece<SMILE_DTYPE_F32>::load(x.m, at), r.v = Piece<SMILE_DTYPE_F32>::load(x.v, at);
        }
        if constexpr (EIGHT) {
            if ((long long)at < (x.n + 127) / 128 * 128) {
                r.m = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(x.m) + at), r.v = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(x.v) + at);
                r.m_scale = x.m_scale[at / 128], r.v_scale = x.v_scale[at / 128];
            }
        }
    };
    Raw cur, nxt;
    fetch(c, cur);
    const float inv1 = (float)(1.0 / one_minus_power(a.beta1, t)), inv2 = (float)(1.0 / one_minus_power(a.beta2, t));
    for (long long n = blockIdx.x; n < a.chunks; n += gridDim.x) {
        AdamwChunk ahead = c;
        if (n + gridDim.x < a.chunks) {
            ahead = a.list[n + gridDim.x];
            fetch(ahead, nxt);
        }
        const AdamwTensor &x = a.tensors[c.tensor];
        const size_t at = (size_t)c.chunk * kAdamwChunk + threadIdx.x * 8;
        const int live = (int)min(x.n - (long long)at, 8ll);
        // (8-bit states: the lanes of a block that holds an element stay together, behind the tensor's end too)
        if (EIGHT ? (long long)at < (x.n + 127) / 128 * 128 : live > 0) {
            float g[8], p[8], m[8], v[8];
            if (live == 8) {
                Piece<GDT>::widen(cur.g, g);
                Piece<MASTER ? SMILE_DTYPE_F32 : DT>::widen(cur.p, p);
                if constexpr (!EIGHT) Piece<SMILE_DTYPE_F32>::widen(cur.m, m), Piece<SMILE_DTYPE_F32>::widen(cur.v, v);
            } else {
                load_some<GDT>(x.grad, at, live, g);
                load_some<MASTER ? SMILE_DTYPE_F32 : DT>(MASTER ? x.master : x.param, at, live, p);
                if constexpr (!EIGHT) load_some<SMILE_DTYPE_F32>(x.m, at, live, m), load_some<SMILE_DTYPE_F32>(x.v, at, live, v);
            }
            if constexpr (EIGHT) {
                m_units(cur.m, m), scaled(m, (int)cur.m_scale - 127);
                v_units(cur.v, v), scaled(v, (int)cur.v_scale - 127);
            }
            const float decay = x.weight_decay;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                moments(a, g[i], m[i], v[i]);
                const float update = m[i] * inv1 * __builtin_amdgcn_rcpf(root(v[i] * inv2) + a.eps);
                p[i] -= lr * fmaf(decay, p[i], update);
            }
            store8<DT>(x.param, at, live, p);
            if constexpr (MASTER) store8<SMILE_DTYPE_F32>(x.master, at, live, p);
            if constexpr (!EIGHT) {
                store8<SMILE_DTYPE_F32>(x.m, at, live, m);
                store8<SMILE_DTYPE_F32>(x.v, at, live, v);
            } else {
                uint32_t top_m = 0u, top_v = 0u;   // largest magnitudes, which as bits have the order of their values
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i >= live) m[i] = v[i] = 0.f;
                    top_m = max(top_m, __float_as_uint(m[i]) & 0x7fffffffu), top_v = max(top_v, __float_as_uint(v[i]) & 0x7fffffffu);
                }
                top_m = block_max(top_m), top_v = block_max(top_v);
                uint32_t odd = 0u;                 // elements that are not finite: their codes are set below
                if (max(top_m, top_v) >= kInfinity) {
                    top_m = top_v = 0u;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t mm = __float_as_uint(m[i]) & 0x7fffffffu, vv = __float_as_uint(v[i]) & 0x7fffffffu;
                        if (mm >= kInfinity) odd |= 1u << i, m[i] = 0.f;
                        else top_m = max(top_m, mm);
                        if (vv >= kInfinity) odd |= 256u << i, v[i] = 0.f;
                        else top_v = max(top_v, vv);
                    }
                    top_m = block_max(top_m), top_v = block_max(top_v);
                }
                const int em = m_exponent(__uint_as_float(top_m)), ev = v_exponent(__uint_as_float(top_v));
                const uint32_t key = mix(key_step ^ (uint32_t)c.tensor) + (uint32_t)at;
                uint32_t mc[2] = {0u, 0u}, vc[2] = {0u, 0u};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t r = mix(key + i);
                    mc[i / 4] |= m_code(m[i], em, r & 0xffffu) << 8 * (i % 4);
                    vc[i / 4] |= v_code(v[i], ev, r >> 16) << 8 * (i % 4);
                }
                if (odd)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (odd >> i & 1u) mc[i / 4] |= 0x7fu << 8 * (i % 4);
                        if (odd >> i & 256u) vc[i / 4] |= 0xffu << 8 * (i % 4);
                    }
                store_codes(x.m, at, mc);
                store_codes(x.v, at, vc);
                if ((threadIdx.x & 15) == 0) x.m_scale[at / 128] = (uint8_t)(em + 127), x.v_scale[at / 128] = (uint8_t)(ev + 127);
            }
        }
        cur = nxt, c = ahead;
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void adamw_unpack_kernel(long long n, const uint8_t *m, const uint8_t *m_scale, const uint8_t *v, const uint8_t *v_scale,
                                                                void *m_value, void *v_value)
{
    const long long stride = (long long)gridDim.x * kAdamwChunk;
    for (long long at = ((long long)blockIdx.x * kThreads + threadIdx.x) * 8; at < n; at += stride) {
        float f[8];
        m_units(*reinterpret_cast<const uint2 *>(m + at), f), scaled(f, (int)m_scale[at / 128] - 127);
        store8<DT>(m_value, at, 8, f);
        v_units(*reinterpret_cast<const uint2 *>(v + at), f), scaled(f, (int)v_scale[at / 128] - 127);
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
    const int grid = (int)std::min((long long)a.chunks, (long long)workgroup_slots(tune, kPerCu));
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
