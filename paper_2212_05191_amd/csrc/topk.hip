// k experts for a token: softmax over N columns, the k largest values, their weights, the column sums of the probabilities; and the
// gradient of the logits.
//
// A token is L lanes of a wave, each with V of its values in registers (column 4 (i L + lane) + q, 16 bytes at a time), so that a row is
// read once and nothing of it is kept anywhere else.  A choice takes the largest of the lane's values, each with its column
// one double, then of the lanes by DPP, and removes it.  Bound: HBM for many tokens (4 N bytes read each, and 4 N written by
// the gradient); by instructions where k is large (3 V a choice); by latency for few tokens.
#include "gemm_device.hpp"
#include "sorted_internal.hpp"

#include <algorithm>

namespace smile {

namespace {

// Workgroups of the choice: more of them make more partial sums, fewer leave the CUs short of waves (65536 x 128, k = 8: 512 31 us, 1024 25, 2048 25 and a longer sum)
constexpr int kThreads = 256, kMaxBlocks = 1024;
// tokens that one workgroup takes alone, without a second launch for p_sum: rounds of its lanes.  The launch costs 2 to 3 us; a second round 1 (64 tokens of 24: 4.5 us against
// 5.5), of more columns 3 to 9 (16 of 256: 9.2 against 8.0; 8 of 4096: 27.7 against 18.3).
constexpr int alone_lanes(int N) { return (N <= 64 ? 2 : 1) * kThreads; }

// Reductions over the L lanes of a token (L = 4 .. 64, aligned); every lane ends with the same bits
template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
template <int L, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f)
{
    auto step = [&](int other) { v = f(v, __builtin_bit_cast(T, other)); };
    step(dpp<0xB1>(__builtin_bit_cast(int, v)));                        // quads: 1 0 3 2
    step(dpp<0x4E>(__builtin_bit_cast(int, v)));                        // 2 3 0 1
    if constexpr (L >= 8) step(dpp<0x141>(__builtin_bit_cast(int, v)));   // mirrored in 8
    if constexpr (L >= 16) step(dpp<0x140>(__builtin_bit_cast(int, v)));  // mirrored in 16
    if constexpr (L >= 32) step(__shfl_xor(__builtin_bit_cast(int, v), 16, 64));
    if constexpr (L >= 64) step(__shfl_xor(__builtin_bit_cast(int, v), 32, 64));
    return v;
}
template <int L>
__device__ __forceinline__ float max_over(float v) { return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int L>
__device__ __forceinline__ float sum_over(float v) { return over_lanes<L>(v, [](float a, float b) { return a + b; }); }

// exp(x), x <= 0, to 2 units of the last place: the exponent's rounding error is multiplied in
__device__ __forceinline__ float exp_near(float x)
{
    const float hi = x * 1.44269504f;
    const float lo = fmaf(x, 1.44269504f, -hi) + x * 1.92596303e-8f;    // log2(e) = 1.44269504 + 1.926e-8
    const float e = __builtin_amdgcn_exp2f(hi);
    return x < -150.f ? 0.f : fmaf(e, lo * 0.69314718f, e);             // (also -infinity, whose lo is NaN)
}

// This lane's elements of a row of N (what is beyond it repeats its end): all loads without a branch between them, so that they are in flight together
template <int L, int V, typename T>
__device__ __forceinline__ void load_row(T (&v)[V], const T *row, int N, int lane)
{
    typedef __attribute__((__vector_size__(16))) T quad;
    if (!(N & 3)) {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const quad a = *reinterpret_cast<const quad *>(row + min(4 * (i * L + lane), N - 4));
#pragma unroll
            for (int q = 0; q < 4; ++q) v[4 * i + q] = a[q];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = row[min(4 * ((i / 4) * L + lane) + i % 4, N - 1)];
    }
}

// The values of token t in this lane, -infinity where there is none
template <int L, int V>
__device__ __forceinline__ void load_values(float (&v)[V], const float *logits, const float *bias, int t, int N, int lane)
{
    load_row<L, V>(v, logits + (size_t)t * N, N, lane);
    if (bias) {
        float b[V];
        load_row<L, V>(b, bias, N, lane);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = b[i] == -INFINITY ? -INFINITY : v[i] + b[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (4 * ((i / 4) * L + lane) + i % 4 >= N) v[i] = -INFINITY;
}

// v -> e = exp(v - base), base the largest (0 if there is none); returns 1 / sum (0 for a token without an expert)
template <int L, int V>
__device__ __forceinline__ float exponentials(const float (&v)[V], float (&e)[V], float &base)
{
    float top = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, v[i]);
    top = max_over<L>(top);
    base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = exp_near(v[i] - base), sum += e[i];
    sum = sum_over<L>(sum);
    return sum == 0.f ? 0.f : 1.f / sum;
}

// A value and its column as one double, ordered by the value and among equal ones from the highest column to the lowest: the value's bits are the upper word (three bits
// of its fraction count as exponent, which keeps the order, and no finite or infinite value becomes a NaN), the column, or its complement under a positive value, the
// lower.  One v_max_f64 compares both.  What cannot be chosen (-infinity, NaN, chosen before) is kGone, below all of them.
constexpr uint32_t kGone = 0xffe00000u;
__device__ __forceinline__ double ordered(float v, int col)
{
    const uint32_t hi = __float_as_uint(v + 0.f);           // (-0 is 0)
    const uint32_t lo = (int)hi < 0 ? (uint32_t)col : ~(uint32_t)col;
    const bool none = !(v > -INFINITY);
    return __hiloint2double((int)(none ? kGone : hi), (int)(none ? 0u : lo));
}
__device__ __forceinline__ double larger(double a, double b)
{
    double r;   // (fmax would quiet NaNs first, of which there are none)
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
template <int CTRL>
__device__ __forceinline__ double larger_of(double v)
{
    return larger(v, __hiloint2double(dpp<CTRL>(__double2hiint(v)), dpp<CTRL>(__double2loint(v))));
}
template <int L>
__device__ __forceinline__ double largest_over(double v)
{
    v = larger_of<0xB1>(v), v = larger_of<0x4E>(v);
    if constexpr (L >= 8) v = larger_of<0x141>(v);
    if constexpr (L >= 16) v = larger_of<0x140>(v);
    if constexpr (L >= 32) v = larger(v, __shfl_xor(v, 16, 64));
    if constexpr (L >= 64) v = larger(v, __shfl_xor(v, 32, 64));
    return v;
}

template <int L, int V>
__global__ __launch_bounds__(kThreads, V == 4 ? 8 : V == 8 ? 6 : V == 16 ? 4 : V == 32 ? 2 : 1) void topk_kernel(TopkIo io, int per_block)
{
    constexpr int TPB = kThreads / L;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L;
    const int first = blockIdx.x * per_block, last = min(io.T, first + per_block);
    float total[V];
#pragma unroll
    for (int i = 0; i < V; ++i) total[i] = 0.f;
    for (int t0 = first; t0 < last; t0 += TPB) {
        const int t = t0 + slot;
        const bool live = t < last;
        float v[V], e[V];
        int own = lane;
        const float *bias = io.bias;
        asm volatile("" : "+v"(own), "+s"(bias));   // (what the loads need is not kept in registers from token to token)
        load_values<L, V>(v, io.logits, bias, min(t, last - 1), io.N, own);
        float base;
        const float inv = exponentials<L, V>(v, e, base);
        if (io.partial || io.p_sum) {
            const float scale = live ? inv : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) total[i] = live ? fmaf(e[i], scale, total[i]) : total[i];
        }
        double key[V];
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = ordered(v[i], 4 * ((i / 4) * L + lane) + i % 4);
        // the choices, L at a time: lane j % L keeps the j-th.  Their weights are divided when all are known: those of earlier rounds lie in the output until then.
        float sum = 0.f, mine = 0.f;
        bool more = true;
        int32_t *idx = io.idx + (size_t)t * io.k + lane;
        float *weight = io.weight + (size_t)t * io.k + lane;
        for (int j0 = 0; j0 < io.k; j0 += L) {
            int chosen = -1;
            mine = 0.f;
            for (int jj = 0; more && jj < L && j0 + jj < io.k; ++jj) {
                double top[V / 2];      // (pairs, then pairs of those: not one chain of V)
#pragma unroll
                for (int i = 0; i < V / 2; ++i) top[i] = larger(key[2 * i], key[2 * i + 1]);
#pragma unroll
                for (int m = V / 4; m >= 1; m /= 2)
#pragma unroll
                    for (int i = 0; i < m; ++i) top[i] = larger(top[i], top[i + m]);
                const double best = largest_over<L>(top[0]);
                const int hi = __double2hiint(best), lo = __double2loint(best);
                more = (uint32_t)hi != kGone;
                if (!more) break;
#pragma unroll
                for (int i = 0; i < V; ++i) key[i] = key[i] == best ? __hiloint2double((int)kGone, lo) : key[i];
                const float ex = exp_near(__int_as_float(hi) - base);
                sum += ex;
                if (lane == jj) chosen = hi < 0 ? lo : ~lo, mine = ex;
            }
            if (live && j0 + lane < io.k) {
                idx[j0] = chosen;
                if (j0 + L < io.k) weight[j0] = mine;
            }
        }
        if (live) {
            for (int j0 = 0; j0 < io.k; j0 += L)
                if (j0 + lane < io.k) {
                    const float ex = j0 + L < io.k ? weight[j0] : mine;
                    weight[j0] = !io.normalize || inv != inv ? ex * inv : sum == 0.f ? 0.f : ex / sum;   // (NaN stays; a single choice has the weight 1)
                }
        }
    }
    if (!io.partial && !io.p_sum) return;
    // columns of this workgroup: over the tokens of a wave, then of the four waves in their order
    __shared__ float wave_sum[kThreads / 64][L * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float s = total[i];
#pragma unroll
        for (int off = L; off < 64; off <<= 1) s += __shfl_xor(s, off, 64);
        if ((threadIdx.x & 63) < L) wave_sum[threadIdx.x >> 6][4 * ((i / 4) * L + lane) + i % 4] = s;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < io.N; c += kThreads) {
        const float s = (wave_sum[0][c] + wave_sum[1][c]) + (wave_sum[2][c] + wave_sum[3][c]);
        if (io.partial) io.partial[(size_t)blockIdx.x * io.N + c] = s;
        else io.p_sum[c] = s;
    }
}

// p_sum[c] = sum over the workgroups' rows of partial[blocks][N], in 64 bits: four columns a workgroup, 64 threads each
__global__ __launch_bounds__(kThreads) void topk_sum_kernel(const float *partial, float *p_sum, int blocks, int N)
{
    __shared__ double part[kThreads];
    const int c = blockIdx.x * 4 + threadIdx.x % 4, row0 = threadIdx.x / 4;
    double s = 0.0;
    if (c < N)
#pragma unroll 8
        for (int b = row0; b < blocks; b += kThreads / 4) s += (double)partial[(size_t)b * N + c];
    part[threadIdx.x] = s;
    __syncthreads();
    for (int n = kThreads / 2; n >= 4; n >>= 1) {
        if ((int)threadIdx.x < n) part[threadIdx.x] += part[threadIdx.x + n];
        __syncthreads();
    }
    if (threadIdx.x < 4 && c < N) p_sum[c] = (float)part[threadIdx.x];
}

// dlogits = p (u - sum p u), + w (dweight - sum w dweight) at the chosen columns of normalised weights.  The chosen values are gathered through the
// token's lanes: each lane compares the columns that it holds.
template <int L, int V>
__global__ __launch_bounds__(kThreads, V <= 8 ? 8 : V == 16 ? 5 : V == 32 ? 2 : 1) void topk_backward_kernel(TopkGradIo io)
{
    const int lane = threadIdx.x % L;
    const long long id = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads / L) + threadIdx.x / L;
    if (id >= io.T) return;
    const int t = (int)id;
    float v[V], p[V], u[V];
    load_values<L, V>(v, io.logits, io.bias, t, io.N, lane);
    float base;
    const float inv = exponentials<L, V>(v, p, base);
    int count[V];
    if (io.count) load_row<L, V>(count, io.count, io.N, lane);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        p[i] *= inv;
        u[i] = io.count ? io.coef * (float)(count[i] - io.count[0]) : 0.f;   // (a constant added to u changes nothing: even counts are told apart exactly)
        v[i] = 0.f;                                                     // from here on: the gradient that reaches a chosen column
    }
    const size_t at = (size_t)t * io.k;
    std::conditional_t<(V > 32), uint64_t, uint32_t> picked = 0;        // of the lane's values
    constexpr decltype(picked) one = 1;
#pragma unroll 1
    for (int j0 = 0; j0 < io.k; j0 += 4) {                              // four choices' loads at a time
        int col[4];
        float dw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) col[j] = j0 + j < io.k ? io.idx[at + j0 + j] : -1, dw[j] = j0 + j < io.k ? io.dweight[at + j0 + j] : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int rel = (unsigned)col[j] < (unsigned)io.N ? col[j] - 4 * lane : -1;
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += 4 * (i / 4) * L + i % 4 == rel ? dw[j] : 0.f;
            if (rel >= 0 && rel % (4 * L) < 4) picked |= one << (rel / (4 * L) * 4 + rel % 4);
        }
    }
    // A weight as p / sum with its rounding mended, so that it is 1 where one is chosen: what the weights' gradient then leaves is exactly nothing, which its rounding, beside a
    // small coef, would not be.
    float of_chosen = 0.f, sum = 0.f, dot = 0.f;
    auto weight_of = [&](float p) {
        const float w = p * of_chosen;
        return fmaf(fmaf(-w, sum, p), of_chosen, w);
    };
    if (io.normalize) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (picked >> i & 1) sum += p[i];
        sum = sum_over<L>(sum);
        of_chosen = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (picked >> i & 1) dot = fmaf(weight_of(p[i]), v[i], dot);
        dot = sum_over<L>(dot);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (picked >> i & 1) u[i] += v[i];
    }
    float mean = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) mean = fmaf(p[i], u[i], mean);
    mean = sum_over<L>(mean);
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const int col = 4 * (i * L + lane);
        f32x4 d;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = 4 * i + q;
            d[q] = p[n] * (u[n] - mean);
            if (io.normalize && (picked >> n & 1)) d[q] = fmaf(weight_of(p[n]), v[n] - dot, d[q]);
        }
        float *to = io.dlogits + (size_t)t * io.N + col;
        if (!(io.N & 3)) {
            if (col < io.N) *reinterpret_cast<f32x4 *>(to) = d;
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (col + q < io.N) to[q] = d[q];
        }
    }
}

// f(lanes, values) of the smallest shape that holds N columns.  Few tokens leave lanes idle and their time is that of a lane's values one after another: twice the
// lanes with half of the values (choice with sum, gradient; 1 token of 128, k = 8: 7.0 -> 4.8, 5.4 -> 3.7 us; 8192: 11.4 -> 9.2, 6.1 -> 4.8; many repeat less with
// fewer lanes: 65536 27.7 against 31.1).
template <typename F>
auto with_shape(int T, int N, F &&f)
{
#define SMILE_SHAPE(l, v) return f(std::integral_constant<int, l>{}, std::integral_constant<int, v>{})
    if (N <= 16) SMILE_SHAPE(4, 4);
    if ((long long)T * N <= 1 << 20) {
        if (N <= 32) SMILE_SHAPE(8, 4);
        if (N <= 64) SMILE_SHAPE(16, 4);
        if (N <= 128) SMILE_SHAPE(16, 8);
        if (N <= 256) SMILE_SHAPE(32, 8);
        if (N <= 512) SMILE_SHAPE(64, 8);
    }
    if (N <= 32) SMILE_SHAPE(4, 8);
    if (N <= 64) SMILE_SHAPE(8, 8);
    if (N <= 128) SMILE_SHAPE(8, 16);
    if (N <= 256) SMILE_SHAPE(16, 16);
    if (N <= 512) SMILE_SHAPE(32, 16);
    if (N <= 1024) SMILE_SHAPE(64, 16);
    if (N <= 2048) SMILE_SHAPE(64, 32);
    SMILE_SHAPE(64, 64);
#undef SMILE_SHAPE
}

int lanes(int T, int N) { return with_shape(T, N, [](auto l, auto) { return (int)decltype(l)::value; }); }

// tokens of a workgroup (a whole number of rounds of its lanes) and workgroups
void plan(int T, int N, bool sum, int &per_block, int &blocks)
{
    const int tpb = kThreads / lanes(T, N);
    if (sum && (long long)T * lanes(T, N) <= alone_lanes(N)) {
        per_block = T, blocks = 1;
        return;
    }
    const int rounds = (T + tpb - 1) / tpb;
    per_block = (rounds + kMaxBlocks - 1) / kMaxBlocks * tpb;
    blocks = (T + per_block - 1) / per_block;
}

}  // namespace

size_t topk_workspace(int T, int N)
{
    int per_block, blocks;
    plan(T, N, true, per_block, blocks);
    return blocks > 1 ? (size_t)blocks * N * sizeof(float) : 0;
}

hipError_t launch_topk(const TopkIo &given, hipStream_t s)
{
    TopkIo io = given;
    int per_block, blocks;
    plan(io.T, io.N, io.p_sum != nullptr, per_block, blocks);
    if (!io.p_sum || blocks == 1) io.partial = nullptr;
    with_shape(io.T, io.N, [&](auto l, auto v) {
        SMILE_LAUNCH((topk_kernel<decltype(l)::value, decltype(v)::value>), dim3(blocks), dim3(kThreads), 0, s, io, per_block);
        return 0;
    });
    if (io.partial) SMILE_LAUNCH(topk_sum_kernel, dim3((io.N + 3) / 4), dim3(kThreads), 0, s, (const float *)io.partial, io.p_sum, blocks, io.N);
    return hipGetLastError();
}

hipError_t launch_topk_backward(const TopkGradIo &io, hipStream_t s)
{
    with_shape(io.T, io.N, [&](auto l, auto v) {
        const int tpb = kThreads / decltype(l)::value;
        const int blocks = (io.T + tpb - 1) / tpb, wide = std::min(blocks, 1 << 20);   // (less than 2^32 threads a dimension)
        SMILE_LAUNCH((topk_backward_kernel<decltype(l)::value, decltype(v)::value>), dim3(wide, (blocks + wide - 1) / wide), dim3(kThreads), 0, s, io);
        return 0;
    });
    return hipGetLastError();
}

}  // namespace smile
