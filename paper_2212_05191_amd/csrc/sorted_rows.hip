// The (token, choice) pairs sorted by expert, and their rows: the stable counting sort, the tokens' rows moved to the sorted order, the weighted
// sum of each token's rows, and its gradients.
#include "fp8_device.hpp"
#include "sorted_internal.hpp"

#include <algorithm>

namespace smile {

namespace {

// ------------------------------------------------------------------ sort
//
// The pairs are cut into at most kSortBlocks blocks.  sort_hist_kernel counts a block's experts; every workgroup of sort_finish_kernel adds up the
// counts of all blocks and of those before its own (at most 128 x N words, read from L2), which with a prefix sum over the experts
// is where its pairs begin, and ranks its pairs: each wave has a consecutive part of the block, whose experts it counts first, then takes 64
// pairs at a time; lanes with equal experts find each other by one ballot for each bit of the expert's number.  A block alone needs no counts from
// others.  Bound: latency (one or two launches of a few dependent reads); 8 bytes a pair read and 8 written.
constexpr int kSortThreads = 1024, kSortBlocks = 128;

int sort_block_pairs(int pairs)
{
    const long long each = ((long long)pairs + kSortBlocks - 1) / kSortBlocks;
    return (int)((each + kSortThreads - 1) / kSortThreads * kSortThreads);
}
int sort_blocks(int pairs) { return (int)(((long long)pairs + sort_block_pairs(pairs) - 1) / sort_block_pairs(pairs)); }
// Few pairs are counted by every workgroup itself, instead of by a launch ahead (random experts, 10006 pairs among 16 5.5 against 6.1 us, among 4096 11.1 against 16.0; 20000
// among 16 7.7 against 6.4, among 1024 9.2 against 9.8).
bool sort_recounts(int pairs, int N) { return pairs <= 12288 + 8 * N; }

// the pair's expert, N where it has none
__device__ __forceinline__ int expert_of(const int32_t *idx, int p, int end, int N)
{
    if (p >= end) return N;
    const int e = idx[p];
    return (unsigned)e < (unsigned)N ? e : N;
}

__global__ __launch_bounds__(kSortThreads) void sort_hist_kernel(const int32_t *idx, int32_t *hist, int pairs, int N, int block_pairs)
{
    extern __shared__ int count[];
    const long long first = (long long)blockIdx.x * block_pairs;
    const int begin = (int)first, end = (int)min(first + block_pairs, (long long)pairs);
    for (int e = threadIdx.x; e < N; e += kSortThreads) count[e] = 0;
    __syncthreads();
    for (int p = begin + threadIdx.x; p < end; p += kSortThreads) {
        const int e = expert_of(idx, p, end, N);
        if (e < N) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < N; e += kSortThreads) hist[(size_t)blockIdx.x * N + e] = count[e];
}

// WAVES waves rank pairs (fewer for many experts: a wave's counters are MOST words of LDS)
template <int MOST, int WAVES>
__global__ __launch_bounds__(kSortThreads) void sort_finish_kernel(SortIo io, int block_pairs, int blocks)
{
    __shared__ int before[MOST], total[MOST], mine[WAVES][MOST], wave_total[kSortThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, N = io.N;
    const long long first = (long long)blockIdx.x * block_pairs;
    const int begin = (int)first, end = (int)min(first + block_pairs, (long long)io.pairs);
    const int part = block_pairs / WAVES, from = begin + wave * part, to = (int)min((long long)from + part, (long long)end);
    for (int e = tid; e < MOST; e += kSortThreads) {
        before[e] = total[e] = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) mine[w][e] = 0;
    }
    __syncthreads();
    if (wave < WAVES)
        for (int p = from + lane; p < to; p += 64) {
            const int e = expert_of(io.idx, p, to, N);
            if (e < N) atomicAdd(&mine[wave][e], 1);
        }
    if (blocks > 1 && !io.hist) {
        // every pair is counted here, the pairs ahead of the block by themselves
        typedef __attribute__((__vector_size__(16))) int32_t four;
        // the lanes that have the first lane's expert count together, so that one that most pairs have is not counted pair by pair
        auto count = [&](bool ahead, int e) {
            int *counts = ahead ? before : total;
            const int common = __builtin_amdgcn_readfirstlane(e);
            const uint64_t same = __ballot(e == common);
            if (e == common) {
                if (lane == __builtin_ctzll(same) && (unsigned)e < (unsigned)N) atomicAdd(&counts[e], __builtin_popcountll(same));
            } else if ((unsigned)e < (unsigned)N) {
                atomicAdd(&counts[e], 1);
            }
        };
        const int quads = io.pairs & ~3;
        for (int p0 = 4 * tid; p0 < quads; p0 += 16 * kSortThreads) {
            four v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const four *>(io.idx + min(p0 + 4 * u * kSortThreads, quads - 4));
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int p = p0 + 4 * u * kSortThreads;
                if (p < quads)
#pragma unroll
                    for (int i = 0; i < 4; ++i) count(p < begin, v[u][i]);
            }
        }
        if (tid < io.pairs - quads) count(quads < begin, io.idx[quads + tid]);
        __syncthreads();
        for (int e = tid; e < N; e += kSortThreads) total[e] += before[e];
    } else if (blocks > 1) {
        // counts of all blocks, as many threads an expert as there are to spare
        int lanes = 1;
        while (lanes * 2 * N <= kSortThreads) lanes *= 2;
        const int e0 = tid / lanes, b0 = tid % lanes;
        for (int e = e0; e < N; e += kSortThreads / lanes) {
            int all = 0, ahead = 0;
#pragma unroll 8
            for (int b = b0; b < blocks; b += lanes) {
                const int c = io.hist[(size_t)b * N + e];
                all += c;
                if (b < (int)blockIdx.x) ahead += c;
            }
            if (all) atomicAdd(&total[e], all);
            if (ahead) atomicAdd(&before[e], ahead);
        }
    }
    __syncthreads();
    if (blocks == 1) {
        for (int e = tid; e < N; e += kSortThreads) {
            int all = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all += mine[w][e];
            total[e] = all;
        }
        __syncthreads();
    }
    // exclusive prefix sum of the totals: MOST / 1024 neighbouring experts a thread (one for fewer experts)
    constexpr int PER = MOST > kSortThreads ? MOST / kSortThreads : 1;
    int own[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = tid * PER + i;
        own[i] = e < N ? total[e] : 0, sum += own[i];
    }
    const int incl = LiveTileWalk<1>::scan(sum);
    if (lane == 63) wave_total[wave] = incl;
    __syncthreads();
    int at = incl - sum, live = 0;
#pragma unroll
    for (int w = 0; w < kSortThreads / 64; ++w) {
        if (w < wave) at += wave_total[w];
        live += wave_total[w];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = tid * PER + i;
        if (e < N) {
            if (blockIdx.x == 0) io.count[e] = own[i], io.start[e] = at;
            int base = at + before[e];          // the first row of the block's pairs of this expert, then of each wave's
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int c = mine[w][e];
                mine[w][e] = base, base += c;
            }
        }
        at += own[i];
    }
    if (blockIdx.x == 0 && tid == 0) io.start[N] = live;
    for (int p = begin + tid; p < end; p += kSortThreads)
        if (p >= live) io.source[p] = -1;       // rows behind the last expert's
    __syncthreads();
    if (wave >= WAVES) return;
    const int bits = 32 - __builtin_clz(N);     // N itself: no expert
    for (int p0 = from; p0 < to; p0 += 64) {
        const int p = p0 + lane, e = expert_of(io.idx, p, to, N);
        uint64_t same = ~0ull;
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot(e >> b & 1);
            same &= e >> b & 1 ? set : ~set;
        }
        const int leader = __builtin_ctzll(same), rank = __builtin_popcountll(same & ((1ull << lane) - 1));
        int base = 0;
        if (e < N && lane == leader) base = atomicAdd(&mine[wave][e], __builtin_popcountll(same));
        base = __shfl(base, leader, 64);
        if (p < to) {
            io.pos[p] = e < N ? base + rank : -1;
            if (e < N) io.source[base + rank] = p;
        }
    }
}

// ------------------------------------------------------------------ rows
//
// A token is L lanes of a wave (a power of two up to 64, at least as many as its row has 16-byte pieces): a row is read once, in whole lines, and
// k rows are written or read, all of a token's loads in flight before the first is used.  Bound: HBM.
constexpr int kRowThreads = 256, kJ = 4;   // choices handled at a time

template <int DT>
struct Vec;   // a 16-byte piece and its elements
template <>
struct Vec<SMILE_DTYPE_F32> {
    static constexpr int kElems = 4;
    __device__ static __forceinline__ void widen(u32x4 r, float *v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
    }
    __device__ static __forceinline__ u32x4 narrow(const float *v)
    {
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};
template <typename E>
struct HalfVec {
    static constexpr int kElems = 8;
    __device__ static __forceinline__ void widen(u32x4 r, float *v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = Half<E>::lo(r[i]), v[2 * i + 1] = Half<E>::hi(r[i]);
    }
    __device__ static __forceinline__ u32x4 narrow(const float *v)
    {
        return u32x4{Half<E>::pack(v[0], v[1]), Half<E>::pack(v[2], v[3]), Half<E>::pack(v[4], v[5]), Half<E>::pack(v[6], v[7])};
    }
};
template <>
struct Vec<SMILE_DTYPE_BF16> : HalfVec<__bf16> {};
template <>
struct Vec<SMILE_DTYPE_F16> : HalfVec<_Float16> {};

struct RowShape {
    int pieces, shift;   // 16-byte pieces of a row, log2 of the lanes of a token
};

// this lane's token and its place among the token's lanes; false: none
__device__ __forceinline__ bool token_of(const SortedRowsIo &io, const RowShape &sh, int &t, int &lane)
{
    const long long id = (long long)blockIdx.x * kRowThreads + threadIdx.x;
    lane = threadIdx.x & ((1 << sh.shift) - 1);
    t = (int)(id >> sh.shift);
    return (id >> sh.shift) < io.T;
}
// a pair's row, -1 where it has none
__device__ __forceinline__ int row_of(const SortedRowsIo &io, int t, int j)
{
    if (j >= io.k) return -1;
    const int r = io.pos[(size_t)t * io.k + j];
    return (unsigned)r < (unsigned)io.R ? r : -1;
}

__global__ __launch_bounds__(kRowThreads) void sorted_dispatch_kernel(SortedRowsIo io, RowShape sh)
{
    int t, lane;
    if (!token_of(io, sh, t, lane)) return;
    const u32x4 *x = static_cast<const u32x4 *>(io.x) + (size_t)t * sh.pieces;
    u32x4 *xs = static_cast<u32x4 *>(io.y);
    for (int c = lane; c < sh.pieces; c += 1 << sh.shift) {
        const u32x4 v = x[c];
        for (int j0 = 0; j0 < io.k; j0 += kJ) {
            int r[kJ];
#pragma unroll
            for (int j = 0; j < kJ; ++j) r[j] = row_of(io, t, j0 + j);
#pragma unroll
            for (int j = 0; j < kJ; ++j)
                if (r[j] >= 0) xs[(size_t)r[j] * sh.pieces + c] = v;
        }
    }
}

template <int DT>
__global__ __launch_bounds__(kRowThreads) void sorted_combine_kernel(SortedRowsIo io, RowShape sh)
{
    constexpr int E = Vec<DT>::kElems;
    int t, lane;
    if (!token_of(io, sh, t, lane)) return;
    const u32x4 *ys = static_cast<const u32x4 *>(io.x);
    for (int c = lane; c < sh.pieces; c += 1 << sh.shift) {
        float sum[E];
        u32x4 res = {0u, 0u, 0u, 0u};
        if (io.residual) res = static_cast<const u32x4 *>(io.residual)[(size_t)t * sh.pieces + c];
        Vec<DT>::widen(res, sum);
        for (int j0 = 0; j0 < io.k; j0 += kJ) {
            u32x4 v[kJ];
            int r[kJ];
            float w[kJ];
#pragma unroll
            for (int j = 0; j < kJ; ++j) {
                r[j] = row_of(io, t, j0 + j);
                w[j] = io.weight && r[j] >= 0 ? io.weight[(size_t)t * io.k + j0 + j] : 1.f;
                v[j] = u32x4{0u, 0u, 0u, 0u};
                if (r[j] >= 0) v[j] = ys[(size_t)r[j] * sh.pieces + c];
            }
#pragma unroll
            for (int j = 0; j < kJ; ++j) {
                if (r[j] < 0) continue;
                float f[E];
                Vec<DT>::widen(v[j], f);
#pragma unroll
                for (int i = 0; i < E; ++i) sum[i] = fmaf(w[j], f[i], sum[i]);
            }
        }
        static_cast<u32x4 *>(io.y)[(size_t)t * sh.pieces + c] = Vec<DT>::narrow(sum);
    }
}

template <int DT>
__global__ __launch_bounds__(kRowThreads) void sorted_combine_backward_kernel(SortedRowsIo io, RowShape sh)
{
    constexpr int E = Vec<DT>::kElems;
    int t, lane;
    if (!token_of(io, sh, t, lane)) return;                             // (whole tokens: the lanes of a sum leave together)
    const u32x4 *dy = static_cast<const u32x4 *>(io.x) + (size_t)t * sh.pieces, *ys = static_cast<const u32x4 *>(io.rows);
    u32x4 *dys = static_cast<u32x4 *>(io.y);
    for (int j0 = 0; j0 < io.k; j0 += kJ) {
        int r[kJ];
        float w[kJ], dot[kJ];
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
            r[j] = row_of(io, t, j0 + j), dot[j] = 0.f;
            w[j] = r[j] >= 0 ? io.weight[(size_t)t * io.k + j0 + j] : 0.f;
        }
        for (int c = lane; c < sh.pieces; c += 1 << sh.shift) {
            const u32x4 g = dy[c];
            u32x4 v[kJ];
            if (ys)
#pragma unroll
                for (int j = 0; j < kJ; ++j)
                    if (r[j] >= 0) v[j] = ys[(size_t)r[j] * sh.pieces + c];
            float f[E];
            Vec<DT>::widen(g, f);
#pragma unroll
            for (int j = 0; j < kJ; ++j) {
                if (r[j] < 0) continue;
                float o[E];
#pragma unroll
                for (int i = 0; i < E; ++i) o[i] = w[j] * f[i];
                if (ys) {
                    float y[E];
                    Vec<DT>::widen(v[j], y);
#pragma unroll
                    for (int i = 0; i < E; ++i) dot[j] = fmaf(f[i], y[i], dot[j]);
                }
                dys[(size_t)r[j] * sh.pieces + c] = Vec<DT>::narrow(o);
            }
        }
        if (!ys) continue;
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
            for (int off = 1; off < 1 << sh.shift; off <<= 1) dot[j] += __shfl_xor(dot[j], off, 64);
            if (j0 + j < io.k && lane == 0) io.dweight[(size_t)t * io.k + j0 + j] = dot[j];
        }
    }
}

RowShape row_shape(int dtype, int d, int T)
{
    RowShape sh{d * elem_size(dtype) / 16, 0};
    const int most = T > 1 << 24 ? 5 : 6;   // (less than 2^32 threads a launch)
    while (sh.shift < most && (1 << sh.shift) < sh.pieces) ++sh.shift;
    return sh;
}
int row_grid(const SortedRowsIo &io, const RowShape &sh) { return (int)((((long long)io.T << sh.shift) + kRowThreads - 1) / kRowThreads); }

}  // namespace

size_t sort_experts_workspace(int pairs, int N)
{
    const int blocks = sort_blocks(pairs);
    return blocks > 1 && !sort_recounts(pairs, N) ? (size_t)blocks * N * sizeof(int32_t) : 0;
}

hipError_t launch_sort_experts(const SortIo &given, hipStream_t s)
{
    SortIo io = given;
    if (sort_recounts(io.pairs, io.N)) io.hist = nullptr;
    const int block_pairs = sort_block_pairs(io.pairs), blocks = sort_blocks(io.pairs);
    if (io.hist && blocks > 1) SMILE_LAUNCH(sort_hist_kernel, dim3(blocks), dim3(kSortThreads), io.N * sizeof(int), s, io.idx, io.hist, io.pairs, io.N, block_pairs);
    if (io.N <= 256) SMILE_LAUNCH((sort_finish_kernel<256, 16>), dim3(blocks), dim3(kSortThreads), 0, s, io, block_pairs, blocks);
    else if (io.N <= 1024) SMILE_LAUNCH((sort_finish_kernel<1024, 16>), dim3(blocks), dim3(kSortThreads), 0, s, io, block_pairs, blocks);
    else SMILE_LAUNCH((sort_finish_kernel<4096, 4>), dim3(blocks), dim3(kSortThreads), 0, s, io, block_pairs, blocks);
    return hipGetLastError();
}

hipError_t launch_sorted_dispatch(int dtype, const SortedRowsIo &io, hipStream_t s)
{
    const RowShape sh = row_shape(dtype, io.d, io.T);
    SMILE_LAUNCH(sorted_dispatch_kernel, dim3(row_grid(io, sh)), dim3(kRowThreads), 0, s, io, sh);
    return hipGetLastError();
}

hipError_t launch_sorted_combine(int dtype, const SortedRowsIo &io, hipStream_t s)
{
    const RowShape sh = row_shape(dtype, io.d, io.T);
    const dim3 grid(row_grid(io, sh));
    if (dtype == SMILE_DTYPE_F32) SMILE_LAUNCH(sorted_combine_kernel<SMILE_DTYPE_F32>, grid, dim3(kRowThreads), 0, s, io, sh);
    else if (dtype == SMILE_DTYPE_BF16) SMILE_LAUNCH(sorted_combine_kernel<SMILE_DTYPE_BF16>, grid, dim3(kRowThreads), 0, s, io, sh);
    else SMILE_LAUNCH(sorted_combine_kernel<SMILE_DTYPE_F16>, grid, dim3(kRowThreads), 0, s, io, sh);
    return hipGetLastError();
}

hipError_t launch_sorted_combine_backward(int dtype, const SortedRowsIo &io, hipStream_t s)
{
    const RowShape sh = row_shape(dtype, io.d, io.T);
    const dim3 grid(row_grid(io, sh));
    if (dtype == SMILE_DTYPE_F32) SMILE_LAUNCH(sorted_combine_backward_kernel<SMILE_DTYPE_F32>, grid, dim3(kRowThreads), 0, s, io, sh);
    else if (dtype == SMILE_DTYPE_BF16) SMILE_LAUNCH(sorted_combine_backward_kernel<SMILE_DTYPE_BF16>, grid, dim3(kRowThreads), 0, s, io, sh);
    else SMILE_LAUNCH(sorted_combine_backward_kernel<SMILE_DTYPE_F16>, grid, dim3(kRowThreads), 0, s, io, sh);
    return hipGetLastError();
}

}  // namespace smile
