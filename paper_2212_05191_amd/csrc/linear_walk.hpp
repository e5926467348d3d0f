// The tiles of a product over sorted rows, as the kernels of smile_linear and of its gradients walk them (HIP, gfx950).
#pragma once

#include "gemm_device.hpp"
#include "linear_internal.hpp"

namespace smile {

namespace {

struct LinearTile {
    int e;       // group
    int first;   // row 0 of the tile: of x and y (rows), of y[e] (weights' gradient)
    int rows;    // output rows that exist from there on (may be more than a tile)
    int col0;
    int from, kv;   // first term of the sum and terms
    int part;
};

// rows [lo, hi) of group g, whatever `start` holds.  Read through the constant address space: with a uniform g by the scalar unit, whose counter is not that of
// the loads in flight.
__device__ __forceinline__ void group_rows(const int32_t *start, int rows, int g, int &lo, int &hi)
{
    if (!start) {
        lo = 0, hi = rows;
        return;
    }
    typedef const __attribute__((address_space(4))) int32_t *constant;
    const constant s = (constant)(uintptr_t)start;
    lo = min(max(s[g], 0), rows);
    hi = min(max(s[g + 1], lo), rows);
}

// Live row tiles of groups whose first rows the device alone knows.  Lane c of every wave holds the row tiles of groups 64 c .. 64 c + 63 and their
// prefix sum (N <= 4096), so that two ballots find the group of a ticket: no LDS, no further launch.  Tickets run over the groups; inside
// a group over bands of BAND row tiles, the columns of a band, its rows: BAND x the columns' tiles side by side share operands.  The XCDs (own L2 each;
// workgroup ids go round them) take contiguous eighths.
template <int BM, int BAND>
struct RowWalk {
    const int32_t *start;
    int N, rows, col_tiles, lane;
    int chunk_incl, cur_chunk, cur_incl, whole, tickets;   // whole: tiles of one part of the sums

    __device__ __forceinline__ int tiles_of(int g) const
    {
        if (g >= N) return 0;
        int lo, hi;
        group_rows(start, rows, g, lo, hi);
        return (hi - lo + BM - 1) / BM;
    }
    __device__ __forceinline__ void init(const LinearGemm &a)
    {
        start = a.start, N = a.N, rows = a.rows, col_tiles = a.col_tiles, lane = threadIdx.x & 63;
        cur_chunk = 0, cur_incl = LiveTileWalk<1>::scan(tiles_of(lane));
        const int first = __builtin_amdgcn_readlane(cur_incl, 63), chunks = (N + 63) / 64;
        chunk_incl = first;
        if (chunks > 1) {
            int mine = lane == 0 ? first : 0;
            for (int c0 = 1; c0 < chunks; c0 += 4) {
                int v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = tiles_of((c0 + u) * 64 + lane);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int sum = __builtin_amdgcn_readlane(LiveTileWalk<1>::scan(v[u]), 63);
                    if (lane == c0 + u) mine = sum;
                }
            }
            chunk_incl = LiveTileWalk<1>::scan(mine);
        }
        whole = __builtin_amdgcn_readlane(chunk_incl, 63) * col_tiles;
        tickets = whole * a.parts;
    }
    // the n-th tile of this workgroup; false behind its last
    __device__ __forceinline__ bool tile(const LinearGemm &a, int n, int tile_cols, LinearTile &t)
    {
        const int each = (tickets + 7) / 8, local = blockIdx.x / 8 + n * (gridDim.x / 8);
        int ticket = (blockIdx.x % 8) * each + local;
        if (local >= each || ticket >= tickets) return false;
        t.part = a.parts > 1 ? ticket / whole : 0;
        ticket -= t.part * whole;
        const int I = ticket / col_tiles;
        const int c = __builtin_ctzll(__ballot(chunk_incl > I));
        const int before = c ? __builtin_amdgcn_readlane(chunk_incl, c - 1) : 0;
        if (c != cur_chunk) cur_chunk = c, cur_incl = LiveTileWalk<1>::scan(tiles_of(c * 64 + lane));
        const int l = __builtin_ctzll(__ballot(before + cur_incl > I));
        const int first = before + (l ? __builtin_amdgcn_readlane(cur_incl, l - 1) : 0), cnt = before + __builtin_amdgcn_readlane(cur_incl, l) - first;
        int u = ticket - first * col_tiles;
        const int band = u / (BAND * col_tiles);
        u -= band * BAND * col_tiles;
        const int height = min(BAND, cnt - band * BAND), ct = u / height, rt = band * BAND + u - ct * height;
        int lo, hi;
        t.e = c * 64 + l;
        group_rows(start, rows, t.e, lo, hi);
        t.first = lo + rt * BM, t.rows = hi - t.first, t.col0 = ct * tile_cols;
        t.from = t.part * a.chunk, t.kv = a.parts > 1 ? min(a.chunk, a.K - t.from) : a.K;
        return true;
    }
};

// Tiles of the weights' gradient: every group's, or those of the parts of the groups' rows.  Rows are cut at the multiples of a.chunk and at the groups'
// ends; the part of group e in the b-th chunk has the number b + e, which grows along the rows, so that group and chunk follow from the number
// by a search over `start`.  Numbers that no part has are passed over.  Groups differ in their rows: the XCDs take runs of at most 16 tickets in turn.
template <int BM>
struct GradWalk {
    int per_part, tickets, run;

    __device__ __forceinline__ void init(const LinearGemm &a)
    {
        per_part = a.row_tiles * a.col_tiles;
        tickets = a.parts * per_part;
        run = max(1, min(16, (tickets + 7) / 8));
    }
    // number n of this workgroup's tickets: 1 a tile, 0 none here, -1 none from here on
    __device__ __forceinline__ int tile(const LinearGemm &a, int n, int tile_cols, LinearTile &t)
    {
        const int local = blockIdx.x / 8 + n * (gridDim.x / 8);
        const long long at = ((long long)(local / run) * 8 + blockIdx.x % 8) * run + local % run;
        if (at >= tickets) return (long long)(local / run) * 8 * run >= tickets ? -1 : 0;
        const int ticket = (int)at;
        t.part = ticket / per_part;
        const int u = ticket - t.part * per_part, ct = u / a.row_tiles, rt = u - ct * a.row_tiles;
        int lo, hi;
        if (a.chunk == 0) {
            t.e = t.part;
            group_rows(a.start, a.rows, t.e, lo, hi);
        } else {
            int e = 0, above = a.N;   // the last group whose first part has a number of at most t.part
            while (above - e > 1) {
                const int mid = (e + above) / 2;
                if (min(max(a.start[mid], 0), a.rows) / a.chunk + mid <= t.part) e = mid;
                else above = mid;
            }
            t.e = e;
            group_rows(a.start, a.rows, e, lo, hi);
            const long long begin = (long long)(t.part - e) * a.chunk;
            lo = (int)max((long long)lo, begin), hi = (int)min((long long)hi, begin + a.chunk);
            if (lo >= hi) return 0;
        }
        t.first = rt * BM, t.rows = a.Mrows - t.first, t.col0 = ct * tile_cols, t.from = lo, t.kv = hi - lo;
        return 1;
    }
};

// activation and derivative; ReLU hands NaN on.  EXACT: by erff (32-bit storage), else the rational form of the 16-bit paths
template <bool EXACT>
__device__ __forceinline__ float linear_act(int act, float v)
{
    if (act == 0) return v;
    if (act == 1) return v < 0.f ? 0.f : v;
    if constexpr (EXACT) return v < -40.f ? 0.f : activate<2>(v);   // (infinity times the tail's 0)
    else return activate<4>(v);
}
template <bool EXACT>
__device__ __forceinline__ float linear_act_grad(int act, float v)
{
    if (act == 0) return 1.f;
    if (act == 1) return v > 0.f ? 1.f : v <= 0.f ? 0.f : v;
    if (fabsf(v) > 40.f) return v > 0.f ? 1.f : 0.f;
    if constexpr (EXACT) return 0.5f * (1.0f + erff(v * 0.70710678118654752f)) + v * 0.3989422804014327f * expf(-0.5f * v * v);
    else return activate_grad<2>(v);
}

}  // namespace

}  // namespace smile
