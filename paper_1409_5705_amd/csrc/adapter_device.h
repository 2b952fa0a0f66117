// Device functions of the adapter calls' kernels.
#pragma once
#include "adapter.h"
#include "device.h"

namespace sfb {

// The request of row t, or -1 (empty requests are passed over: the last q with start[q] <= t).  By a whole wavefront: 64
// probes a step.
__device__ __forceinline__ int64_t request_of(const int64_t* start, int64_t requests, int64_t t, int lane)
{
    if (requests <= 0 || t < start[0] || t >= start[requests]) return -1;
    int64_t lo = 0, n = requests;                  // start[lo] <= t; the answer is in [lo, lo + n)
    while (n > 1) {
        const int64_t step = (n + 63) / 64, at = lane * step;
        const uint64_t below = __builtin_amdgcn_ballot_w64(at < n && start[lo + at] <= t);
        const int64_t k = 63 - __builtin_clzll(below | 1);
        lo += k * step;
        n = n - k * step < step ? n - k * step : step;
    }
    return lo;
}
__device__ __forceinline__ int rank_of(const int32_t* ranks, int rank, int64_t a)
{
    const int r = ranks ? ranks[a] : rank;
    return r < 0 ? 0 : r < rank ? r : rank;
}

struct ProjectParams {
    AdapterRows rows;
    const void* X;
    const void* F;
    int64_t K;
    int32_t* row_adapter;
    float* H;
    float* H_out;
    uint16_t* Hx;
    int pitch;
};
hipError_t launch_adapter_project_tiles(const ProjectParams& p, DeviceInfo& dev, hipStream_t stream);

// Two bf16 terms of a value: its upper half as it is and what is left, rounded (together off by at most 2^-17 of the value, and
// of its sign); one that is not finite as itself twice.
__device__ __forceinline__ void two_terms(float v, uint16_t& first, uint16_t& second)
{
    const uint32_t bits = __float_as_uint(v);
    const bool finite = (~bits & 0x7f800000u) != 0;
    first = (uint16_t)(finite ? bits >> 16 : pack_bf16(v, 0.f));
    second = (uint16_t)pack_bf16(finite ? v - __uint_as_float(bits & 0xffff0000u) : v, 0.f);
}
// Place of pair r's first term in a row of the two-term array; the second one is 16 further.
__device__ __forceinline__ int term_at(int r) { return (r >> 4) * 32 + (r & 15); }

// The rows of a workgroup: up to R of one request.  Workgroup w < windows takes the rows from R w on, workgroup windows + q those
// from the first row of request q on, both to the next multiple of R or to the end of their request: every row once, and never
// two blocks in a workgroup.  (Tiles of 32 rows whatever the requests, gone through once for every block in them: 8192 rows in
// 24 requests, K = 4096, 64 pairs 62 us.)  Neighbours, which are likely to use the same factors, go to the same XCD.
// Writes row_adapter.  False: nothing is left to do for the factors r0 .. r0 + width - 1 (those that are not there are zeros).
struct ProjectTile {
    int64_t t0;
    int rows, a, rank;
};
template <int R>
__device__ __forceinline__ bool project_tile(const ProjectParams& p, unsigned windows, unsigned xcds, int r0, int width, int tid, int threads, int lane,
                                             ProjectTile& tile)
{
    const AdapterRows& rows = p.rows;
    unsigned w = blockIdx.x;
    {
        const unsigned first = w < windows ? 0 : windows, count = first ? gridDim.x - windows : windows;
        const unsigned whole = count / xcds * xcds, i = w - first;
        if (i < whole) w = first + i % xcds * (whole / xcds) + i / xcds;
    }
    int64_t t0, q;
    if (w < windows) {
        t0 = (int64_t)w * R;
        const int64_t t = t0 + tid;
        if (tid < R && r0 == 0 && t < rows.T && (t < rows.start[0] || t >= rows.start[rows.requests])) p.row_adapter[t] = ROW_OUTSIDE;
        q = request_of(rows.start, rows.requests, t0, lane);
        if (q < 0) return false;
    } else {
        q = w - windows;
        t0 = rows.start[q];
        if (t0 < 0 || t0 >= rows.T || (t0 & (R - 1)) == 0) return false;
    }
    int64_t t1 = (t0 | (R - 1)) + 1;
    if (rows.start[q + 1] < t1) t1 = rows.start[q + 1];
    if (rows.T < t1) t1 = rows.T;
    const int n_rows = (int)(t1 - t0);
    if (n_rows <= 0) return false;
    int a = rows.adapter[q];
    const int rank = a < 0 || a >= rows.count ? 0 : rank_of(rows.ranks, rows.rank, a);
    if (rank == 0) a = ROW_NONE;
    if (r0 == 0 && tid < n_rows) p.row_adapter[t0 + tid] = a;
    if (r0 >= rank) {
        for (int i = tid; i < n_rows * width; i += threads) {
            const int64_t t = t0 + i / width;
            const int r = r0 + i % width;
            if (r < p.pitch) {
                p.H[t * p.pitch + r] = 0.f;
                if (p.Hx) p.Hx[t * 2 * p.pitch + term_at(r)] = p.Hx[t * 2 * p.pitch + term_at(r) + 16] = 0;
            }
            if (p.H_out && r < rows.rank) p.H_out[t * rows.rank + r] = 0.f;
        }
        return false;
    }
    tile = ProjectTile{t0, n_rows, __builtin_amdgcn_readfirstlane(a), __builtin_amdgcn_readfirstlane(rank)};
    return true;
}

// Row t's projections on the factors r .. r + 3 from their sums (in: whether the lane has such a row).
__device__ __forceinline__ void store_projection(const ProjectParams& p, const ProjectTile& tile, int64_t t, bool in, int r,
                                                 float __attribute__((ext_vector_type(4))) sum)
{
    if (!in || r >= p.pitch) return;
    const float s = p.rows.scale ? p.rows.scale[tile.a] : 1.f;
    float h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = r + e < tile.rank ? s * sum[e] : 0.f;
    typedef float vec4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<vec4*>(p.H + t * p.pitch + r) = vec4{h[0], h[1], h[2], h[3]};
    if (p.Hx) {
        uint16_t first[4], second[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) two_terms(h[e], first[e], second[e]);
        uint16_t* const at = p.Hx + t * 2 * p.pitch + term_at(r);
        *reinterpret_cast<uint2*>(at) = uint2{(uint32_t)first[0] | (uint32_t)first[1] << 16, (uint32_t)first[2] | (uint32_t)first[3] << 16};
        *reinterpret_cast<uint2*>(at + 16) = uint2{(uint32_t)second[0] | (uint32_t)second[1] << 16, (uint32_t)second[2] | (uint32_t)second[3] << 16};
    }
    if (p.H_out) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (r + e < p.rows.rank) p.H_out[t * p.rows.rank + r + e] = h[e];
    }
}

}  // namespace sfb
