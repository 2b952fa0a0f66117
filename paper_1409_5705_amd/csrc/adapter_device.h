// Device functions of the adapter calls' kernels.
#pragma once
#include "adapter.h"
#include "planes.h"

namespace sfb {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int64_t MAX_BLOCKS = 1 << 22;      // workgroups of a launch (threads of a grid are counted in 32 bits)

// 16 bytes of a row (eight bf16, four fp32).  fp32 rows need not be 16-byte aligned.
typedef u32x4 u32x4_by_word __attribute__((aligned(4)));
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const T* p)
{
    return *reinterpret_cast<const u32x4_by_word*>(p);
}
// The same from element k of a row on; what lies at or behind `end` is zero (bf16: a multiple of eight).
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const T* row, int64_t k, int64_t end)
{
    u32x4 v = {0u, 0u, 0u, 0u};
    if (k + 16 / (int)sizeof(T) <= end) return load_chunk(row + k);
    if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k + e < end) v[e] = *reinterpret_cast<const uint32_t*>(row + k + e);
    }
    return v;
}

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;

// A buffer descriptor of 2 GiB from base on (raw bytes; reads beyond it give zeros).
__device__ __forceinline__ u32x4 descriptor(uint64_t at)
{
    const uint64_t base = uniform64(at);
    return u32x4{(uint32_t)base, (uint32_t)(base >> 32), OUT_OF_RANGE, 0x00020000u};
}
template <uint32_t OFF>
__device__ __forceinline__ void buffer_to_lds_16(uint32_t lds_addr, u32x4 rsrc, uint32_t voff)
{
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(voff), "s"(rsrc), "n"(OFF)
                 : "memory", "scc");
}

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
// Factors of a workgroup, in MFMA tiles of 16: as few as give every compute unit a
// workgroup (64 pairs, K = 4096: 700 rows 22 us with 64 a workgroup, 13 with 16; 8192 rows 27, with 16 and 32 31; fp32, 8 rows 37
// and 14).
inline int project_factors(int64_t tiles, int pitch, const DeviceInfo& dev)
{
    int rt = 1;
    while (rt < 4 && 16 * rt < pitch && tiles * ((pitch + 16 * rt - 1) / (16 * rt)) > dev.cus) rt *= 2;
    return rt;
}

// Two bf16 terms of a value: its upper half as it is and what is left, rounded; one that is not finite as itself twice.  Together
// they are off by at most 2^-16 of the value (what is left is below 2^-7 of it and keeps eight bits; 1 + 2^-8 + 2^-16 is off by
// that) and both of its sign: where products with them overflow they do so to the same side.  The first term rounded would halve
// the error and lose that.
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
                                                 floatx4 sum)
{
    if (!in || r >= p.pitch) return;
    const float s = p.rows.scale ? p.rows.scale[tile.a] : 1.f;
    float h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = r + e < tile.rank ? s * sum[e] : 0.f;
    *reinterpret_cast<floatx4*>(p.H + t * p.pitch + r) = floatx4{h[0], h[1], h[2], h[3]};
    if (p.Hx) {
        uint16_t first[4], second[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) two_terms(h[e], first[e], second[e]);
        uint16_t* const at = p.Hx + t * 2 * p.pitch + term_at(r);
        *reinterpret_cast<u32x2*>(at) = u32x2{(uint32_t)first[0] | (uint32_t)first[1] << 16, (uint32_t)first[2] | (uint32_t)first[3] << 16};
        *reinterpret_cast<u32x2*>(at + 16) = u32x2{(uint32_t)second[0] | (uint32_t)second[1] << 16, (uint32_t)second[2] | (uint32_t)second[3] << 16};
    }
    if (p.H_out) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (r + e < p.rows.rank) p.H_out[t * p.rows.rank + r + e] = h[e];
    }
}

}  // namespace sfb
