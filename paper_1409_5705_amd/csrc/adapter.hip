// Factor blocks beside a shared projection (low-rank adapters of many requests): the contractions with the blocks.
//
//   project:  H[t][r] = scale_a sum_k X[t][k] F_a[r][k]            (a: the block of row t's request)
//   join:     out[t][n] = base[t][n] + sum_r H[t][r] F'_a[r][n]    (base: the product with the shared matrix)
//
// Rows of one matrix belong to different blocks, so what one row holds (an infinity, a NaN) never meets another row's sum:
// a product takes rows of ONE block at a time, and the others' results are dropped, not multiplied by zero.
#include "adapter_device.h"
#include "device.h"

#include <algorithm>

namespace sfb {
namespace {

constexpr int PW = 8;      // wavefronts (16, also for few workgroups: 14.5 and 14.2 us for 8 rows, K = 4096)

// fp32 rows: up to 16 of one request against the 16 RT factors 16 RT * blockIdx.y ..; the wavefronts share k.  What bounds it is
// how soon everything is on its way: a wavefront's loads of U k-steps are in flight together.
template <int RT>
__global__ __launch_bounds__(64 * PW) void adapter_project_kernel(ProjectParams p, unsigned windows, unsigned xcds)
{
    constexpr int CE = 4, STEP = 4 * CE, U = RT == 1 ? 8 : 4;
    __shared__ floatx4 part[PW][RT][64];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r0 = (int)blockIdx.y * 16 * RT;
    const AdapterRows& rows = p.rows;
    ProjectTile tile;
    if (!project_tile<16>(p, windows, xcds, r0, 16 * RT, tid, 64 * PW, lane, tile)) return;
    const int64_t t0 = tile.t0;
    const int n_rows = tile.rows, rank = tile.rank, a = tile.a;

    const int64_t steps = (p.K + STEP - 1) / STEP, per = (steps + PW - 1) / PW;
    const int64_t k_begin = wave * per * STEP, k_end = k_begin + per * STEP < p.K ? k_begin + per * STEP : p.K;
    const float* const x = static_cast<const float*>(p.X) + (t0 + (l16 < n_rows ? l16 : n_rows - 1)) * p.K + CE * quad;
    const float* f[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = r0 + 16 * i + l16;
        f[i] = static_cast<const float*>(p.F) + ((int64_t)a * rows.rank + (r < rank ? r : rank - 1)) * p.K + CE * quad;
    }
    floatx4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    // register i of lane (q, c) of an MFMA: factor 4 q + i, row c
    auto add = [](u32x4 fv, u32x4 xv, floatx4 sum) {
#pragma unroll
        for (int e = 0; e < CE; ++e)
            sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((uint32_t)fv[e]), __uint_as_float((uint32_t)xv[e]), sum, 0, 0, 0);
        return sum;
    };
    int64_t k = k_begin;
    for (; k + U * STEP <= k_end; k += U * STEP) {
        u32x4 xv[U], fv[U][RT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            xv[u] = load_chunk(x + k + u * STEP);
#pragma unroll
            for (int i = 0; i < RT; ++i) fv[u][i] = load_chunk(f[i] + k + u * STEP);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < RT; ++i) acc[i] = add(fv[u][i], xv[u], acc[i]);
    }
    for (; k < k_end; k += STEP) {
        const u32x4 xv = load_chunk(x, k, k_end - CE * quad);
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[i] = add(load_chunk(f[i], k, k_end - CE * quad), xv, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave >= RT) return;
    // wavefront i: factors 16 i ..
    floatx4 sum = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < PW; ++w) sum += part[w][wave][lane];
    store_projection(p, tile, t0 + l16, l16 < n_rows, r0 + 16 * wave + 4 * quad, sum);
}

// A thread: four columns of RW rows of the output, which read their block's factors once where it is the same one.  The rows'
// projections come from H, or (dense) from the planes, which hold the products with the factors of all blocks behind the
// columns of the output; then the first workgroup of a row stores them.
// PRE: so many factors of the row's block are on their way before its projections are known.
template <typename T, int RW, int PRE>
__global__ __launch_bounds__(128) void adapter_join_kernel(AdapterJoinArgs p, int blocks_n, int64_t t0)
{
    __shared__ float h_of[RW][256];
    __shared__ int a_of[RW], rank_at[RW];
    const int64_t t = t0 + (int64_t)(blockIdx.x / blocks_n) * RW, n = ((int64_t)(blockIdx.x % blocks_n) * 128 + threadIdx.x) * 4;
    const int live = p.N - n < 4 ? p.N - n < 0 ? 0 : (int)(p.N - n) : 4;
    const int64_t plane = p.T * p.width;
    // a row's block and projections are looked for by threads of its own
    constexpr int OF_ROW = 128 / RW;
    const int mine = RW == 1 ? 0 : threadIdx.x / OF_ROW, pitch = adapter_pitch(p.rank);
    const int64_t row = t + mine;
    const int of = RW == 1 || row < p.T ? p.row_adapter[row] : ROW_OUTSIDE;
    floatx4 v[RW];
    const float* src[RW];
#pragma unroll
    for (int j = 0; j < RW; ++j) {
        v[j] = floatx4{0.f, 0.f, 0.f, 0.f};
        src[j] = p.planes + (RW == 1 || t + j < p.T ? t + j : p.T - 1) * p.width + n;
    }
    if (live == 4) {
#pragma unroll 4
        for (int s = 0; s < p.split; ++s)
#pragma unroll
            for (int j = 0; j < RW; ++j) v[j] += __builtin_bit_cast(floatx4, load_chunk(src[j] + s * plane));
    } else {
        for (int s = 0; s < p.split; ++s)
#pragma unroll
            for (int j = 0; j < RW; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < live) v[j][e] += src[j][s * plane + e];
    }
    if (RW == 1 && of == ROW_OUTSIDE) return;
    // the factors that columns n .. n + 3 have for pair r
    auto factors = [&](const T* F, int r) {
        floatx4 f;
        if constexpr (sizeof(T) == 2) {      // (N % 8 == 0: all four columns)
            const u32x2 w = *reinterpret_cast<const u32x2*>(F + r * p.N);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        } else {
            f = __builtin_bit_cast(floatx4, load_chunk(F + r * p.N, 0, live));
        }
        return f;
    };
    static_assert(PRE == 0 || (RW == 1 && sizeof(T) == 2), "one row, four whole columns a thread");
    floatx4 pre[PRE > 0 ? PRE : 1];
    int its_rank = 0;
    if (of >= 0 && of < p.count) {
#pragma unroll
        for (int r = 0; r < PRE; ++r)
            pre[r] = factors(static_cast<const T*>(p.F) + (int64_t)of * p.rank * p.N + (live == 4 ? n : 0), r < p.rank ? r : p.rank - 1);
        its_rank = rank_of(p.ranks, p.rank, of);
        const float scale = p.scale ? p.scale[of] : 1.f;
        // (all of the row's, those that are not in use too: their number is still on its way)
        for (int r = threadIdx.x % OF_ROW; r < p.rank; r += OF_ROW) {
            float h;
            if (p.dense) {
                h = 0.f;
                const float* from = p.planes + row * p.width + p.N + (int64_t)of * p.rank + r;
#pragma unroll 4
                for (int s = 0; s < p.split; ++s) h += from[s * plane];
                h *= scale;
            } else {
                h = p.H[row * pitch + r];
            }
            h_of[mine][r] = h;
        }
        if (RW == 1) __syncthreads();
    }
    int a[RW], rank[RW];
    bool same = RW > 1;
    if constexpr (RW == 1) {
        a[0] = of;
        rank[0] = its_rank;
    } else {
        if (threadIdx.x % OF_ROW == 0) {
            a_of[mine] = of;
            rank_at[mine] = its_rank;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < RW; ++j) {
            a[j] = __builtin_amdgcn_readfirstlane(a_of[j]);
            rank[j] = __builtin_amdgcn_readfirstlane(rank_at[j]);
            same = same && a[j] == a[0];
        }
    }
    if (p.dense && blockIdx.x % blocks_n == 0 && of != ROW_OUTSIDE) {
        for (int r = threadIdx.x % OF_ROW; r < pitch; r += OF_ROW) {
            const float h = r < its_rank ? h_of[mine][r] : 0.f;
            p.H[row * pitch + r] = h;
            if (p.H_out && r < p.rank) p.H_out[row * p.rank + r] = h;
        }
    }
    if (live == 0) return;
    floatx4 low[RW];
#pragma unroll
    for (int j = 0; j < RW; ++j) low[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (same) {
        const T* const F = static_cast<const T*>(p.F) + (int64_t)a[0] * p.rank * p.N + n;
#pragma unroll 8
        for (int r = 0; r < rank[0]; ++r) {
            const floatx4 f = factors(F, r);
#pragma unroll
            for (int j = 0; j < RW; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) low[j][e] = fmaf(h_of[j][r], f[e], low[j][e]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < RW; ++j) {
            const T* const F = static_cast<const T*>(p.F) + (int64_t)a[j] * p.rank * p.N + n;
#pragma unroll
            for (int r = 0; r < PRE; ++r) {
                const float h = h_of[j][r];
#pragma unroll
                for (int e = 0; e < 4; ++e) low[j][e] = r < rank[j] ? fmaf(h, pre[r][e], low[j][e]) : low[j][e];
            }
#pragma unroll 8
            for (int r = PRE; r < rank[j]; ++r) {
                const floatx4 f = factors(F, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) low[j][e] = fmaf(h_of[j][r], f[e], low[j][e]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < RW; ++j) {
        if (a[j] == ROW_OUTSIDE) continue;
        if (rank[j] > 0) v[j] += low[j];
        T* const out = static_cast<T*>(p.out) + (t + j) * p.N + n;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x2*>(out) = u32x2{pack_bf16(v[j][0], v[j][1]), pack_bf16(v[j][2], v[j][3])};
        } else if (live == 4) {
            *reinterpret_cast<u32x4_by_word*>(out) = __builtin_bit_cast(u32x4, v[j]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < live) out[e] = v[j][e];
        }
    }
}

// dst [rows_out][cols_out] = src [rows][cols] and zeros behind it, for two matrices.
__global__ __launch_bounds__(256) void pad_kernel(AdapterPad a, AdapterPad b, int64_t blocks_a)
{
    const bool second = blockIdx.x >= blocks_a;
    const AdapterPad& m = second ? b : a;
    const int64_t i = ((int64_t)(second ? blockIdx.x - blocks_a : blockIdx.x) * 256 + threadIdx.x) * 4;      // (cols_out % 4 == 0)
    if (i >= m.rows_out * m.cols_out) return;
    const int64_t r = i / m.cols_out, c = i % m.cols_out;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (r < m.rows) v = load_chunk(m.src + r * m.cols, c, m.cols);
    *reinterpret_cast<u32x4*>(m.dst + i) = v;
}

}  // namespace

hipError_t launch_adapter_project(const AdapterProjectArgs& a, DeviceInfo& dev, hipStream_t stream)
{
    if (a.rows.T <= 0) return hipSuccess;
    const ProjectParams p = {a.rows, a.X, a.F, a.K, a.row_adapter, a.H, a.H_out, a.Hx, adapter_pitch(a.rows.rank)};
    if (a.bf16) return launch_adapter_project_tiles(p, dev, stream);
    const int64_t windows = (p.rows.T + 15) / 16, tiles = windows + p.rows.requests;
    const int rt = project_factors(tiles, p.pitch, dev);
    const dim3 grid((unsigned)tiles, (unsigned)std::max(1, (p.pitch + 16 * rt - 1) / (16 * rt)));
    const unsigned xcds = dev.xcds > 0 ? dev.xcds : 1;
    if (rt == 1)
        adapter_project_kernel<1><<<grid, 64 * PW, 0, stream>>>(p, (unsigned)windows, xcds);
    else if (rt == 2)
        adapter_project_kernel<2><<<grid, 64 * PW, 0, stream>>>(p, (unsigned)windows, xcds);
    else
        adapter_project_kernel<4><<<grid, 64 * PW, 0, stream>>>(p, (unsigned)windows, xcds);
    return hipGetLastError();
}

hipError_t launch_adapter_pad(const AdapterPad& a, const AdapterPad& b, hipStream_t stream)
{
    const int64_t blocks_a = (a.rows_out * a.cols_out + 1023) / 1024, blocks = blocks_a + (b.rows_out * b.cols_out + 1023) / 1024;
    if (blocks == 0) return hipSuccess;
    pad_kernel<<<(unsigned)blocks, 256, 0, stream>>>(a, b, blocks_a);
    return hipGetLastError();
}

template <typename T, int RW, int PRE>
static hipError_t join_rows(const AdapterJoinArgs& a, hipStream_t stream)
{
    const int blocks_n = (int)((a.N + 511) / 512);
    const int64_t groups = (a.T + RW - 1) / RW, most = std::max<int64_t>(1, MAX_BLOCKS / blocks_n);
    for (int64_t g = 0; g < groups; g += most) {
        const unsigned blocks = (unsigned)(std::min(most, groups - g) * blocks_n);
        adapter_join_kernel<T, RW, PRE><<<blocks, 128, 0, stream>>>(a, blocks_n, g * RW);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_adapter_join(const AdapterJoinArgs& a, hipStream_t stream)
{
    if (a.T <= 0) return hipSuccess;
    // Two rows a workgroup where there are eight workgroups and more a compute unit: what the L2s give bounds it then, the factors
    // most of it (fp32, 64 pairs: 2000 rows, 4096 columns 76 us and with two 47; 300 rows, 1024 columns 11 and 15).
    const bool two = a.T * ((a.N + 511) / 512) >= 2048;
    if (!a.bf16) return two ? join_rows<float, 2, 0>(a, stream) : join_rows<float, 1, 0>(a, stream);
    if (two) return join_rows<uint16_t, 2, 0>(a, stream);
    // 16 factors ahead, for rows with 9 to 15 pairs in use: the loop takes eight at a time and what is left one after another.  us of a
    // call with / without: 64 rows, 4096 x 4096, 12 pairs 20.1 / 21.2, 8 to 16 of them 17.5 / 18.5, 16 20.2 / 20.3, 32 22.0 / 22.0, 64 25.7
    // / 25.5; 64 rows, 2048 x 4096, 12 pairs 17.1 / 18.3; one row, 1024 x 1024, 8 pairs 8.0 / 7.5, 16 8.0 / 7.7, 256 15.4 / 15.0.
    return a.rank > 8 ? join_rows<uint16_t, 1, 16>(a, stream) : join_rows<uint16_t, 1, 0>(a, stream);
}

}  // namespace sfb
