// The gradients of factor blocks:  out[a][r][c] = sum over the rows t of block a of H[t][r] G[t][c],  two such sums at once.
//
// A block's rows are listed from row_adapter, so requests that share a block, of whatever lengths, are one sum in the order of
// the rows; where blocks are few the rows are divided over workgroups and a second launch adds up the parts in their order.
// What bounds it is the stream of G.
#include "adapter_device.h"

#include <algorithm>

namespace sfb {
namespace {

constexpr int OW = 8, WINDOW = 4096;      // wavefronts; rows of which one list is made at most

struct OuterParams {
    AdapterOuter sum[2];
    const int32_t* row_adapter;
    const int32_t* ranks;
    int64_t count;
    int rank;
    const int64_t* start;      // of the requests, where a block's rows are looked for by them (requests > 0)
    const int32_t* adapter;
    int64_t requests;
    int64_t T, per;            // rows, rows of a split (a multiple of eight)
    unsigned tiles0, tiles;
    int64_t first;             // workgroups of the launches before
    int window;                // rows of a list (bf16: their offsets in G have 31 bits)
    float* partial;            // with splits: [split][count][rank][C of the first + C of the second]
};

// What a workgroup sums: a tile of `width` columns and 16 RT factors of one block's gradient, over `per` rows of the matrix.
struct OuterTile {
    const AdapterOuter* sum;
    int a, r0, rank;
    int64_t c0, t_begin, t_end;
    float* out;                // factor 0, column 0 of the block's gradient (or of its part)
};
__device__ __forceinline__ OuterTile outer_tile(const OuterParams& p, int width, int factors)
{
    OuterTile t;
    const unsigned tile = (unsigned)((p.first + blockIdx.x) % p.tiles);
    const int64_t block = (p.first + blockIdx.x) / p.tiles;
    const bool second = tile >= p.tiles0;
    t.sum = &p.sum[second ? 1 : 0];
    t.a = (int)(block % p.count);
    t.r0 = (int)(block / p.count) * factors;
    t.rank = rank_of(p.ranks, p.rank, t.a);
    t.c0 = (int64_t)(second ? tile - p.tiles0 : tile) * width;
    t.t_begin = (int64_t)blockIdx.y * p.per;
    t.t_end = t.t_begin + p.per < p.T ? t.t_begin + p.per : p.T;
    t.out = p.partial ? p.partial + ((int64_t)blockIdx.y * p.count + t.a) * p.rank * (p.sum[0].C + p.sum[1].C) + (second ? p.rank * p.sum[0].C : 0)
                      : t.sum->out + (int64_t)t.a * p.rank * t.sum->C;
    return t;
}

// Cuts the tile's rows down to those between the first and the last one of its block's requests: a window without any costs
// 3 us (8192 rows, 4096 + 4096 columns, 16 pairs: 16 blocks 47 us without and 34 with it and lists made from 16-byte loads, 64
// blocks 110 and 60; 32768 rows, 64 blocks, 1024 + 1024 columns 93 and 36).  counts: 2 OW.
__device__ __forceinline__ void narrow_rows(const OuterParams& p, OuterTile& tile, int* counts)
{
    if (p.requests == 0) return;
    const int tid = threadIdx.x, wave = tid >> 6;
    int lo = 0x7fffffff, hi = 0;      // (T is below 2^24)
    for (int64_t q = tid; q < p.requests; q += 64 * OW) {
        if (p.adapter[q] != tile.a) continue;
        const int64_t s = p.start[q], e = p.start[q + 1] < p.T ? p.start[q + 1] : p.T, b = s > 0 ? s : 0;
        if (b >= e) continue;
        lo = (int)b < lo ? (int)b : lo;
        hi = (int)e > hi ? (int)e : hi;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const int l = __shfl_xor(lo, d), h = __shfl_xor(hi, d);
        lo = l < lo ? l : lo;
        hi = h > hi ? h : hi;
    }
    if ((tid & 63) == 0) {
        counts[wave] = lo;
        counts[OW + wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < OW; ++w) {
        lo = counts[w] < lo ? counts[w] : lo;
        hi = counts[OW + w] > hi ? counts[OW + w] : hi;
    }
    __syncthreads();
    lo = __builtin_amdgcn_readfirstlane(lo) & ~7;
    hi = __builtin_amdgcn_readfirstlane(hi);
    if (lo > tile.t_begin) tile.t_begin = lo;
    if (hi < tile.t_end) tile.t_end = hi;
}

// The rows of the window from w0 on (a multiple of eight) that belong to the block, in their order, as offsets from w0; their
// number.  (What follows row_adapter up to a multiple of eight may be read.)
__device__ __forceinline__ int list_rows(const OuterParams& p, const OuterTile& tile, int64_t w0, uint16_t* list, int* counts)
{
    constexpr int PER = WINDOW / (64 * OW);
    static_assert(PER == 8, "two loads of 16 bytes");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int found = 0;
    uint32_t bits = 0;
    const int64_t t0 = w0 + tid * PER;
    if (tid * PER < p.window && t0 < tile.t_end) {      // (the window is a multiple of 64)
        const u32x4* const at = reinterpret_cast<const u32x4*>(p.row_adapter + t0);
        const u32x4 v[2] = {at[0], at[1]};
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (t0 + i < tile.t_end && (int)v[i >> 2][i & 3] == tile.a) {
                bits |= 1u << i;
                ++found;
            }
        }
    }
    int before = found;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(before, d);
        if (lane >= d) before += o;
    }
    if (lane == 63) counts[wave] = before;
    before -= found;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < OW; ++w) {
        const int c = counts[w];
        if (w < wave) before += c;
        total += c;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (bits >> i & 1) list[before++] = (uint16_t)(tid * PER + i);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(total);
}

// The sums of a tile on the fp32 matrix pipes.  The wavefronts take four rows of the block at a time: the MFMA's k.  Both
// operands come from memory in the lanes' own order: lane (q, c) loads 16 bytes of row q, columns CE c .. , which are the columns
// CE c + f of MFMA f.  part: OW x CE x 64.
template <typename T, int RT>
__device__ __forceinline__ void outer_fp32(const OuterParams& p, const OuterTile& tile, uint16_t* list, int* counts, floatx4* part)
{
    constexpr int CE = 16 / (int)sizeof(T), U = RT == 1 ? 8 : 4;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const AdapterOuter& sum = *tile.sum;
    const int64_t c0 = tile.c0 + CE * l16;
    floatx4 acc[RT][CE];
#pragma unroll
    for (int f = 0; f < RT; ++f)
#pragma unroll
        for (int e = 0; e < CE; ++e) acc[f][e] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int64_t w0 = tile.t_begin; w0 < tile.t_end && tile.r0 < tile.rank; w0 += p.window) {
        const int total = list_rows(p, tile, w0, list, counts);
        for (int i0 = wave * 4 * U; i0 < total; i0 += OW * 4 * U) {
            u32x4 g[U];
            float h[U][RT];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + 4 * u + quad;
                const bool in = i < total;
                const int64_t t = w0 + list[in ? i : 0];
                g[u] = u32x4{0u, 0u, 0u, 0u};
                if (in) g[u] = load_chunk(static_cast<const T*>(sum.G) + t * sum.C, c0, sum.C);
#pragma unroll
                for (int f = 0; f < RT; ++f) {
                    const int r = tile.r0 + 16 * f + l16;
                    h[u][f] = in && r < tile.rank ? sum.H[t * sum.ldh + r] : 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < CE; ++e) {
                    const uint32_t w = g[u][sizeof(T) == 2 ? e >> 1 : e];
                    const float ge = __uint_as_float(sizeof(T) == 4 ? w : (e & 1) ? w & 0xffff0000u : w << 16);
#pragma unroll
                    for (int f = 0; f < RT; ++f) acc[f][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(h[u][f], ge, acc[f][e], 0, 0, 0);
                }
        }
        __syncthreads();
    }
    // register i of lane (q, c): factor 4 q + i, column CE c + e of acc[.][e]
#pragma unroll
    for (int f = 0; f < RT; ++f) {
#pragma unroll
        for (int e = 0; e < CE; ++e) part[(wave * CE + e) * 64 + lane] = acc[f][e];
        __syncthreads();
        for (int e = wave; e < CE; e += OW) {
            floatx4 s = part[e * 64 + lane];
#pragma unroll
            for (int w = 1; w < OW; ++w) s += part[(w * CE + e) * 64 + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = tile.r0 + 16 * f + 4 * quad + i;
                if (r < p.rank && c0 + e < sum.C) tile.out[(int64_t)r * sum.C + c0 + e] = r < tile.rank ? s[i] : 0.f;
            }
        }
        __syncthreads();
    }
}

template <int RT>
__global__ __launch_bounds__(64 * OW, 4) void adapter_outer_f32_kernel(OuterParams p)
{
    __shared__ uint16_t list[WINDOW];
    __shared__ int counts[2 * OW];
    __shared__ floatx4 part[OW * 4 * 64];
    OuterTile tile = outer_tile(p, 64, 16 * RT);
    narrow_rows(p, tile, counts);
    outer_fp32<float, RT>(p, tile, list, counts, part);
}

// bf16 rows: tiles of 128 columns, 64 rows of the block at a time, on the bf16 matrix pipes.  A value of H is three bf16 terms
// (24 bits: exact), so every product is exact and the sums are those of fp32 products; on the fp32 pipes, at a sixteenth of the
// rate, 8192 rows in 16 blocks with 64 pairs of 4096 + 4096 columns took 122 us and with 16 pairs 64; here 54 and 34 (G alone at
// the rate of a copy: 28).  G and H come row by row straight into
// LDS, PS stages of them; G is read with the transposing LDS read, H value by value and cut into its terms in registers.
// A sum that is not finite may come of an infinity met by a zero term: the tile is then made once more in fp32.
// Wavefront w: columns 32 (w % 4) .. of the tile, rows 32 (w / 4) .. of the 64.
constexpr int outer_stages(int rt) { return rt == 4 ? 2 : 3; }
constexpr uint32_t outer_stage_bytes(int rt) { return 64 * 256 + 64 * 64 * (uint32_t)rt; }
constexpr uint32_t outer_lds(int rt)
{
    const uint32_t ring = outer_stages(rt) * outer_stage_bytes(rt) + (rt == 1 ? 1024 : 0), part = OW * 8 * 64 * 16;
    return (ring > part ? ring : part) + WINDOW * 2;      // (two workgroups a CU)
}
template <int RT>
__global__ __launch_bounds__(64 * OW, 4) void adapter_outer_bf16_kernel(OuterParams p)
{
    constexpr int PS = outer_stages(RT), HL = RT == 4 ? 2 : 1, LOADS = 2 + HL;
    constexpr uint32_t STAGE_BYTES = outer_stage_bytes(RT), G_BYTES = 64 * 256, NOWHERE = PS * STAGE_BYTES;
    extern __shared__ u32x4 smem[];
    char* const lds = reinterpret_cast<char*>(smem);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    uint16_t* const list = reinterpret_cast<uint16_t*>(lds + outer_lds(RT) - WINDOW * 2);
    int* const counts = reinterpret_cast<int*>(lds);      // (used while nothing is on its way into the stages)
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    OuterTile tile = outer_tile(p, 128, 16 * RT);
    narrow_rows(p, tile, counts);
    const AdapterOuter& sum = *tile.sum;

    // G's rows of 256 bytes, 16-byte chunk u of row r in slot u ^ 4 (r % 4): a load is four rows.  H's rows of RT pieces of 64 bytes:
    // row r in place 4 (r % 8) + r / 8 of its 32, and the pieces of a row dealt so that the four rows 8 q + j that a read takes
    // lie in different banks; a load is 16 pieces.
    uint32_t g_off[2], h_off[HL];
    int g_row[2], h_row[HL];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        g_row[i] = 4 * (2 * wave + i) + quad;
        const int u = l16 ^ ((g_row[i] & 3) << 2);
        g_off[i] = tile.c0 + 8 * u < sum.C ? (uint32_t)u * 16u : OUT_OF_RANGE;
    }
    auto piece = [](int pos, int f) { return RT == 4 ? f ^ (pos & 3) : RT == 2 ? f ^ ((pos >> 1) & 1) : f; };
#pragma unroll
    for (int i = 0; i < HL; ++i) {
        const int slot = (HL * wave + i) * 16 + (lane >> 2), pos = slot / RT, f = piece(pos, slot % RT);
        h_row[i] = (pos & 32) + ((pos & 31) >> 2) + ((pos & 3) << 3);
        h_off[i] = (RT > 1 || wave < 4) && tile.r0 + 16 * f + 4 * (lane & 3) < sum.ldh ? (uint32_t)(tile.r0 + 16 * f + 4 * (lane & 3)) * 4u : OUT_OF_RANGE;
    }
    floatx4 acc[RT][2];
#pragma unroll
    for (int f = 0; f < RT; ++f)
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[f][c] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int wc = wave & 3, ks = wave >> 2;
    for (int64_t w0 = tile.t_begin; w0 < tile.t_end && tile.r0 < tile.rank; w0 += p.window) {
        const int total = list_rows(p, tile, w0, list, counts);
        const int slices = (total + 63) / 64;
        const uint64_t gg = uniform64(reinterpret_cast<uint64_t>(sum.G) + (uint64_t)(w0 * sum.C + tile.c0) * 2u);
        const uint64_t gh = uniform64(reinterpret_cast<uint64_t>(sum.H) + (uint64_t)(w0 * sum.ldh) * 4u);
        auto issue = [&](int s) {      // (past the last row: nothing is in range)
            const uint32_t stage = lds_base + (uint32_t)(s % PS) * STAGE_BYTES;
            static_for<0, 2>([&](auto I) {
                constexpr int i = decltype(I)::value;
                const int e = 64 * s + g_row[i];
                const uint32_t t = e < total ? list[e] : 0u;
                buffer_to_lds_16<i * 1024u>(stage + (uint32_t)(2 * wave) * 1024u, descriptor(gg),
                                            e < total && g_off[i] != OUT_OF_RANGE ? t * (uint32_t)(sum.C * 2) + g_off[i] : OUT_OF_RANGE);
            });
            static_for<0, HL>([&](auto I) {
                constexpr int i = decltype(I)::value;
                const int e = 64 * s + h_row[i];
                const uint32_t t = e < total ? list[e] : 0u;
                const uint32_t at = RT > 1 || wave < 4 ? stage + G_BYTES + (uint32_t)(HL * wave + i) * 1024u : lds_base + NOWHERE;
                buffer_to_lds_16<0>(at, descriptor(gh), e < total && h_off[i] != OUT_OF_RANGE ? t * (uint32_t)(sum.ldh * 4) + h_off[i] : OUT_OF_RANGE);
            });
        };
        for (int s = 0; s < PS - 1; ++s) issue(s);
        for (int s = 0; s < slices; ++s) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS * (PS - 2)) : "memory");
            __syncthreads();                               // slice s is in LDS; every wavefront has read the slice before
            issue(s + PS - 1);
            const char* const stage = lds + (uint32_t)(s % PS) * STAGE_BYTES;
            bf16x8 g[2];
            const int row = 32 * ks + 8 * quad + (l16 >> 2), u = 4 * wc + ((l16 & 3) >> 1);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const char* const at = stage + row * 256 + (((u + 2 * c) ^ ((row & 3) << 2)) << 4) + (l16 & 1) * 8;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * 256));
                g[c] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
#pragma unroll
            for (int f = 0; f < RT; ++f) {
                uint32_t h[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int pos = 32 * ks + 4 * j + quad;
                    h[j] = *reinterpret_cast<const uint32_t*>(stage + G_BYTES + (pos * RT + piece(pos, f)) * 64 + l16 * 4);
                }
                u32x4 term[3];
#pragma unroll
                for (int k = 0; k < 3; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        term[k][j] = pack_hi(h[2 * j], h[2 * j + 1]);
                        if (k < 2) {
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                h[2 * j + e] = __float_as_uint(__uint_as_float(h[2 * j + e]) - __uint_as_float(h[2 * j + e] & 0xffff0000u));
                        }
                    }
#pragma unroll
                for (int k = 2; k >= 0; --k)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, term[k]), g[c], acc[f][c], 0, 0, 0);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    // register i of lane (q, c) of acc[f][d]: factor 16 f + 4 q + i, column 32 wc + 16 d + c
    floatx4* const part = reinterpret_cast<floatx4*>(lds);
    if (ks == 1) {
#pragma unroll
        for (int f = 0; f < RT; ++f)
#pragma unroll
            for (int c = 0; c < 2; ++c) part[((wc * RT + f) * 2 + c) * 64 + lane] = acc[f][c];
    }
    __syncthreads();
    int bad = 0;
    if (ks == 0) {
#pragma unroll
        for (int f = 0; f < RT; ++f)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const floatx4 v = acc[f][c] + part[((wc * RT + f) * 2 + c) * 64 + lane];
                const int64_t col = tile.c0 + 32 * wc + 16 * c + l16;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = tile.r0 + 16 * f + 4 * quad + i;
                    if (r >= p.rank || col >= sum.C) continue;
                    if (r < tile.rank && (~__float_as_uint(v[i]) & 0x7f800000u) == 0) bad = 1;
                    tile.out[(int64_t)r * sum.C + col] = r < tile.rank ? v[i] : 0.f;
                }
            }
    }
    if (__syncthreads_or(bad) == 0) return;
#pragma unroll 1
    for (int f = 0; f < RT; ++f) {
        OuterTile one = tile;
        one.r0 += 16 * f;
        if (one.r0 < tile.rank) outer_fp32<uint16_t, 1>(p, one, list, counts, part);
    }
}

// dst[t][0 .. pitch) = src[t][0 .. rank) and zeros.
__global__ __launch_bounds__(256) void pad_projections_kernel(const float* src, float* dst, int rank, int pitch, int64_t total)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / pitch;
        const int r = (int)(i % pitch);
        dst[i] = r < rank ? src[t * rank + r] : 0.f;
    }
}

// Adds the splits' sums up, in their order.
__global__ __launch_bounds__(256) void adapter_outer_join_kernel(OuterParams p, int splits)
{
    const int64_t first = p.rank * p.sum[0].C, all = first + p.rank * p.sum[1].C, total = p.count * all;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        float v = p.partial[i];
        for (int s = 1; s < splits; ++s) v += p.partial[s * total + i];
        const int64_t a = i / all, at = i % all;
        if (at < first)
            p.sum[0].out[a * first + at] = v;
        else
            p.sum[1].out[a * (all - first) + at - first] = v;
    }
}

int outer_rt(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : 4; }
int64_t outer_blocks(int64_t C0, int64_t C1, int64_t count, int rank, bool bf16)
{
    const int64_t width = 16 * (bf16 ? 8 : 4), rt = outer_rt(rank);
    return ((C0 + width - 1) / width + (C1 + width - 1) / width) * count * ((rank + 16 * rt - 1) / (16 * rt));
}

template <int RT>
hipError_t outer_start(const OuterParams& p, dim3 blocks, bool bf16, DeviceInfo& dev, hipStream_t stream)
{
    if (!bf16) {
        adapter_outer_f32_kernel<RT><<<blocks, 64 * OW, 0, stream>>>(p);
        return hipGetLastError();
    }
    bool& set = dev.adapter_outer_lds_set[RT == 1 ? 0 : RT == 2 ? 1 : 2];
    if (!set) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&adapter_outer_bf16_kernel<RT>), hipFuncAttributeMaxDynamicSharedMemorySize, outer_lds(RT));
        if (e != hipSuccess) return e;
        set = true;
    }
    adapter_outer_bf16_kernel<RT><<<blocks, 64 * OW, outer_lds(RT), stream>>>(p);
    return hipGetLastError();
}
hipError_t outer_rank(OuterParams p, int splits, bool bf16, DeviceInfo& dev, hipStream_t stream)
{
    const int rt = outer_rt(p.rank);
    const int64_t workgroups = (int64_t)p.tiles * p.count * ((p.rank + 16 * rt - 1) / (16 * rt));
    for (p.first = 0; p.first < workgroups; p.first += MAX_BLOCKS) {
        const dim3 blocks((unsigned)std::min(MAX_BLOCKS, workgroups - p.first), (unsigned)splits);
        const hipError_t e = rt == 1 ? outer_start<1>(p, blocks, bf16, dev, stream)
                             : rt == 2 ? outer_start<2>(p, blocks, bf16, dev, stream)
                                       : outer_start<4>(p, blocks, bf16, dev, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

// Parts of the rows: as many workgroups as the chip takes (ranks up to 32 one a CU: 8192 rows, one block of 16 pairs of 4096 + 4096
// columns 86 us in one part, 33 in four, 36 in eight; more two: of 64 pairs 162, 55 and 50), and of a block, were all equal, 256
// rows at least (2048 rows, 8 blocks, 1024 + 1024 columns: one part 11 us, two 14).
int adapter_outer_splits(int64_t C0, int64_t C1, int64_t count, int rank, bool bf16, int64_t T)
{
    if (count <= 0 || T <= 0) return 1;
    const int64_t blocks = outer_blocks(C0, C1, count, rank, bf16), target = rank <= 32 ? 256 : 512;
    const int64_t s = std::min((target + blocks - 1) / blocks, T / (256 * count));
    return s < 2 ? 1 : s > 16 ? 16 : (int)s;
}

hipError_t launch_adapter_outer(const AdapterOuterArgs& a, DeviceInfo& dev, hipStream_t stream)
{
    if (a.count <= 0) return hipSuccess;
    const int64_t width = 16 * (a.bf16 ? 8 : 4);
    OuterParams p = {};
    p.sum[0] = a.sum[0];
    p.sum[1] = a.sum[1];
    p.row_adapter = a.row_adapter;
    p.ranks = a.ranks;
    p.count = a.count;
    p.rank = a.rank;
    p.T = a.T;
    p.tiles0 = (unsigned)((a.sum[0].C + width - 1) / width);
    p.tiles = p.tiles0 + (unsigned)((a.sum[1].C + width - 1) / width);
    const int splits = adapter_outer_splits(a.sum[0].C, a.sum[1].C, a.count, a.rank, a.bf16, a.T);
    p.per = ((a.T + splits - 1) / splits + 7) / 8 * 8;
    p.partial = splits > 1 ? a.partial : nullptr;
    // (one window: nothing to find; nearly as many requests as rows: the rows are as soon gone through)
    if (p.per > WINDOW && a.requests <= a.T / 4) {
        p.start = a.start;
        p.adapter = a.adapter;
        p.requests = a.requests;
    }
    p.window = WINDOW;
    if (a.bf16) {
        const int64_t widest = std::max(a.sum[0].C, a.sum[1].C), most = (int64_t(1) << 30) / widest;
        if (most < WINDOW) p.window = (int)(most < 64 ? 64 : most / 64 * 64);
        for (int i = 0; i < 2; ++i) {      // (16-byte pieces of H's rows)
            if (p.sum[i].ldh % 4 == 0 || a.T == 0) continue;
            const int pitch = adapter_pitch(a.rank);
            const int64_t total = a.T * pitch;
            pad_projections_kernel<<<(unsigned)std::min<int64_t>((total + 255) / 256, 2048), 256, 0, stream>>>(p.sum[i].H, a.padded, a.rank, pitch, total);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            p.sum[i].H = a.padded;
            p.sum[i].ldh = pitch;
        }
    }
    const hipError_t e = outer_rank(p, splits, a.bf16, dev, stream);
    if (e != hipSuccess || splits == 1) return e;
    const int64_t total = a.count * a.rank * (a.sum[0].C + a.sum[1].C);
    adapter_outer_join_kernel<<<(unsigned)std::min<int64_t>((total + 255) / 256, 4096), 256, 0, stream>>>(p, splits);
    return hipGetLastError();
}

}  // namespace sfb
