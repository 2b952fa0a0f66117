// The product of bf16 rows with a shared bf16 matrix as it lies in memory, and the factor blocks' part of it:
//
//   forward   out[t][j] = sum_d X[t][d] W[j][d]  + sum_r H[t][r] U_a[r][j]       W contiguous along k
//   backward  out[t][d] = sum_j dY[t][j] W[j][d] + sum_r dH[t][r] V_a[r][d]      W contiguous along the output's columns
//
// Neither operand is copied or transposed first.  Tiles go from memory straight into LDS through buffer descriptors, whose
// range check fills what lies behind the last row, column or k with zeros.  In the backward W's tile lies in LDS as 64 rows
// (k) of TBN columns and is read with the transposing LDS read (four rows of 16 columns a group of 16 lanes; lane i gets
// column i); so are the blocks' factors in both.
// W is the first operand of the MFMA, so a lane's results are one row of the output, and the columns are dealt to the MFMA
// tiles such that a lane owns runs of eight consecutive ones and the four lanes of a row 32 of them: 16-byte stores, 64 bytes
// of a row together.
//
// The blocks' part comes first and is what the accumulators start from.  H is held as two bf16 terms side by side along k
// against the same factors: 16 pairs are one MFMA of k = 32.  Per block that occurs in a tile its factors are loaded and
// multiplied with the rows that use it; the others' H counts as zeros there.  A factor that is not finite must not meet those
// zeros: it counts as zero too, as does an H that is not finite, which must not meet these, and the rows that use the block get
// the products of either when they are stored.
//
// The matrix pipes bound it where there are tiles enough: 8192 rows, 4096 x 4096 with 16 blocks of 16 pairs in 210 to 227 us
// either way (1.2 to 1.3 PFLOP/s; the library's product alone 207 to 219, along W's rows 251).  What a tile costs besides its k-loop is instructions that are executed once, so their number
// counts, and a register that is spilled around them more so (an earlier form with scratch memory and 80 KB of code: 30 us a
// tile, this one 8).
#include "adapter_device.h"
#include "planes.h"

#include <algorithm>

namespace sfb {
namespace {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

struct BaseParams {
    const uint16_t* A;
    const uint16_t* W;
    int64_t M, N, K, ldw;
    int64_t pitch;             // blocked W: columns of the operand; 0: rows of ldw
    float* planes;             // split: [split][M][N]
    int split;
    uint16_t* out;             // not split: [M][N]
    const int32_t* row_adapter;
    const uint16_t* Hx;        // [M][2 adapter_pitch(rank)]
    const float* H;            // [M][adapter_pitch(rank)]
    const uint16_t* F;         // [count][rank][N]
    const int32_t* ranks;
    int count, rank;
    int tiles_m, tiles_n, group_m, num_xcd;
};

// The accumulators stay in the accumulation registers: left to itself the compiler moves them to ordinary ones, all at once,
// for any arithmetic on them, and spills.  The caller sees to it that the MFMAs that wrote them have retired.
__device__ __forceinline__ float acc_read(float element)
{
    float v;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(element));
    return v;
}
// More wait states than the longest MFMA needs to write back its result.
__device__ __forceinline__ void mfma_settle() { asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory"); }

// The same value, and nothing that the compiler can work out ahead of time from it: what is needed once a tile is not to be
// kept in registers over the k-loop.
__device__ __forceinline__ int here(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ int here_scalar(int v)
{
    asm volatile("" : "+s"(v));
    return v;
}

// Column of the output's tile that row i of MFMA tile tb of a wavefront holds.
__device__ __forceinline__ constexpr int column_of(int tb, int i) { return 32 * (tb >> 1) + 8 * (i >> 2) + 4 * (tb & 1) + (i & 3); }

// The i-th of n things goes after MFMA (2 i + 1) m / (2 n) of the m MFMAs of a window; how many go after MFMA j, and which first.
constexpr int first_slot(int j, int n, int m)
{
    for (int i = 0; i < n; ++i)
        if ((2 * i + 1) * m / (2 * n) >= j) return i;
    return n;
}

// Tiles of 32 TM rows x 32 TN columns, 2 x 2 wavefronts of 16 TM x 16 TN.  Workgroups are persistent (one or two a CU); two
// LDS stages of a k-slice (64) each.  The loads of slice s + 2 go out once every wavefront has read the last fragments of slice
// s, spread between the MFMAs of its second k-step; fragments are double-buffered in registers across the barriers.
template <int TM, int TN, bool TRANSPOSED, bool SPLIT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(TM == 8 ? 1 : 2, TM == 8 ? 1 : 2))) void adapter_base_kernel(BaseParams p)
{
    constexpr int TBM = 32 * TM, TBN = 32 * TN, STEP = TM * TN;
    constexpr uint32_t A_BYTES = TBM * 128, STAGE_BYTES = A_BYTES + TBN * 128;
    constexpr uint32_t F_CHUNK = 16 * TBN * 2, F_OFF = 2 * STAGE_BYTES;
    constexpr int LOADS = TM + TN, BPOS = STEP / 2, N2B = LOADS / 2, N3 = LOADS - N2B;
    constexpr int READS = TM + (TRANSPOSED ? 2 : 1) * TN;
    extern __shared__ u32x4 smem[];
    char* const lds = reinterpret_cast<char*>(smem);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave0 = __builtin_amdgcn_readfirstlane(tid >> 6), wave = wave0;
    const int wm0 = (wave >> 1) * 16 * TM, wn0 = (wave & 1) * 16 * TN;

    // ---- persistent schedule: each XCD a contiguous range of a raster of groups of group_m row-tiles, row-tile index fastest
    const uint32_t tiles = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n;
    const uint32_t xcds = (uint32_t)p.num_xcd, xcd = blockIdx.x % xcds, wi = blockIdx.x / xcds;
    const uint32_t per_xcd = gridDim.x / xcds + (xcd < gridDim.x % xcds ? 1 : 0);      // workgroups of this XCD
    const uint32_t xcd_start = xcd * (tiles / xcds) + (xcd < tiles % xcds ? xcd : tiles % xcds);
    const uint32_t xcd_count = tiles / xcds + (xcd < tiles % xcds ? 1 : 0);
    if (wi >= xcd_count) return;
    const int n_my = (int)((xcd_count - wi + per_xcd - 1) / per_xcd);
    auto tile_origin = [&](int ordinal, int64_t& m0, int64_t& n0) {
        const uint32_t t = xcd_start + (uint32_t)ordinal * per_xcd + wi;
        const uint32_t per_group = (uint32_t)p.group_m * (uint32_t)p.tiles_n;
        const uint32_t grp = t / per_group, rr = t % per_group, first = grp * (uint32_t)p.group_m;
        const uint32_t gm = (uint32_t)p.tiles_m - first < (uint32_t)p.group_m ? (uint32_t)p.tiles_m - first : (uint32_t)p.group_m;
        m0 = (int64_t)(first + rr % gm) * TBM;
        n0 = (int64_t)(rr / gm) * TBN;
    };
    const int slices = (int)((p.K + BK - 1) / BK);
    const int s_begin = SPLIT ? (int)((int64_t)slices * blockIdx.y / p.split) : 0;
    const int nk = (SPLIT ? (int)((int64_t)slices * (blockIdx.y + 1) / p.split) : slices) - s_begin;
    const bool has_tail = p.K % BK != 0 && s_begin + nk == slices;

    // ---- loader: A (and W, k-contiguous) as 128-byte LDS rows of 64 k, chunk c of row r in slot c ^ swz(r); W, transposed: LDS
    // rows of TBN columns, 16-byte chunk u of row r in slot u ^ 4 (r % 4)
    const uint32_t lda = (uint32_t)p.K * 2u, ldw = p.pitch ? (uint32_t)BK * 2u : (uint32_t)p.ldw * 2u;
    constexpr int SLOTS = TBN / 8, RPL = 64 / SLOTS;      // chunks of a row, rows of a load
    uint32_t offA[TM], offB[TN];
    uint64_t gA = 0, gB = 0;
    int64_t load_n0 = 0;
    int iss_k = 0, iss_tile = 0;
    uint32_t iss_to = lds_base + (uint32_t)(TM * wave) * 1024u;      // (a stage is as large as a power of two, the LDS begins at 0)
    auto w_address = [&](int64_t k0) {      // W's tile at slice k0
        if (TRANSPOSED)
            return reinterpret_cast<uint64_t>(p.W) + (p.pitch ? (uint64_t)(((k0 / BM) * (p.pitch / BK) + load_n0 / BK) * (BM * BK) + (k0 % BM) * BK) * 2u
                                                              : (uint64_t)(k0 * p.ldw + load_n0) * 2u);
        return reinterpret_cast<uint64_t>(p.W) + (p.pitch ? (uint64_t)(((load_n0 / BM) * (p.pitch / BK) + k0 / BK) * (BM * BK) + (load_n0 % BM) * BK) * 2u
                                                          : (uint64_t)(load_n0 * p.ldw + k0) * 2u);
    };
    const int k_left = (int)(p.K - (int64_t)(slices - 1) * BK);      // of the last slice (a multiple of eight)
    auto cut_tail = [&]() {                                          // the loads to come are those of the last slice
        const int lane = here(threadIdx.x & 63), wave = here_scalar(wave0);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int r = 8 * (TM * wave + i) + (lane >> 3);
            if (8 * ((lane & 7) ^ swz(r)) >= k_left) offA[i] = OUT_OF_RANGE;
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int r = TRANSPOSED ? (TN * wave + i) * RPL + lane / SLOTS : 8 * (TN * wave + i) + (lane >> 3);
            if ((TRANSPOSED ? r : 8 * ((lane & 7) ^ swz(r))) >= k_left) offB[i] = OUT_OF_RANGE;
        }
    };
    auto enter_tile = [&](int ordinal) {
        const int lane = here(threadIdx.x & 63), wave = here_scalar(wave0);
        int64_t m0;
        tile_origin(ordinal, m0, load_n0);
        const int last_m = (int)(p.M - m0 < TBM ? p.M - m0 : TBM), last_n = (int)(p.N - load_n0 < TBN ? p.N - load_n0 : TBN);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int r = 8 * (TM * wave + i) + (lane >> 3);
            offA[i] = r < last_m ? (uint32_t)r * lda + (uint32_t)(((lane & 7) ^ swz(r)) << 4) : OUT_OF_RANGE;
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            if (TRANSPOSED) {
                const int r = (TN * wave + i) * RPL + lane / SLOTS, u = (lane % SLOTS) ^ ((r & 3) << 2);
                offB[i] = 8 * u < last_n ? (uint32_t)r * ldw + (p.pitch ? (uint32_t)(u >> 3) * (BM * BK * 2) + (uint32_t)(u & 7) * 16u : (uint32_t)u * 16u)
                                         : OUT_OF_RANGE;
            } else {
                const int r = 8 * (TN * wave + i) + (lane >> 3), w = r % (16 * TN);
                const int n = r - w + column_of(w >> 4, w & 15);
                offB[i] = n < last_n ? (uint32_t)n * ldw + (uint32_t)(((lane & 7) ^ swz(r)) << 4) : OUT_OF_RANGE;
            }
        }
        gA = uniform64(reinterpret_cast<uint64_t>(p.A) + (uint64_t)(m0 * p.K + (int64_t)s_begin * BK) * 2u);
        gB = uniform64(w_address((int64_t)s_begin * BK));
        if (has_tail && nk == 1) cut_tail();
    };
    auto issue_one = [&](auto J) {
        constexpr int j = decltype(J)::value;
        static_assert(TM == TN, "one base of both operands' loads");
        if constexpr (j < TM)
            buffer_to_lds_16<j * 1024u>(iss_to, descriptor(gA), offA[j]);
        else
            buffer_to_lds_16<A_BYTES + (j - TM) * 1024u>(iss_to, descriptor(gB), offB[j - TM]);
    };
    // from a slice of W to the next; blocks of 256 rows, transposed: every fourth slice begins another block
    const uint64_t stepB = TRANSPOSED ? (p.pitch ? BK * BK * 2 : (uint64_t)p.ldw * (BK * 2)) : p.pitch ? BM * BK * 2 : BK * 2;
    const uint64_t jumpB = TRANSPOSED && p.pitch ? (uint64_t)(p.pitch / BK - 1) * (BM * BK * 2) : 0;
    auto issue_done = [&]() {      // the load cursor moves on by a slice
        iss_to ^= STAGE_BYTES;
        iss_k = __builtin_amdgcn_readfirstlane(iss_k + 1);
        if (iss_k < nk) {
            gA += BK * 2;
            gB += stepB;
            if (TRANSPOSED && ((s_begin + iss_k) & (BM / BK - 1)) == 0) gB += jumpB;
            if (has_tail && iss_k + 1 == nk) cut_tail();
        } else {
            iss_k = 0;
            ++iss_tile;
            enter_tile(iss_tile < n_my ? iss_tile : n_my - 1);      // (past the last tile: loads that are never read)
        }
    };

    // ---- fragments: lane (q, c) supplies row c of 16 and k = 8 q .. 8 q + 7 of the 32 of a k-step
    uint32_t ra[4], rb[4], rf[4];
    auto transposed_at = [&](int q, int row) {      // byte of the lane's piece of MFMA tiles 2 q, 2 q + 1 (8 bytes further), LDS row `row`
        return (uint32_t)row * (TBN * 2) + (uint32_t)((((wn0 >> 3) + 4 * q) ^ ((l16 >> 2) << 2)) + (l16 & 3)) * 16u;
    };
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int r = wm0 + 16 * (t % TM) + l16, rn = wn0 + 16 * (t % TN) + l16;
        ra[t] = (uint32_t)(r * 128 + ((quad ^ swz(r)) << 4));
        rb[t] = A_BYTES + (TRANSPOSED ? transposed_at(t, 8 * quad + (l16 >> 2)) : (uint32_t)(rn * 128 + ((quad ^ swz(rn)) << 4)));
        rf[t] = transposed_at(t, 8 * (quad & 1) + (l16 >> 2));
    }
    struct Frags {
        bf16x8 a[TM];
        s16x4 b[TN][2];
    };
    // The i-th fragment read of a k-step: W's first, the rows' all, W's others.
    auto read_one = [&](Frags& f, int ks, int i) {
        constexpr int PER = TRANSPOSED ? 2 : 1;
        if (i >= PER && i < PER + TM) {
            const int t = i - PER;
            f.a[t] = *reinterpret_cast<const bf16x8*>(lds + (ra[t & 3] ^ (64u * ks)) + (t >> 2) * 64 * 128);
            return;
        }
        const int j = i < PER ? i : i - TM, t = j / PER;
        if (TRANSPOSED) {
            f.b[t][j % 2] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4*)(lds + rb[t >> 1] + (t & 1) * 8 + ks * 32 * (TBN * 2) + (j % 2) * 4 * (TBN * 2)));
        } else {
            const u32x4 v = *reinterpret_cast<const u32x4*>(lds + (rb[t & 3] ^ (64u * ks)) + (t >> 2) * 64 * 128);
            f.b[t][0] = __builtin_bit_cast(s16x4, u32x2{v[0], v[1]});
            f.b[t][1] = __builtin_bit_cast(s16x4, u32x2{v[2], v[3]});
        }
    };
    auto b_of = [](const Frags& f, int t) {
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(f.b[t][0], f.b[t][1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto flip_stage = [&]() {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            ra[t] ^= STAGE_BYTES;
            rb[t] ^= STAGE_BYTES;
        }
    };

    floatx4 acc[TM][TN];
    int mine[TM];                     // block of the lane's row of each MFMA tile

    // ---- the blocks' part of a tile, with room for `slots` chunks of their factors from `region` of the LDS on; whether a factor
    // is not finite
    auto blocks_part = [&](int64_t m0, int64_t n0, uint32_t region, int slots) {
        bool special = false;         // whether the wavefront has met a factor that is not finite
        const int lane = here(threadIdx.x & 63), l16 = lane & 15, quad = lane >> 4, wave = here_scalar(wave0);
        uint64_t left[TBM / 64];      // rows of the tile whose block is still to come
        int block[TBM / 64], rank_at[TBM / 64];
#pragma unroll
        for (int i = 0; i < TBM / 64; ++i) {
            const int64_t m = m0 + 64 * i + lane;
            block[i] = m < p.M ? p.row_adapter[m] : ROW_OUTSIDE;
            left[i] = __builtin_amdgcn_ballot_w64(block[i] >= 0 && block[i] < p.count);
        }
#pragma unroll
        for (int i = 0; i < TBM / 64; ++i) rank_at[i] = left[i] >> lane & 1 ? rank_of(p.ranks, p.rank, block[i]) : 0;
        const int pitch = adapter_pitch(p.rank);
        // the H of 16 pairs of all the wavefront's rows (what rows of other blocks hold is not used)
        const uint16_t* hx[TM];
#pragma unroll
        for (int ta = 0; ta < TM; ++ta) {
            const int64_t m = m0 + wm0 + 16 * ta + l16;
            hx[ta] = p.Hx + (m < p.M ? m : p.M - 1) * (2 * pitch) + 8 * quad;
        }
        u32x4 h[TM];
        int h_from = -1;
        // Rounds of `slots` chunks of 16 pairs, the first 16 of all blocks and then the next: LDS rows of TBN columns as W's, transposed.
        // Lane k knows the k-th chunk's block, first pair and the block's rank.
        uint64_t all[TBM / 64];
#pragma unroll
        for (int i = 0; i < TBM / 64; ++i) all[i] = left[i];
        int cur_r = 0;
        for (;;) {
            int of = -1, from = 0, ranks = 0, chunks = 0;
            while (chunks < slots && cur_r < p.rank) {
                int a = -1, rank = 0;
#pragma unroll
                for (int i = 0; i < TBM / 64; ++i)
                    if (a < 0 && left[i]) {
                        const int at = (int)__builtin_ctzll(left[i]);
                        a = __builtin_amdgcn_readlane(block[i], at);
                        rank = __builtin_amdgcn_readlane(rank_at[i], at);
                    }
                if (a < 0) {                       // the next 16
                    cur_r += 16;
#pragma unroll
                    for (int i = 0; i < TBM / 64; ++i) left[i] = all[i];
                    continue;
                }
#pragma unroll
                for (int i = 0; i < TBM / 64; ++i) {
                    const uint64_t its = __builtin_amdgcn_ballot_w64(block[i] == a);
                    left[i] &= ~its;
                    if (rank <= cur_r + 16) all[i] &= ~its;
                }
                if (cur_r >= rank) continue;
                if (lane == chunks) {
                    of = a;
                    from = cur_r;
                    ranks = rank;
                }
                ++chunks;
            }
            if (chunks == 0) break;
            __syncthreads();                       // (the chunks before have been read)
            for (int k = 0; k < chunks; ++k) {
                const int a = __builtin_amdgcn_readlane(of, k), r0 = __builtin_amdgcn_readlane(from, k), rank = __builtin_amdgcn_readlane(ranks, k);
                const uint64_t factors = reinterpret_cast<uint64_t>(p.F) + (uint64_t)(((int64_t)a * p.rank + r0) * p.N + n0) * 2u;
                static_for<0, (int)(F_CHUNK / 4096)>([&](auto I) {
                    constexpr int PER = (int)(F_CHUNK / 4096);
                    const int r = (PER * wave + decltype(I)::value) * RPL + lane / SLOTS, u = (lane % SLOTS) ^ ((r & 3) << 2);
                    const bool in = r0 + r < rank && n0 + 8 * u < p.N;
                    buffer_to_lds_16<decltype(I)::value * 1024u>(lds_base + region + (uint32_t)k * F_CHUNK + (uint32_t)(PER * wave) * 1024u, descriptor(factors),
                                                               in ? (uint32_t)r * (uint32_t)(p.N * 2) + (uint32_t)u * 16u : OUT_OF_RANGE);
                });
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            {
#pragma unroll 1
                for (int c = 0; c < chunks; ++c) {
                    const int a = __builtin_amdgcn_readlane(of, c);
                    const int r0 = __builtin_amdgcn_readlane(from, c);
                    if (r0 != h_from) {
                        h_from = r0;
#pragma unroll
                        for (int ta = 0; ta < TM; ++ta) h[ta] = *reinterpret_cast<const u32x4*>(hx[ta] + 2 * r0);
                    }
                    bool used = false;
#pragma unroll
                    for (int ta = 0; ta < TM; ++ta) used = used || __builtin_amdgcn_ballot_w64(mine[ta] == a) != 0;
                    if (!used) continue;
                    u32x4 f[TN];
                    uint32_t least = 0x7f807f80u;      // of both halves; 0: not finite
#pragma unroll
                    for (int t = 0; t < TN; ++t) {
                        const char* const at = lds + region + rf[t >> 1] + c * F_CHUNK + (t & 1) * 8;
                        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * (TBN * 2)));
                        f[t] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
#pragma unroll
                    for (int t = 0; t < TN; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t w = f[t][e];
                            least = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, least),
                                                                                           __builtin_bit_cast(u16x2, ~w & 0x7f807f80u)));
                        }
                    const bool not_finite = __builtin_amdgcn_ballot_w64((least & 0xffffu) == 0 || least >> 16 == 0) != 0;
                    if (not_finite) {
                        special = true;
#pragma unroll
                        for (int t = 0; t < TN; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                uint32_t w = f[t][e];
                                if ((~w & 0x7f80u) == 0) w &= 0xffff0000u;
                                if ((~w & 0x7f800000u) == 0) w &= 0xffffu;
                                f[t][e] = w;
                            }
                    }
#pragma unroll
                    for (int ta = 0; ta < TM; ++ta) {
                        if (__builtin_amdgcn_ballot_w64(mine[ta] == a) == 0) continue;
                        u32x4 ha = {0u, 0u, 0u, 0u};
                        if (mine[ta] == a) ha = h[ta];
                        if (not_finite) {          // (here, a row at a time: done to h itself it costs the large tiles 31 spilled registers)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if ((~ha[e] & 0x7f80u) == 0) ha[e] &= 0xffff0000u;
                                if ((~ha[e] & 0x7f800000u) == 0) ha[e] &= 0xffffu;
                            }
                        }
#pragma unroll
                        for (int tb = 0; tb < TN; ++tb)
                            acc[ta][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[tb]), __builtin_bit_cast(bf16x8, ha), acc[ta][tb], 0, 0, 0);
                    }
                }
            }
        }
        return special;
    };
    // The products that have a factor or an H that is not finite, an infinity or a not-a-number each, so that the sum's rounding
    // does not matter: no stored sum has those with such factors; those with such an H some sums have, and once more they change
    // nothing there.  The lanes go through their own pieces of the tile once more.
    auto add_special = [&](int64_t m0, int64_t n0) {
        const int pitch = adapter_pitch(p.rank), lane = here(threadIdx.x & 63), l16 = lane & 15, quad = lane >> 4;
#pragma unroll 1
        for (int k = 0; k < TM * TN / 2; ++k) {
            const int64_t m = m0 + wm0 + 16 * (k / (TN / 2)) + l16, n = n0 + wn0 + 32 * (k % (TN / 2)) + 8 * quad;
            const int a = m < p.M && n < p.N ? p.row_adapter[m] : ROW_OUTSIDE;
            if (a < 0 || a >= p.count) continue;
            int rank = p.ranks ? p.ranks[a] : p.rank;
            rank = rank < p.rank ? rank : p.rank;
            uint16_t* const out = p.out + m * p.N + n;
#pragma unroll 1
            for (int r = 0; r < rank; ++r) {
                const float h = p.H[m * pitch + r];
                const bool all = (~__float_as_uint(h) & 0x7f800000u) == 0;
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                    const uint32_t bits = (uint32_t)p.F[((int64_t)a * p.rank + r) * p.N + n + e] << 16;
                    if (all || (~bits & 0x7f800000u) == 0)
                        out[e] = (uint16_t)pack_bf16(fmaf(h, __uint_as_float(bits), __uint_as_float((uint32_t)out[e] << 16)), 0.f);
                }
            }
        }
    };

    auto epilogue = [&](int64_t m0, int64_t n0) {
        // register i of lane (q, c) of tile (ta, tb): row 16 ta + c, column column_of(tb, 4 q + i)
        mfma_settle();
        const int lane = here(threadIdx.x & 63), l16 = lane & 15, quad = lane >> 4;
#pragma unroll
        for (int ta = 0; ta < TM; ++ta) {
            const int64_t m = m0 + wm0 + 16 * ta + l16;
            if (SPLIT) {
                if (m >= p.M) continue;
                float* const row = p.planes + ((int64_t)blockIdx.y * p.M + m) * p.N + n0 + wn0;
#pragma unroll
                for (int tb = 0; tb < TN; ++tb) {
                    const int n = column_of(tb, 4 * quad);
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = acc_read(acc[ta][tb][e]);
                    if (n0 + wn0 + n < p.N) *reinterpret_cast<floatx4*>(row + n) = floatx4{x[0], x[1], x[2], x[3]};
                }
            } else {
                if (mine[ta] == ROW_OUTSIDE) continue;
                uint16_t* const row = p.out + m * p.N + n0 + wn0;
#pragma unroll
                for (int tb = 0; tb < TN; tb += 2) {
                    const int n = column_of(tb, 4 * quad);
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = acc_read(acc[ta][tb + (e >> 2)][e & 3]);
                    if (n0 + wn0 + n >= p.N) continue;
                    *reinterpret_cast<u32x4*>(row + n) = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
                }
            }
        }
    };

    // ---- pipeline: slice s lives in stage s & 1; f0 holds the fragments of its first k-step, f1 of the second
    Frags f0, f1;
    // Small tiles: the first one's blocks come in front of its slices and have all of the LDS for their factors: where a tile has
    // many of them it gains (704 rows, 8192 x 2048, 40 requests with blocks of 32 pairs: 46 us, with four chunks a round 49; 700
    // rows, 8192 x 1024, 200 requests, 64 pairs 97 and 113, four pairs 43 and 46), elsewhere nothing (1500 rows, 2048 x 2048, 30
    // requests, 16 pairs 31 and 31; 2000 rows, 8192 x 512, 8 requests, 128 pairs 54 and 54).  (On the large ones the order costs registers.)
    constexpr bool FIRST = TM == 4 && !SPLIT;
    auto prologue = [&]() {
        enter_tile(0);
#pragma unroll 1
        for (int s = 0; s < 2; ++s) {
            static_for<0, LOADS>(issue_one);
            issue_done();
        }
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < READS; ++i) read_one(f0, 0, i);
    };
    if constexpr (!FIRST) prologue();

    auto slice_body = [&]() {
        auto mfma = [&](const Frags& f, auto J) {
            constexpr int j = decltype(J)::value, tb = j / TM, ta = j % TM;
            acc[ta][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b_of(f, tb), f.a[ta], acc[ta][tb], 0, 0, 0);
        };
        // k-step 0 on f0; the reads of k-step 1 go out over its first three quarters
        static_for<0, STEP>([&](auto J) {
            constexpr int j = decltype(J)::value, M34 = 3 * STEP / 4;
            mfma(f0, J);
            if constexpr (j < M34)
                static_for<first_slot(j, READS, M34), first_slot(j + 1, READS, M34)>([&](auto I) { read_one(f1, 1, decltype(I)::value); });
            __builtin_amdgcn_sched_barrier(0);
        });
        __syncthreads();                                   // every wavefront has read the stage
        // the first half of k-step 1 on f1; the first loads of slice s + 2
        static_for<0, BPOS>([&](auto J) {
            constexpr int j = decltype(J)::value;
            mfma(f1, J);
            static_for<first_slot(j, N2B, BPOS), first_slot(j + 1, N2B, BPOS)>([&](auto I) { issue_one(I); });
            __builtin_amdgcn_sched_barrier(0);
        });
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N2B) : "memory");      // everything but those: slice s + 1 is in LDS
        __syncthreads();
        flip_stage();
        // the rest of k-step 1; the reads of the next slice's k-step 0, the other loads
        static_for<BPOS, STEP>([&](auto J) {
            constexpr int j = decltype(J)::value - BPOS, M = STEP - BPOS;
            mfma(f1, J);
            static_for<first_slot(j, READS, M - STEP / 8), first_slot(j + 1, READS, M - STEP / 8)>([&](auto I) { read_one(f0, 0, decltype(I)::value); });
            static_for<first_slot(j, N3, M), first_slot(j + 1, N3, M)>([&](auto I) { issue_one(std::integral_constant<int, N2B + decltype(I)::value>{}); });
            __builtin_amdgcn_sched_barrier(0);
        });
        issue_done();
    };
    for (int t = 0; t < n_my; ++t) {
        int64_t m0, n0;
        tile_origin(t, m0, n0);
        bool special = false;
#pragma unroll
        for (int ta = 0; ta < TM; ++ta)
#pragma unroll
            for (int tb = 0; tb < TN; ++tb) acc[ta][tb] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (!SPLIT) {
#pragma unroll
            for (int ta = 0; ta < TM; ++ta) {
                const int64_t m = m0 + wm0 + 16 * ta + l16;
                mine[ta] = m < p.M ? p.row_adapter[m] : ROW_OUTSIDE;
            }
            const bool all = FIRST && t == 0;
            special = blocks_part(m0, n0, all ? 0u : F_OFF, all ? (int)((F_OFF + 4 * F_CHUNK) / F_CHUNK) : 4);
            // (vmcnt(0): a load that nobody has waited for, one of H, would have the compiler wait in every slice)
            __builtin_amdgcn_s_waitcnt(0x0f70);
            if (FIRST && t == 0) {
                __syncthreads();                           // (the chunks have been read)
                prologue();
            }
        }
#pragma unroll
        for (int ta = 0; ta < TM; ++ta)
#pragma unroll
            for (int tb = 0; tb < TN; ++tb) asm volatile("" : "+a"(acc[ta][tb]));
        for (int k = 0; k < nk; ++k) slice_body();
        epilogue(m0, n0);
        if (!SPLIT && special) add_special(m0, n0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no load may be in flight when the workgroup's LDS is released
}

template <int TM, int TN, bool TRANSPOSED, bool SPLIT>
hipError_t launch_base(BaseParams& p, DeviceInfo& dev, hipStream_t stream)
{
    constexpr int stages = 2 * (TM + TN) * 32 * 128, lds = stages + 4 * 16 * TN * 32 * 2;
    constexpr int slot = (TM == 8 ? 4 : 0) + (TRANSPOSED ? 2 : 0) + (SPLIT ? 1 : 0);
    if (!dev.adapter_base_lds_set[slot]) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&adapter_base_kernel<TM, TN, TRANSPOSED, SPLIT>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        dev.adapter_base_lds_set[slot] = true;
    }
    p.tiles_m = (int)((p.M + 32 * TM - 1) / (32 * TM));
    p.tiles_n = (int)((p.N + 32 * TN - 1) / (32 * TN));
    p.group_m = 8;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n, slots = (int64_t)(dev.cus > 0 ? dev.cus : 256) * (TM == 8 ? 1 : 2);
    const dim3 grid((unsigned)(tiles < slots || SPLIT ? tiles : slots), (unsigned)p.split);
    adapter_base_kernel<TM, TN, TRANSPOSED, SPLIT><<<grid, 256, lds, stream>>>(p);
    return hipGetLastError();
}

// ---- projections of many rows ---------------------------------------------------------------------------------------------
// H[t][r] = scale_a sum_k X[t][k] F_a[r][k] on tiles of 32 rows of one request (as adapter_project_kernel divides them) x 16 RT
// factors.  The stream of X and the factors' way out of the L2 bound it where rows are many: whole lines straight into LDS (8192
// rows, K = 4096: 16 pairs 22 us, 64 pairs 27 to 29; MFMA operands loaded from memory into their registers, a line for every
// lane, 27 and 49 to 61).  Where they are few it is what a slice takes, so there are 128 k or more in one (600 rows, 32 pairs:
// slices of 64 k 15.7 us, of 128 13.2; twice the stages gain nothing).
// Wavefront w: the k-step w % 2 of every 64 k and the rows 16 (w / 2) .. of the tile.
template <int RT, int KM, int PS>
__global__ __launch_bounds__(256) void adapter_project_tiles_kernel(ProjectParams p, unsigned windows, unsigned xcds)
{
    constexpr int LOADS = KM * (4 + 2 * RT) / 4;      // 64 KM of k a slice; loads of a wavefront
    static_assert(KM * (4 + 2 * RT) % 4 == 0, "as many loads for every wavefront");
    constexpr uint32_t ROWS_BYTES = 32 * 128, SLAB = ROWS_BYTES + 16 * RT * 128, STAGE_BYTES = KM * SLAB;
    __shared__ u32x4 smem[PS * STAGE_BYTES / 16];
    const char* const lds = reinterpret_cast<const char*>(smem);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    ProjectTile tile;
    if (!project_tile<32>(p, windows, xcds, 16 * RT * (int)blockIdx.y, 16 * RT, tid, 256, lane, tile)) return;
    const int r0 = 16 * RT * (int)blockIdx.y;

    // load j of a slice: 8 rows of slab j / (4 + 2 RT), of X or of the factors
    uint32_t off[LOADS], to[LOADS];
    int k_of[LOADS];
    bool is_x[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int j = LOADS * wave + i, slab = j / (4 + 2 * RT), b = j % (4 + 2 * RT);
        is_x[i] = b < 4;
        const int r = 8 * (is_x[i] ? b : b - 4) + (lane >> 3), c = (lane & 7) ^ swz(r);
        k_of[i] = 64 * slab + 8 * c;
        const bool in = is_x[i] ? r < tile.rows : r0 + r < tile.rank;
        off[i] = in ? (uint32_t)r * (uint32_t)(p.K * 2) + (uint32_t)k_of[i] * 2u : OUT_OF_RANGE;
        to[i] = (uint32_t)slab * SLAB + (is_x[i] ? 0u : ROWS_BYTES) + (uint32_t)(is_x[i] ? b : b - 4) * 1024u;
    }
    const uint64_t gx = uniform64(reinterpret_cast<uint64_t>(p.X) + (uint64_t)(tile.t0 * p.K) * 2u);
    const uint64_t gf = uniform64(reinterpret_cast<uint64_t>(p.F) + (uint64_t)(((int64_t)tile.a * p.rows.rank + r0) * p.K) * 2u);
    const int slices = (int)((p.K + 64 * KM - 1) / (64 * KM));
    auto issue = [&](int s) {      // (past the last slice: nothing is in range)
        const int64_t k0 = (int64_t)s * (64 * KM), left = p.K - k0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            buffer_to_lds_16<0>(lds_base + (uint32_t)(s % PS) * STAGE_BYTES + to[i], descriptor((is_x[i] ? gx : gf) + (uint64_t)k0 * 2u),
                                k_of[i] < left ? off[i] : OUT_OF_RANGE);
    };
    floatx4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int ks = wave & 1, row = 16 * (wave >> 1) + l16;
    for (int s = 0; s < PS - 1; ++s) issue(s);
    for (int s = 0; s < slices; ++s) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS * (PS - 2)) : "memory");
        __syncthreads();                                   // slice s is in LDS; every wavefront has read the slice before
        issue(s + PS - 1);
        const char* const stage = lds + (uint32_t)(s % PS) * STAGE_BYTES;
#pragma unroll
        for (int m = 0; m < KM; ++m) {
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(stage + m * SLAB + row * 128 + (((4 * ks + quad) ^ swz(row)) << 4));
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int r = 16 * i + l16;
                const bf16x8 f = *reinterpret_cast<const bf16x8*>(stage + m * SLAB + ROWS_BYTES + r * 128 + (((4 * ks + quad) ^ swz(r)) << 4));
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, x, acc[i], 0, 0, 0);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    floatx4* const part = reinterpret_cast<floatx4*>(smem);      // the odd k-steps' sums
    if (ks == 1) {
#pragma unroll
        for (int i = 0; i < RT; ++i) part[((wave >> 1) * RT + i) * 64 + lane] = acc[i];
    }
    __syncthreads();
    if (ks == 1) return;
#pragma unroll
    for (int i = 0; i < RT; ++i)
        store_projection(p, tile, tile.t0 + row, row < tile.rows, r0 + 16 * i + 4 * quad, acc[i] + part[((wave >> 1) * RT + i) * 64 + lane]);
}

// ---- few rows ------------------------------------------------------------------------------------------------------------
// The stream of W bounds the product of few rows (adapter_few_plan says which).  Tiles of 64 or 128 rows x 64 columns along a
// part of k, five or three LDS stages of a k-slice: about 100 KB of requests of a CU's two workgroups in flight.  The blocks'
// factors are taken for further columns of the matrix: every row is multiplied with the factors of all blocks (the matrix pipes
// have the time), and the join picks its own block's.  64 rows, 4096 x 4096, 32 blocks of 16 pairs: 12.8 us and the join's 5.2, of
// which the matrix takes 7 at the rate of a copy; one row, 8192 x 8192 out of memory 27 to 36 (3.7 to 5 TB/s).
struct FewParams {
    const uint16_t* A;
    const uint16_t* W;
    const uint16_t* F;         // [factors][K]
    int64_t M, N, K, ldw, pitch, factors, width;      // width: columns of a plane
    float* planes;             // [split][M][width]
    int split, tiles_m, tiles_w;
    AdapterRows rows;
    int32_t* row_adapter;      // nullable: written by the last workgroup
};
constexpr int few_stages(int fm) { return fm == 2 ? 5 : 3; }

// FM: 32 FM rows; 2 x 2 wavefronts of 16 FM x 32.
template <bool TRANSPOSED, int FM>
__global__ __launch_bounds__(256) void adapter_few_kernel(FewParams p)
{
    constexpr int NS = few_stages(FM);
    constexpr uint32_t A_BYTES = 32 * FM * 128, STAGE_BYTES = A_BYTES + 64 * 128;
    extern __shared__ u32x4 smem[];
    char* const lds = reinterpret_cast<char*>(smem);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (p.row_adapter && blockIdx.x == gridDim.x - 1) {
        if (blockIdx.y != 0) return;
        const int64_t first = p.rows.start[0], last = p.rows.start[p.rows.requests];
        for (int64_t t = tid; t < p.M; t += 256)
            if (t < first || t >= last) p.row_adapter[t] = ROW_OUTSIDE;
        for (int64_t q = tid; q < p.rows.requests; q += 256) {
            int a = p.rows.adapter[q];
            if (a < 0 || a >= p.rows.count || rank_of(p.rows.ranks, p.rows.rank, a) == 0) a = ROW_NONE;
            const int64_t begin = p.rows.start[q], end = p.rows.start[q + 1];
            for (int64_t t = begin < 0 ? 0 : begin; t < end && t < p.M; ++t) p.row_adapter[t] = a;
        }
        return;
    }
    const int wm0 = (wave >> 1) * 16 * FM, wn0 = (wave & 1) * 32;
    const int64_t m0 = (int64_t)(blockIdx.x % (unsigned)p.tiles_m) * (32 * FM);
    const int tile = (int)(blockIdx.x / (unsigned)p.tiles_m);
    const bool factor = tile >= p.tiles_w;                 // columns of the blocks' factors, k-contiguous
    const bool transposed = TRANSPOSED && !factor;
    const int64_t n0 = (int64_t)(factor ? tile - p.tiles_w : tile) * 64;
    const int64_t N = factor ? p.factors : p.N, ldw_e = factor ? p.K : p.ldw, pitch = factor ? 0 : p.pitch;
    const uint16_t* const W = factor ? p.F : p.W;
    const int slices = (int)((p.K + BK - 1) / BK);
    const int s_begin = (int)((int64_t)slices * blockIdx.y / p.split), nk = (int)((int64_t)slices * (blockIdx.y + 1) / p.split) - s_begin;

    const uint32_t lda = (uint32_t)p.K * 2u, ldw = pitch ? (uint32_t)BK * 2u : (uint32_t)ldw_e * 2u;
    const int last_m = (int)(p.M - m0 < 32 * FM ? p.M - m0 : 32 * FM), last_n = (int)(N - n0 < 64 ? N - n0 : 64);
    uint32_t offA[FM], offB[2];
    int kA[FM], kB[2];                                     // first k of what a lane loads
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int r = 8 * (FM * wave + i) + (lane >> 3), c = (lane & 7) ^ swz(r);
        offA[i] = r < last_m ? (uint32_t)r * lda + (uint32_t)c * 16u : OUT_OF_RANGE;
        kA[i] = 8 * c;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 8 * (2 * wave + i) + (lane >> 3), c = (lane & 7) ^ swz(r);
        if (transposed) {
            const int u = (lane & 7) ^ ((r & 1) << 2);     // LDS rows of 64 columns; chunk u of row r in slot u ^ 4 (r % 2)
            offB[i] = 8 * u < last_n ? (uint32_t)r * ldw + (uint32_t)u * 16u : OUT_OF_RANGE;
            kB[i] = r;
        } else {
            const int w = r & 31, n = r - w + column_of(w >> 4, w & 15);
            offB[i] = n < last_n ? (uint32_t)n * ldw + (uint32_t)c * 16u : OUT_OF_RANGE;
            kB[i] = 8 * c;
        }
    }
    auto issue = [&](int s) {      // (past the last slice: nothing is in range)
        const int64_t k0 = (int64_t)(s_begin + s) * BK;
        const int left = s < nk ? (int)(p.K - k0 < BK ? p.K - k0 : BK) : 0;
        const uint64_t at = transposed ? (pitch ? (uint64_t)(((k0 / BM) * (pitch / BK) + n0 / BK) * (BM * BK) + (k0 % BM) * BK) : (uint64_t)(k0 * ldw_e + n0))
                                       : (pitch ? (uint64_t)(((n0 / BM) * (pitch / BK) + k0 / BK) * (BM * BK) + (n0 % BM) * BK) : (uint64_t)(n0 * ldw_e + k0));
        const u32x4 ra = descriptor(reinterpret_cast<uint64_t>(p.A) + (uint64_t)(m0 * p.K + k0) * 2u);
        const u32x4 rb = descriptor(reinterpret_cast<uint64_t>(W) + at * 2u);
        const uint32_t stage = lds_base + (uint32_t)(s % NS) * STAGE_BYTES;
        static_for<0, FM>([&](auto I) {
            constexpr int i = decltype(I)::value;
            buffer_to_lds_16<i * 1024u>(stage + (uint32_t)(FM * wave) * 1024u, ra, kA[i] < left ? offA[i] : OUT_OF_RANGE);
        });
        static_for<0, 2>([&](auto I) {
            constexpr int i = decltype(I)::value;
            buffer_to_lds_16<A_BYTES + i * 1024u>(stage + (uint32_t)(2 * wave) * 1024u, rb, kB[i] < left ? offB[i] : OUT_OF_RANGE);
        });
    };
    floatx4 acc[FM][2];
#pragma unroll
    for (int ta = 0; ta < FM; ++ta)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) acc[ta][tb] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < NS - 1; ++s) issue(s);
    for (int s = 0; s < nk; ++s) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((FM + 2) * (NS - 2)) : "memory");
        __syncthreads();                                   // slice s is in LDS; every wavefront has read the slice before
        issue(s + NS - 1);
        const char* const stage = lds + (uint32_t)(s % NS) * STAGE_BYTES;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 a[FM], b[2];
#pragma unroll
            for (int t = 0; t < FM; ++t) {
                const int r = wm0 + 16 * t + l16;
                a[t] = *reinterpret_cast<const bf16x8*>(stage + r * 128 + (((4 * ks + quad) ^ swz(r)) << 4));
            }
            if (transposed) {
                // lane i of a group: row i / 4 of four, piece i % 4 of the 32 columns of the wavefront
                const int r = 32 * ks + 8 * quad + (l16 >> 2);
                const char* const at = stage + A_BYTES + r * 128 + ((((wn0 >> 3) + (l16 & 3)) ^ ((r & 1) << 2)) << 4);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * t));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * t + 4 * 128));
                    b[t] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            } else {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int r = wn0 + 16 * t + l16;
                    b[t] = *reinterpret_cast<const bf16x8*>(stage + A_BYTES + r * 128 + (((4 * ks + quad) ^ swz(r)) << 4));
                }
            }
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int ta = 0; ta < FM; ++ta) acc[ta][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[tb], a[ta], acc[ta][tb], 0, 0, 0);
        }
    }
#pragma unroll
    for (int ta = 0; ta < FM; ++ta) {
        const int64_t m = m0 + wm0 + 16 * ta + l16;
        if (m >= p.M) continue;
        float* const row = p.planes + ((int64_t)blockIdx.y * p.M + m) * p.width + (factor ? p.N : 0) + n0 + wn0;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const int n = column_of(tb, 4 * quad);
            if (n0 + wn0 + n < N) *reinterpret_cast<floatx4*>(row + n) = acc[ta][tb];      // (a plane's row ends on a multiple of four)
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <int RT>
hipError_t launch_project_tiles(const ProjectParams& p, DeviceInfo& dev, hipStream_t stream)
{
    const int64_t windows = (p.rows.T + 31) / 32;
    const unsigned ranges = p.pitch > 0 ? (unsigned)((p.pitch + 16 * RT - 1) / (16 * RT)) : 1;      // (rank 0: row_adapter alone)
    const dim3 grid((unsigned)(windows + p.rows.requests), ranges);
    const unsigned xcds = dev.xcds > 0 ? dev.xcds : 1;
    constexpr int KM = RT == 1 ? 4 : 2, PS = RT == 2 ? 4 : 3;
    adapter_project_tiles_kernel<RT, KM, PS><<<grid, 256, 0, stream>>>(p, (unsigned)windows, xcds);
    return hipGetLastError();
}

template <bool TRANSPOSED, int FM>
hipError_t launch_few(const FewParams& p, dim3 grid, DeviceInfo& dev, hipStream_t stream)
{
    constexpr int lds = few_stages(FM) * (32 * FM + 64) * 128;
    bool& set = dev.adapter_few_lds_set[(TRANSPOSED ? 1 : 0) + (FM == 2 ? 0 : 2)];
    if (!set) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&adapter_few_kernel<TRANSPOSED, FM>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        set = true;
    }
    adapter_few_kernel<TRANSPOSED, FM><<<grid, 256, lds, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

// Time of the product on tiles of 128 x 128 with k in s parts, in us: a compute unit with one workgroup takes 0.65 us a slice, with
// more 0.52 each (4096 columns, K = 4096: 512 rows 41, 2048 rows 72, 4096 rows 135, 8192 rows 268); the parts' planes are written
// and read at 6 TB/s, by one launch more.
static double base_us(int64_t M, int64_t N, int64_t K, int64_t s)
{
    const int64_t tiles = ((M + 127) / 128) * ((N + 127) / 128), slices = (K + BK - 1) / BK;
    const int64_t rounds = (tiles * s + 255) / 256, per = (slices + s - 1) / s;
    const double us = 7.0 + (double)per * (rounds == 1 ? 0.65 : 0.52 * (double)rounds);
    return s == 1 ? us : us + (double)(s * M * N) * 8e-6 / 6.0 + 7.0;
}

// Ways the contraction is divided along k, at least four slices each, where the tiles are fewer than the compute units: 512 rows,
// 4096 columns, K = 11008 163 us without, 101 in four parts; 1500 rows, 2048 x 2048 35 us without, 48 in two.
int adapter_base_split(int64_t M, int64_t N, int64_t K)
{
    const int64_t tiles = ((M + 127) / 128) * ((N + 127) / 128), slices = (K + BK - 1) / BK;
    int split = 1;
    if (tiles > 0 && tiles < 256)
        for (int s = 2; s <= 16 && slices / s >= 4; ++s)
            if (base_us(M, N, K, s) < base_us(M, N, K, split)) split = s;
    return split;
}

hipError_t launch_adapter_project_tiles(const ProjectParams& p, DeviceInfo& dev, hipStream_t stream)
{
    const int rt = project_factors((p.rows.T + 31) / 32 + p.rows.requests, p.pitch, dev);
    return rt == 1 ? launch_project_tiles<1>(p, dev, stream) : rt == 2 ? launch_project_tiles<2>(p, dev, stream) : launch_project_tiles<4>(p, dev, stream);
}

// Time of the product of few rows with `factors` more columns and the parts of k that it is best made in, in us: rounds of 512
// workgroups of so many slices, 0.5 us each, and 3 us around them; planes that are written and read at 4 TB/s.  (64 rows, 4096 x
// 4096: one part 34 us, four 21.7, six 21.5, sixteen 27; the model takes seven, 21.9.)
static double few_us(int64_t M, int64_t N, int64_t K, int64_t factors, int tile_m, int* split)
{
    const int64_t tiles = ((M + tile_m - 1) / tile_m) * ((N + 63) / 64 + (factors + 63) / 64), slices = (K + BK - 1) / BK;
    const int64_t width = N + (factors + 3) / 4 * 4;
    double best = 0;
    for (int s = 1; s <= 16 && (s == 1 || slices / s >= 4); ++s) {
        const double us = (double)((tiles * s + 511) / 512) * (0.5 * (double)((slices + s - 1) / s) + 3.0) + (double)(s * M * width) * 8e-6 / 4.0;
        if (s == 1 || us < best) {
            best = us;
            *split = s;
        }
    }
    return best;
}

AdapterFewPlan adapter_few_plan(int64_t M, int64_t N, int64_t K, int64_t factors)
{
    AdapterFewPlan f;
    // one row of tiles, or products of less than 2^33 multiplications: 4096 x 4096, 384 rows 38 us (tiles of 128 x 128 and
    // projections of their own 47), 512 rows 54 (54); 8192 x 8192, 128 rows 61 (70), 192 rows 95 (81)
    f.few = M > 0 && (M <= 128 || (M <= 512 && (M + 127) / 128 * 128 * N * K < (int64_t(1) << 33)));
    if (!f.few) return f;
    f.tile_m = M <= 64 ? 64 : 128;      // (65 rows, 4096 x 4096: 22 us, on two tiles of 64 rows 29)
    // The factors of the whole pool as further columns, which take what the model says or their own bytes at 4 TB/s, or a launch of
    // its own for those that are used.  us of a call from a graph, blocks of 16 pairs, further columns / a launch: 64 rows, 4096
    // x 4096, 256 blocks 24 / 31, 512 of them 37 / 31; 64 rows, 1024 x 1024, 256 blocks 11.7 / 13.5, 800 14.9 / 13.3; 256 rows, 1024
    // x 1024, 64 blocks 13.4 / 16.5, 256 16.8 / 16.5; 512 rows, 512 x 512, 64 blocks 11.9 / 14.1, 256 16.1 / 14.8, 800 26.9 / 14.2; 512
    // rows, 2048 x 2048, 64 blocks 23.3 / 26.8, 256 35.3 / 27.3, 800 61 / 27 (no wrong choice on 56 sizes from 1 to 512 rows).
    int with = 1, without = 1;
    const double more = few_us(M, N, K, factors, f.tile_m, &with) - few_us(M, N, K, 0, f.tile_m, &without);
    f.dense = std::max(more, (double)(factors * K) * 2e-6 / 4.0) <= 3.0 + 1.7e-3 * (double)K;
    f.split = f.dense ? with : without;
    f.width = N + (f.dense ? (factors + 3) / 4 * 4 : 0);
    return f;
}

hipError_t launch_adapter_few(const AdapterBase& a, const AdapterFewPlan& plan, const AdapterRows& rows, int32_t* row_adapter, DeviceInfo& dev,
                              hipStream_t stream)
{
    FewParams p = {};
    p.A = a.A;
    p.W = a.W;
    p.F = a.F;
    p.M = a.M; p.N = a.N; p.K = a.K;
    p.ldw = a.transposed ? a.N : a.K;
    p.pitch = a.blocked ? bf16_pitch(p.ldw) : 0;
    p.factors = plan.dense ? rows.count * rows.rank : 0;
    p.width = plan.width;
    p.planes = a.planes;
    p.split = plan.split;
    p.tiles_m = (int)((a.M + plan.tile_m - 1) / plan.tile_m);
    p.tiles_w = (int)((a.N + 63) / 64);
    p.rows = rows;
    p.row_adapter = row_adapter;
    const dim3 grid((unsigned)(p.tiles_m * (p.tiles_w + (p.factors + 63) / 64) + (row_adapter ? 1 : 0)), (unsigned)plan.split);
    if (plan.tile_m == 64) return a.transposed ? launch_few<true, 2>(p, grid, dev, stream) : launch_few<false, 2>(p, grid, dev, stream);
    return a.transposed ? launch_few<true, 4>(p, grid, dev, stream) : launch_few<false, 4>(p, grid, dev, stream);
}

hipError_t launch_adapter_base_bf16(const AdapterBase& a, DeviceInfo& dev, hipStream_t stream)
{
    if (a.M <= 0) return hipSuccess;
    BaseParams p = {};
    p.A = a.A;
    p.W = a.W;
    p.M = a.M; p.N = a.N; p.K = a.K;
    p.ldw = a.transposed ? a.N : a.K;
    p.pitch = a.blocked ? bf16_pitch(p.ldw) : 0;
    p.planes = a.planes;
    p.split = a.split;
    p.out = a.out;
    p.row_adapter = a.row_adapter;
    p.Hx = a.Hx;
    p.H = a.H;
    p.F = a.F;
    p.ranks = a.ranks;
    p.count = (int)a.count;
    p.rank = a.rank;
    p.num_xcd = dev.xcds > 0 ? dev.xcds : 1;
    // Tiles of 256 x 256: 1.6 us a slice.  They do more with what they read, the small ones fill the last round better (4096
    // columns, K = 4096: 2048 rows 99 us and on small tiles 72, 4096 rows 110 and 135, 5000 rows 186 and 162, 8192 rows 210 and 268).
    const int64_t big = ((a.M + 255) / 256) * ((a.N + 255) / 256), slices = (a.K + BK - 1) / BK;
    const double big_us = (double)((big + 255) / 256) * (5.0 + 1.6 * (double)slices);
    if (a.split > 1) return a.transposed ? launch_base<4, 4, true, true>(p, dev, stream) : launch_base<4, 4, false, true>(p, dev, stream);
    if (big_us <= base_us(a.M, a.N, a.K, 1)) return a.transposed ? launch_base<8, 8, true, false>(p, dev, stream) : launch_base<8, 8, false, false>(p, dev, stream);
    return a.transposed ? launch_base<4, 4, true, false>(p, dev, stream) : launch_base<4, 4, false, false>(p, dev, stream);
}

}  // namespace sfb
