// The product of bf16 rows with a shared bf16 matrix as it lies in memory, for the calls with factor blocks beside it:
//
//   forward   base[t][j] = sum_d X[t][d] W[j][d]         both operands contiguous along k
//   backward  base[t][d] = sum_j dY[t][j] W[j][d]        W contiguous along the output's columns
//
// Neither operand is copied or transposed first.  Tiles go from memory straight into LDS through buffer descriptors, whose
// range check fills what lies behind the last row, column or k with zeros.  In the backward W's tile lies in LDS as 64 rows
// (k) of BN columns, and the matrix operand is read with the transposing LDS read (four rows of 16 columns a group of 16
// lanes; lane i gets column i).
// W is the first operand of the MFMA, so a lane's results are one row of the output, and the columns are dealt to the MFMA
// tiles such that a lane owns runs of eight consecutive ones and the four lanes of a row 32 of them.
#include "adapter.h"
#include "planes.h"

namespace sfb {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct BaseParams {
    const uint16_t* A;
    const uint16_t* W;
    int64_t M, N, K, ldw;
    int64_t pitch;             // blocked W: columns of the operand; 0: rows of ldw
    float* planes;
    int split;
    int tiles_m, tiles_n, group_m, num_xcd;
};

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;

// A buffer descriptor of 2 GiB from base on (raw bytes; reads beyond it give zeros).
__device__ __forceinline__ u32x4 descriptor(uint64_t base)
{
    const uint64_t b = uniform64(base);
    return u32x4{(uint32_t)b, (uint32_t)(b >> 32), OUT_OF_RANGE, 0x00020000u};
}
__device__ __forceinline__ void buffer_to_lds_16(uint32_t lds_addr, u32x4 rsrc, uint32_t voff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(voff), "s"(rsrc) : "memory");
}

// Column of the output's tile that row i of MFMA tile tb of a wavefront holds.
__device__ __forceinline__ int column_of(int tb, int i) { return 32 * (tb >> 1) + 8 * (i >> 2) + 4 * (tb & 1) + (i & 3); }

// Tiles of 32 TM rows x 32 TN columns, 2 x 2 wavefronts of 16 TM x 16 TN.
template <int TM, int TN, bool TRANSPOSED>
__global__ __launch_bounds__(256) void adapter_base_kernel(BaseParams p)
{
    constexpr int TBM = 32 * TM, TBN = 32 * TN;
    constexpr uint32_t A_BYTES = TBM * 128, STAGE_BYTES = A_BYTES + TBN * 128;
    extern __shared__ u32x4 smem[];
    char* const lds = reinterpret_cast<char*>(smem);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm0 = (wave >> 1) * 16 * TM, wn0 = (wave & 1) * 16 * TN;

    // each XCD a contiguous range of a raster of groups of group_m row-tiles, row-tile index fastest
    int64_t m0, n0;
    {
        const uint32_t tiles = gridDim.x, xcds = (uint32_t)p.num_xcd, tiles_n = (uint32_t)p.tiles_n, tiles_m = (uint32_t)p.tiles_m;
        const uint32_t x = blockIdx.x % xcds, wi = blockIdx.x / xcds, q = tiles / xcds, r = tiles % xcds;
        const uint32_t t = x * q + (x < r ? x : r) + wi;
        const uint32_t per_group = (uint32_t)p.group_m * tiles_n;
        const uint32_t grp = t / per_group, rr = t % per_group, first = grp * (uint32_t)p.group_m;
        const uint32_t gm = tiles_m - first < (uint32_t)p.group_m ? tiles_m - first : (uint32_t)p.group_m;
        m0 = (int64_t)(first + rr % gm) * TBM;
        n0 = (int64_t)(rr / gm) * TBN;
    }
    const int64_t slices = (p.K + BK - 1) / BK;
    const int64_t s_begin = slices * blockIdx.y / p.split, s_end = slices * (blockIdx.y + 1) / p.split;
    const int nk = (int)(s_end - s_begin);

    // ---- loader: A (and W, k-contiguous) as 128-byte LDS rows of 64 k, chunk c of row r in slot c ^ swz(r)
    const uint32_t lda = (uint32_t)p.K * 2u, ldw = p.pitch ? (uint32_t)BK * 2u : (uint32_t)p.ldw * 2u;
    uint32_t offA[TM], offB[TN];
    const int last_m = (int)(p.M - m0 < TBM ? p.M - m0 : TBM), last_n = (int)(p.N - n0 < TBN ? p.N - n0 : TBN);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r = 8 * (TM * wave + i) + (lane >> 3);
        offA[i] = r < last_m ? (uint32_t)r * lda + (uint32_t)(((lane & 7) ^ swz(r)) << 4) : OUT_OF_RANGE;
    }
    // W, transposed: LDS rows of TBN columns, 16-byte chunk u of row r in slot u ^ 4 (r % 4)
    constexpr int SLOTS = TBN / 8, RPL = 64 / SLOTS;      // chunks of a row, rows of a load
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
    auto w_address = [&](int64_t k0) {      // W's tile at slice k0
        if (TRANSPOSED)
            return reinterpret_cast<uint64_t>(p.W) + (p.pitch ? (uint64_t)(((k0 / BM) * (p.pitch / BK) + n0 / BK) * (BM * BK) + (k0 % BM) * BK) * 2u
                                                              : (uint64_t)(k0 * p.ldw + n0) * 2u);
        return reinterpret_cast<uint64_t>(p.W) + (p.pitch ? (uint64_t)(((n0 / BM) * (p.pitch / BK) + k0 / BK) * (BM * BK) + (n0 % BM) * BK) * 2u
                                                          : (uint64_t)(n0 * p.ldw + k0) * 2u);
    };
    auto issue = [&](int s) {
        const int64_t k0 = (s_begin + s) * BK;
        const u32x4 ra = descriptor(reinterpret_cast<uint64_t>(p.A) + (uint64_t)(m0 * p.K + k0) * 2u);
        const u32x4 rb = descriptor(w_address(k0));
        const uint32_t dst = lds_base + (uint32_t)(s & 1) * STAGE_BYTES;
        const int left = (int)(p.K - k0 < BK ? p.K - k0 : BK);      // (a multiple of eight)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int r = 8 * (TM * wave + i) + (lane >> 3);
            buffer_to_lds_16(dst + (uint32_t)(TM * wave + i) * 1024u, ra, 8 * ((lane & 7) ^ swz(r)) < left ? offA[i] : OUT_OF_RANGE);
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            bool in;
            if (TRANSPOSED) {
                in = (TN * wave + i) * RPL + lane / SLOTS < left;
            } else {
                const int r = 8 * (TN * wave + i) + (lane >> 3);
                in = 8 * ((lane & 7) ^ swz(r)) < left;
            }
            buffer_to_lds_16(dst + A_BYTES + (uint32_t)(TN * wave + i) * 1024u, rb, in ? offB[i] : OUT_OF_RANGE);
        }
    };

    floatx4 acc[TM][TN];
#pragma unroll
    for (int ta = 0; ta < TM; ++ta)
#pragma unroll
        for (int tb = 0; tb < TN; ++tb) acc[ta][tb] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (nk > 0) issue(0);
    if (nk > 1) issue(1);
    for (int s = 0; s < nk; ++s) {
        if (s + 1 < nk)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TM + TN) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const char* const stage = lds + (uint32_t)(s & 1) * STAGE_BYTES;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            bf16x8 a[TM], b[TN];
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                const int r = wm0 + 16 * t + l16;
                a[t] = *reinterpret_cast<const bf16x8*>(stage + r * 128 + (((4 * ks + quad) ^ swz(r)) << 4));
            }
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                if (TRANSPOSED) {
                    // lane i of a group: row i / 4 of four, columns of piece i % 4 (column_of(t, 4 (i % 4)) ..)
                    const int r = 32 * ks + 8 * quad + (l16 >> 2), n = wn0 + column_of(t, 4 * (l16 & 3));
                    const uint32_t at = A_BYTES + (uint32_t)r * (TBN * 2) + (uint32_t)(((n >> 3) ^ ((r & 3) << 2)) << 4) + (uint32_t)(n & 7) * 2u;
                    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(stage + at));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(stage + at + 4 * (TBN * 2)));
                    b[t] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                } else {
                    const int r = wn0 + 16 * t + l16;
                    b[t] = *reinterpret_cast<const bf16x8*>(stage + A_BYTES + r * 128 + (((4 * ks + quad) ^ swz(r)) << 4));
                }
            }
#pragma unroll
            for (int tb = 0; tb < TN; ++tb)
#pragma unroll
                for (int ta = 0; ta < TM; ++ta) acc[ta][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[tb], a[ta], acc[ta][tb], 0, 0, 0);
        }
        if (s + 2 < nk) {
            __syncthreads();                 // every wavefront has read the stage
            issue(s + 2);
        }
    }
    // register i of lane (q, c) of tile (ta, tb): row 16 ta + c, column column_of(tb, 4 q + i)
#pragma unroll
    for (int ta = 0; ta < TM; ++ta) {
        const int64_t m = m0 + wm0 + 16 * ta + l16;
        if (m >= p.M) continue;
        float* const row = p.planes + ((int64_t)blockIdx.y * p.M + m) * p.N + n0 + wn0;
#pragma unroll
        for (int tb = 0; tb < TN; ++tb) {
            const int n = column_of(tb, 4 * quad);
            if (n0 + wn0 + n < p.N) *reinterpret_cast<floatx4*>(row + n) = acc[ta][tb];
        }
    }
}

template <int TM, int TN>
hipError_t launch_base(BaseParams& p, bool transposed, DeviceInfo& dev, hipStream_t stream)
{
    constexpr int lds = 2 * (TM + TN) * 32 * 128;
    p.tiles_m = (int)((p.M + 32 * TM - 1) / (32 * TM));
    p.tiles_n = (int)((p.N + 32 * TN - 1) / (32 * TN));
    p.group_m = 8;
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n), (unsigned)p.split);
    if (transposed)
        adapter_base_kernel<TM, TN, true><<<grid, 256, lds, stream>>>(p);
    else
        adapter_base_kernel<TM, TN, false><<<grid, 256, lds, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

int adapter_base_split(int64_t, int64_t, int64_t) { return 1; }

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
    p.num_xcd = dev.xcds > 0 ? dev.xcds : 1;
    return launch_base<4, 4>(p, a.transposed, dev, stream);
}

}  // namespace sfb
