// Internal launch interface of the adapter calls (factor blocks beside a shared projection, their gradients) and of the
// norm and clipping of gradients.  Every function only enqueues work on `stream` and returns the launch status.
#pragma once
#include "../../include/sfb.h"
#include "kernels.h"

namespace sfb {

// Which rows belong to whom: request q is the rows start[q] .. start[q + 1] - 1 and uses factor block adapter[q] of the pool
// (outside [0, count): none).  Device arrays; the kernels clamp what they read from them.
struct AdapterRows {
    const int64_t* start;
    const int32_t* adapter;
    int64_t requests;
    const int32_t* ranks;      // nullable: every block has all `rank` pairs
    const float* scale;        // nullable: 1
    int64_t count;             // factor blocks in the pool
    int rank;                  // pairs a block has room for
    int64_t T;                 // rows of the buffers
};
// Leading dimension of the kernels' own array of projections: `rank` rounded up to whole MFMA tiles.
__host__ __device__ inline int adapter_pitch(int rank) { return (rank + 15) / 16 * 16; }
constexpr int ROW_NONE = -1, ROW_OUTSIDE = -2;      // row_adapter: a request without a block; no request at all

// H[t][r] = scale_a sum_k X[t][k] F_a[r][k], F [count][rank][K] of X's type; zeros for r >= ranks[a] and for rows without a
// block.  row_adapter[t] (written): the block of row t, ROW_NONE or ROW_OUTSIDE (a `start` that is not as it has to be may
// leave entries as they were: what reads them passes over numbers outside the pool).  H: [T][adapter_pitch(rank)] fp32;
// H_out (nullable): [T][rank], rows of a request only.
struct AdapterProjectArgs {
    AdapterRows rows;
    const void* X;
    const void* F;
    int64_t K;
    bool bf16;
    int32_t* row_adapter;
    float* H;
    float* H_out;
    uint16_t* Hx;              // nullable: [T][2 adapter_pitch(rank)]: H in two bf16 terms, the 16 first and then the 16 second ones
                               // of every 16 pairs
};
hipError_t launch_adapter_project(const AdapterProjectArgs& a, DeviceInfo& dev, hipStream_t stream);

// A bf16 [M][K] row-major times B(n, k) = W[n][k] or, transposed, W[k][n], with W [rows][cols] bf16 row-major or a bf16 operand
// in blocks of 256 x 64.  split 1: out[t][n] = sum_k A[t][k] B(n, k) + sum_r H[t][r] F_a[r][n] for the rows of requests (H and Hx:
// launch_adapter_project's).  More: planes[s][t][n], the s-th part of the first sum alone, for launch_adapter_join.
struct AdapterBase {
    const uint16_t* A;
    const uint16_t* W;
    bool transposed, blocked;
    int64_t M, N, K;
    float* planes;             // [split][M][N]
    int split;
    uint16_t* out;
    const int32_t* row_adapter;
    const uint16_t* Hx;
    const float* H;
    const uint16_t* F;
    const int32_t* ranks;
    int64_t count;
    int rank;
};
hipError_t launch_adapter_base_bf16(const AdapterBase& a, DeviceInfo& dev, hipStream_t stream);
int adapter_base_split(int64_t M, int64_t N, int64_t K);

// The same for few rows: planes alone, of `width` columns; with `dense` those behind the N of the product are A times the
// factors of all blocks ([count][rank][K]).  row_adapter (nullable): written as launch_adapter_project does.
struct AdapterFewPlan {
    bool few = false, dense = false;
    int split = 1, tile_m = 64;
    int64_t width = 0;
};
AdapterFewPlan adapter_few_plan(int64_t M, int64_t N, int64_t K, int64_t factors);
hipError_t launch_adapter_few(const AdapterBase& a, const AdapterFewPlan& plan, const AdapterRows& rows, int32_t* row_adapter, DeviceInfo& dev,
                              hipStream_t stream);

// fp32 matrices with zeros behind their rows and columns (cols_out % 4 == 0; rows_out 0: none), both by one launch.
struct AdapterPad {
    const float* src = nullptr;
    float* dst = nullptr;
    int64_t rows = 0, cols = 0, rows_out = 0, cols_out = 0;
};
hipError_t launch_adapter_pad(const AdapterPad& a, const AdapterPad& b, hipStream_t stream);

// out[t][n] = sum_s planes[s][t][n] + sum_r H[t][r] F_a[r][n] for the rows of requests; out and F [count][rank][N] fp32 or bf16.
struct AdapterJoinArgs {
    const float* planes;       // [split][T][width]
    int64_t width;
    int split;
    const int32_t* row_adapter;
    bool dense;                // H is made from the planes and written, otherwise read
    float* H;                  // [T][adapter_pitch(rank)]
    float* H_out;              // dense: nullable, [T][rank]
    const float* scale;        // dense
    const void* F;
    const int32_t* ranks;
    int64_t count;
    int rank;
    void* out;
    bool bf16;
    int64_t T, N;
};
hipError_t launch_adapter_join(const AdapterJoinArgs& a, hipStream_t stream);

// out[a][r][c] = sum over the rows t of block a of H[t][r] G[t][c] for two such sums at once (r >= ranks[a]: zeros).
struct AdapterOuter {
    const float* H;
    int64_t ldh;
    const void* G;             // [T][C]
    int64_t C;
    float* out;                // [count][rank][C]
};
struct AdapterOuterArgs {
    AdapterOuter sum[2];
    const int32_t* row_adapter;      // 16-byte aligned, with room for a multiple of eight
    const int64_t* start;
    const int32_t* adapter;
    int64_t requests;
    const int32_t* ranks;
    int64_t count;
    int rank;
    bool bf16;
    int64_t T;
    float* padded;             // bf16: room for [T][adapter_pitch(rank)] where an H has rows that are no multiple of 16 bytes
    float* partial;            // with adapter_outer_splits > 1: so many times the size of both outputs
};
hipError_t launch_adapter_outer(const AdapterOuterArgs& a, DeviceInfo& dev, hipStream_t stream);
// Parts that the rows are divided into, C0 and C1 the columns of the two sums.
int adapter_outer_splits(int64_t C0, int64_t C1, int64_t count, int rank, bool bf16, int64_t T);

// Norm over the tensors of a list and their scaling.  partial: grad_norm_partials(...) + 1 doubles.  Where launch_clip follows
// (clip), with the same list and `partial`, it may be that which writes *norm.  table (nullable): what tensor_table_fill wrote
// for this list, in device memory.
int64_t grad_norm_partials(const sfb_tensor* list, int64_t count);
int64_t tensor_table_bytes(int64_t count);
void tensor_table_fill(const sfb_tensor* list, int64_t count, void* host);
hipError_t launch_grad_norm(const sfb_tensor* list, int64_t count, const void* table, double* partial, float* norm, bool clip, hipStream_t stream);
hipError_t launch_clip(const sfb_tensor* list, int64_t count, const void* table, const double* partial, double max_norm, float* norm, hipStream_t stream);

}  // namespace sfb
