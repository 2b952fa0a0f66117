// Norm over the tensors of a list and their scaling to a largest norm.
//
//   norm = sqrt(sum_i sum_k g_i[k]^2),   g_i <- g_i min(1, max_norm / norm)
//
// Squares are added up in 64 bits (fp32 squares overflow from 1.8e19 on and vanish below 1e-23), each workgroup its piece of
// one tensor, the pieces' sums in their order: the same bits on every call.
//
// Memory bounds both passes.  A thread has eight 16-byte loads in flight (one: 2.5 TB/s), loads and stores are non-temporal
// (norm of 1.7 GB in 150 tensors 307 -> 268 us, 6.4 TB/s; clipping of 435 MB in 300 tensors 299 -> 265 us).
#include "adapter.h"
#include "device.h"

namespace sfb {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int64_t TARGET = 4096;    // pieces of a whole list, about (1024: a list of 1.7 GB 6 % slower, too few to even out)
constexpr int64_t MOST = 1 << 23;   // workgroups of a launch

// Tensors of one launch: their description travels as a kernel argument (4 KB of them).
template <int N, bool CLIP>
struct ListParams {
    const void* src[N];
    void* dst[CLIP ? N : 1];
    uint32_t first[N + 1];          // first workgroup of a tensor
    uint32_t tail[N];               // elements of its last piece; BF16_FLAG
    int count;
    int64_t piece;                  // elements of a workgroup
};
constexpr uint32_t BF16_FLAG = 0x80000000u;
typedef ListParams<240, false> NormList;
typedef ListParams<160, true> ClipList;
// Any number of tensors in one launch, their description in device memory.
struct TableParams {
    const void* const* src;
    void* const* dst;
    const uint32_t* first;
    const uint32_t* tail;
    int count;
    int64_t piece;
};

struct Piece {
    const char* src;
    char* dst;
    int64_t n;                      // elements
    bool bf16, vec;                 // vec: 16-byte accesses
};
template <typename List>
__device__ __forceinline__ Piece piece_at(const List& p, uint32_t block, bool clip)
{
    int lo = 0, hi = p.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.first[mid] <= block)
            lo = mid;
        else
            hi = mid;
    }
    Piece r;
    const uint32_t tail = p.tail[lo];
    r.bf16 = tail & BF16_FLAG;
    const int64_t at = (int64_t)(block - p.first[lo]) * p.piece * (r.bf16 ? 2 : 4);
    r.src = static_cast<const char*>(p.src[lo]) + at;
    r.dst = clip ? static_cast<char*>(p.dst[lo]) + at : nullptr;
    r.n = block + 1 == p.first[lo + 1] ? (int64_t)(tail & ~BF16_FLAG) : p.piece;
    r.vec = ((reinterpret_cast<uintptr_t>(r.src) | reinterpret_cast<uintptr_t>(r.dst)) & 15u) == 0;
    return r;
}

__device__ __forceinline__ float element(const Piece& p, int64_t i)
{
    return p.bf16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p.src)[i] << 16) : reinterpret_cast<const float*>(p.src)[i];
}

__device__ __forceinline__ float scaled(float v, double coef) { return (float)((double)v * coef); }

template <int WAVES>
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[WAVES];
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += part[w];
    return v;
}

__device__ __forceinline__ double square(double sum, u32x4 v, bool bf16)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t w = v[e];
        const double x = (double)__uint_as_float(bf16 ? w & 0xffff0000u : w);
        sum = fma(x, x, sum);
        if (bf16) {
            const double y = (double)__uint_as_float(w << 16);
            sum = fma(y, y, sum);
        }
    }
    return sum;
}

constexpr int AHEAD = 8;            // 16-byte loads of a thread in flight

template <typename List>
__global__ __launch_bounds__(256) void grad_norm_kernel(List p, double* partial)
{
    const Piece t = piece_at(p, blockIdx.x, false);
    double sum = 0.0;
    int64_t i = 0;
    if (t.vec) {
        const int64_t chunks = t.n / (t.bf16 ? 8 : 4);
        const u32x4* src = reinterpret_cast<const u32x4*>(t.src);
        int64_t c = threadIdx.x;
        for (; c + 256 * (AHEAD - 1) < chunks; c += 256 * AHEAD) {
            u32x4 v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) v[k] = __builtin_nontemporal_load(src + c + 256 * k);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) sum = square(sum, v[k], t.bf16);
        }
        for (; c < chunks; c += 256) sum = square(sum, src[c], t.bf16);
        i = chunks * (t.bf16 ? 8 : 4);
    }
    for (i += threadIdx.x; i < t.n; i += 256) {
        const double x = (double)element(t, i);
        sum = fma(x, x, sum);
    }
    sum = block_sum<4>(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <int WAVES>
__device__ __forceinline__ double sum_of(const double* partial, int64_t count)
{
    double sum = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < count; i += 64 * WAVES) sum += partial[i];
    return block_sum<WAVES>(sum);
}

// partial[count] = the sum of the `count` before it; *norm its root.
__global__ __launch_bounds__(1024) void grad_norm_final_kernel(double* partial, int64_t count, float* norm)
{
    const double sum = sum_of<16>(partial, count);
    if (threadIdx.x == 0) {
        partial[count] = sum;
        *norm = (float)sqrt(sum);
    }
}

// norm: null, or where the one workgroup with `writes` puts it (the sum is then made here, of `count` pieces).
template <typename List>
__global__ __launch_bounds__(256) void clip_kernel(List p, const double* partial, int64_t count, double max_norm, float* norm, bool writes)
{
    const uint32_t block = gridDim.x - 1 - blockIdx.x;      // what the first pass has read last is still in the caches
    const Piece t = piece_at(p, block, true);
    const double total = sqrt(norm ? sum_of<4>(partial, count) : partial[count]);
    if (writes && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    // (a norm that is no number: neither is this; in 64 bits, since an fp32 scale below 1e-38 would lose its digits)
    const double coef = total <= max_norm ? 1.0 : max_norm / total;
    if (coef == 1.0 && t.src == t.dst) return;
    int64_t i = 0;
    if (t.vec) {
        const int64_t chunks = t.n / (t.bf16 ? 8 : 4);
        const u32x4* src = reinterpret_cast<const u32x4*>(t.src);
        u32x4* dst = reinterpret_cast<u32x4*>(t.dst);
        auto scale = [&](u32x4 v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = v[e];
                v[e] = t.bf16 ? pack_bf16(scaled(__uint_as_float(w << 16), coef), scaled(__uint_as_float(w & 0xffff0000u), coef))
                              : __float_as_uint(scaled(__uint_as_float(w), coef));
            }
            return v;
        };
        int64_t c = threadIdx.x;
        for (; c + 256 * (AHEAD - 1) < chunks; c += 256 * AHEAD) {
            u32x4 v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) v[k] = __builtin_nontemporal_load(src + c + 256 * k);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) __builtin_nontemporal_store(scale(v[k]), dst + c + 256 * k);
        }
        for (; c < chunks; c += 256) dst[c] = scale(src[c]);
        i = chunks * (t.bf16 ? 8 : 4);
    }
    for (i += threadIdx.x; i < t.n; i += 256) {
        const float v = scaled(element(t, i), coef);
        if (t.bf16)
            reinterpret_cast<uint16_t*>(t.dst)[i] = (uint16_t)pack_bf16(v, 0.f);
        else
            reinterpret_cast<float*>(t.dst)[i] = v;
    }
}

int64_t piece_of(const sfb_tensor* list, int64_t count)
{
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) total += list[i].n;
    const int64_t per = (total + TARGET - 1) / TARGET;
    return per <= 4096 ? 4096 : per <= (1 << 30) ? (per + 4095) / 4096 * 4096 : 1 << 30;
}

// Whether every workgroup of the second pass adds up the pieces' sums itself, or a launch of its own does: few pieces, or long
// ones beside which that is nothing.  64 tensors of 65536 elements (1024 pieces) 18 us and 19 with the launch, 4000 of 4096 50 and 44,
// 8 of 2^24 (4096 pieces) 284 and 287, 12000 of 4096 161 and 119.
bool sums_itself(const sfb_tensor* list, int64_t count, int64_t pieces)
{
    return pieces <= 2048 || (pieces <= 8192 && piece_of(list, count) >= 32768);
}

// Last piece of a tensor of n elements, and its type.
uint32_t tail_of(const sfb_tensor& t, int64_t pieces, int64_t piece)
{
    return (uint32_t)(t.n - (pieces - 1) * piece) | (t.dtype == SFB_BF16 ? BF16_FLAG : 0u);
}

// run(list, workgroups, first workgroup of the launch) for every launch that a list takes.
template <int N, bool CLIP, typename F>
hipError_t for_list(const sfb_tensor* list, int64_t count, F&& run)
{
    ListParams<N, CLIP> p;
    p.piece = piece_of(list, count);
    p.count = 0;
    uint32_t blocks = 0;
    int64_t done = 0;
    for (int64_t i = 0; i <= count; ++i) {
        if (p.count == N || (i == count && p.count > 0)) {
            p.first[p.count] = blocks;
            const hipError_t e = run(p, blocks, done);
            if (e != hipSuccess) return e;
            done += blocks;
            p.count = 0;
            blocks = 0;
        }
        if (i == count || list[i].n == 0) continue;
        const int k = p.count++;
        const int64_t pieces = (list[i].n + p.piece - 1) / p.piece;
        p.src[k] = list[i].src;
        if (CLIP) p.dst[k] = list[i].dst;
        p.tail[k] = tail_of(list[i], pieces, p.piece);
        p.first[k] = blocks;
        blocks += (uint32_t)pieces;
    }
    return hipSuccess;
}

TableParams table_params(const sfb_tensor* list, int64_t count, const void* table)
{
    TableParams p = {};
    for (int64_t i = 0; i < count; ++i) p.count += list[i].n > 0;
    const char* at = static_cast<const char*>(table);
    p.src = reinterpret_cast<const void* const*>(at);
    p.dst = reinterpret_cast<void* const*>(at + 8 * count);
    p.first = reinterpret_cast<const uint32_t*>(at + 16 * count);
    p.tail = p.first + count + 1;
    p.piece = piece_of(list, count);
    return p;
}

}  // namespace

int64_t tensor_table_bytes(int64_t count) { return 24 * count + 4; }

void tensor_table_fill(const sfb_tensor* list, int64_t count, void* host)
{
    char* const at = static_cast<char*>(host);
    const void** const src = reinterpret_cast<const void**>(at);
    void** const dst = reinterpret_cast<void**>(at + 8 * count);
    uint32_t* const first = reinterpret_cast<uint32_t*>(at + 16 * count);
    uint32_t* const tail = first + count + 1;
    const int64_t piece = piece_of(list, count);
    uint32_t blocks = 0;
    int64_t k = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (list[i].n == 0) continue;
        const int64_t pieces = (list[i].n + piece - 1) / piece;
        src[k] = list[i].src;
        dst[k] = list[i].dst;
        tail[k] = tail_of(list[i], pieces, piece);
        first[k++] = blocks;
        blocks += (uint32_t)pieces;
    }
    for (; k <= count; ++k) {      // (behind the tensors that have elements)
        first[k] = blocks;
        if (k < count) {
            src[k] = nullptr;
            dst[k] = nullptr;
            tail[k] = 0;
        }
    }
}

int64_t grad_norm_partials(const sfb_tensor* list, int64_t count)
{
    const int64_t piece = piece_of(list, count);
    int64_t blocks = 0;
    for (int64_t i = 0; i < count; ++i) blocks += (list[i].n + piece - 1) / piece;
    return blocks;
}

hipError_t launch_grad_norm(const sfb_tensor* list, int64_t count, const void* table, double* partial, float* norm, bool clip, hipStream_t stream)
{
    const int64_t pieces = grad_norm_partials(list, count);
    if (table && pieces > 0 && pieces <= MOST) {
        const TableParams p = table_params(list, count, table);
        grad_norm_kernel<TableParams><<<(unsigned)pieces, 256, 0, stream>>>(p, partial);
    } else {
        const hipError_t e = for_list<240, false>(list, count, [&](const NormList& p, uint32_t blocks, int64_t done) {
            grad_norm_kernel<NormList><<<blocks, 256, 0, stream>>>(p, partial + done);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    if (!(clip && pieces > 0 && sums_itself(list, count, pieces))) grad_norm_final_kernel<<<1, 1024, 0, stream>>>(partial, pieces, norm);
    return hipGetLastError();
}

hipError_t launch_clip(const sfb_tensor* list, int64_t count, const void* table, const double* partial, double max_norm, float* norm, hipStream_t stream)
{
    const int64_t pieces = grad_norm_partials(list, count);
    float* const own = sums_itself(list, count, pieces) ? norm : nullptr;
    if (table && pieces > 0 && pieces <= MOST) {
        const TableParams p = table_params(list, count, table);
        clip_kernel<TableParams><<<(unsigned)pieces, 256, 0, stream>>>(p, partial, pieces, max_norm, own, own != nullptr);
        return hipGetLastError();
    }
    return for_list<160, true>(list, count, [&](const ClipList& p, uint32_t blocks, int64_t done) {
        clip_kernel<ClipList><<<blocks, 256, 0, stream>>>(p, partial, pieces, max_norm, own, own && done == 0);
        return hipGetLastError();
    });
}

}  // namespace sfb
