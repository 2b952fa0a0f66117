// Norm over the tensors of a list and their scaling to a largest norm.
//
//   norm = sqrt(sum_i sum_k g_i[k]^2),   g_i <- g_i min(1, max_norm / norm)
//
// Squares are added up in 64 bits (fp32 squares overflow from 1.8e19 on and vanish below 1e-23), each workgroup its piece of
// one tensor, the pieces' sums by one workgroup in their order: the same bits on every call.
#include "adapter.h"
#include "device.h"

namespace sfb {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int LIST = 96;            // tensors of a launch: their description travels as a kernel argument
constexpr int64_t TARGET = 1024;    // workgroups over a whole list, about

struct ListParams {
    const void* src[LIST];
    void* dst[LIST];
    int64_t n[LIST];
    uint32_t first[LIST + 1];       // first workgroup of a tensor
    uint8_t bf16[LIST], vec[LIST];
    int count;
    int64_t piece;                  // elements of a workgroup
};

__device__ __forceinline__ int tensor_of(const ListParams& p, uint32_t block)
{
    int lo = 0, hi = p.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.first[mid] <= block)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float element(const void* p, bool bf16, int64_t i)
{
    return bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16) : static_cast<const float*>(p)[i];
}

__device__ __forceinline__ float scaled(float v, double coef) { return (float)((double)v * coef); }

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[4];
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0] + part[1] + part[2] + part[3];
    __syncthreads();
    return v;
}

__global__ __launch_bounds__(256) void grad_norm_kernel(ListParams p, double* partial)
{
    const int t = tensor_of(p, blockIdx.x);
    const bool bf16 = p.bf16[t];
    const int64_t begin = (int64_t)(blockIdx.x - p.first[t]) * p.piece, end = begin + p.piece < p.n[t] ? begin + p.piece : p.n[t];
    double sum = 0.0;
    int64_t i = begin;
    if (p.vec[t]) {
        const int per = bf16 ? 8 : 4;
        const int64_t whole = begin + (end - begin) / per * per;
        for (i = begin + (int64_t)threadIdx.x * per; i < whole; i += 256 * per) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.src[t]) + i * (bf16 ? 2 : 4));
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
        }
        i = whole;
    }
    for (i += threadIdx.x; i < end; i += 256) {
        const double x = (double)element(p.src[t], bf16, i);
        sum = fma(x, x, sum);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// partial[count] = the sum of the `count` before it; *norm its root.
__global__ __launch_bounds__(256) void grad_norm_final_kernel(double* partial, int64_t count, float* norm)
{
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += 256) sum += partial[i];
    sum = block_sum(sum);
    if (threadIdx.x == 0) {
        partial[count] = sum;
        *norm = (float)sqrt(sum);
    }
}

__global__ __launch_bounds__(256) void clip_kernel(ListParams p, const double* total, double max_norm)
{
    const int t = tensor_of(p, blockIdx.x);
    const bool bf16 = p.bf16[t];
    const double norm = sqrt(*total);
    // (a norm that is no number: neither is this; in 64 bits, since an fp32 scale below 1e-38 would lose its digits)
    const double coef = norm <= max_norm ? 1.0 : max_norm / norm;
    if (coef == 1.0 && p.src[t] == p.dst[t]) return;
    const int64_t begin = (int64_t)(blockIdx.x - p.first[t]) * p.piece, end = begin + p.piece < p.n[t] ? begin + p.piece : p.n[t];
    int64_t i = begin;
    if (p.vec[t]) {
        const int per = bf16 ? 8 : 4;
        const int64_t whole = begin + (end - begin) / per * per;
        for (i = begin + (int64_t)threadIdx.x * per; i < whole; i += 256 * per) {
            u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.src[t]) + i * (bf16 ? 2 : 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = v[e];
                v[e] = bf16 ? pack_bf16(scaled(__uint_as_float(w << 16), coef), scaled(__uint_as_float(w & 0xffff0000u), coef))
                            : __float_as_uint(scaled(__uint_as_float(w), coef));
            }
            *reinterpret_cast<u32x4*>(static_cast<char*>(p.dst[t]) + i * (bf16 ? 2 : 4)) = v;
        }
        i = whole;
    }
    for (i += threadIdx.x; i < end; i += 256) {
        const float v = scaled(element(p.src[t], bf16, i), coef);
        if (bf16)
            static_cast<uint16_t*>(p.dst[t])[i] = (uint16_t)pack_bf16(v, 0.f);
        else
            static_cast<float*>(p.dst[t])[i] = v;
    }
}

int64_t piece_of(const sfb_tensor* list, int64_t count)
{
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) total += list[i].n;
    const int64_t per = (total + TARGET - 1) / TARGET;
    return per <= 4096 ? 4096 : (per + 4095) / 4096 * 4096;
}

// run(ListParams, workgroups, first workgroup of the launch) for every launch that a list takes.
template <typename F>
hipError_t for_list(const sfb_tensor* list, int64_t count, F&& run)
{
    ListParams p;
    p.piece = piece_of(list, count);
    p.count = 0;
    uint32_t blocks = 0;
    int64_t done = 0;
    for (int64_t i = 0; i <= count; ++i) {
        if (p.count == LIST || (i == count && p.count > 0)) {
            p.first[p.count] = blocks;
            const hipError_t e = run(p, blocks, done);
            if (e != hipSuccess) return e;
            done += blocks;
            p.count = 0;
            blocks = 0;
        }
        if (i == count || list[i].n == 0) continue;
        const int k = p.count++;
        p.src[k] = list[i].src;
        p.dst[k] = list[i].dst;
        p.n[k] = list[i].n;
        p.bf16[k] = list[i].dtype == SFB_BF16;
        p.vec[k] = ((reinterpret_cast<uintptr_t>(list[i].src) | reinterpret_cast<uintptr_t>(list[i].dst)) & 15u) == 0;
        p.first[k] = blocks;
        blocks += (uint32_t)((list[i].n + p.piece - 1) / p.piece);
    }
    return hipSuccess;
}

}  // namespace

int64_t grad_norm_partials(const sfb_tensor* list, int64_t count)
{
    const int64_t piece = piece_of(list, count);
    int64_t blocks = 0;
    for (int64_t i = 0; i < count; ++i) blocks += (list[i].n + piece - 1) / piece;
    return blocks;
}

hipError_t launch_grad_norm(const sfb_tensor* list, int64_t count, double* partial, float* norm, hipStream_t stream)
{
    const hipError_t e = for_list(list, count, [&](const ListParams& p, uint32_t blocks, int64_t done) {
        grad_norm_kernel<<<blocks, 256, 0, stream>>>(p, partial + done);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    grad_norm_final_kernel<<<1, 256, 0, stream>>>(partial, grad_norm_partials(list, count), norm);
    return hipGetLastError();
}

hipError_t launch_clip(const sfb_tensor* list, int64_t count, const double* partial, double max_norm, hipStream_t stream)
{
    const double* total = partial + grad_norm_partials(list, count);
    return for_list(list, count, [&](const ListParams& p, uint32_t blocks, int64_t) {
        clip_kernel<<<blocks, 256, 0, stream>>>(p, total, max_norm);
        return hipGetLastError();
    });
}

}  // namespace sfb
