// Sums over blocks' parts, in a fixed order (esc_norm.hip, esc_product.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace esc {
namespace {

// to[i] (+)= sum over k < splits of part[k][i], i < n.  32 neighbouring results a block, 32 threads for each (8 and 128 where results are few): a thread
// adds every 32nd part up, eight under way at a time, then the threads' sums are added in halves.  (One thread a result, 512 parts of 8192 results: 120 us.)
constexpr int kPartsThreads = 1024;

struct PartsParams {
    const float *part;
    float *to[2];     // results below n0 go to the first, the others to the second (either may be nullptr)
    long n, n0;
    int splits, accumulate;
};

template <int kPartsColumns>
__global__ __launch_bounds__(kPartsThreads) void parts_kernel(const PartsParams p)
{
    constexpr int kRows = kPartsThreads / kPartsColumns;
    __shared__ float s[kRows][kPartsColumns + 1];
    const int column = threadIdx.x % kPartsColumns, row = threadIdx.x / kPartsColumns;
    const long i = (long)blockIdx.x * kPartsColumns + column, at = i < p.n ? i : p.n - 1;
    float t = 0.f;
    int k = row;
    for (; k + 7 * kRows < p.splits; k += 8 * kRows) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = p.part[(long)(k + j * kRows) * p.n + at];
#pragma unroll
        for (int j = 0; j < 8; ++j) t += v[j];
    }
    for (; k < p.splits; k += kRows) t += p.part[(long)k * p.n + at];
    s[row][column] = t;
#pragma unroll
    for (int half = kRows / 2; half > 0; half /= 2) {
        __syncthreads();
        if (row < half) s[row][column] += s[row + half][column];
    }
    if (row != 0 || i >= p.n) return;
    float *to = i < p.n0 ? p.to[0] : p.to[1];
    if (to == nullptr) return;
    to += i < p.n0 ? i : i - p.n0;
    const float v = s[0][column];
    *to = p.accumulate ? *to + v : v;
}

// Few parts: a thread a result.
__global__ __launch_bounds__(256) void few_parts_kernel(const PartsParams p)
{
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.n) return;
    float t = 0.f;
    for (int k = 0; k < p.splits; ++k) t += p.part[(long)k * p.n + i];
    float *to = i < p.n0 ? p.to[0] : p.to[1];
    if (to == nullptr) return;
    to += i < p.n0 ? i : i - p.n0;
    *to = p.accumulate ? *to + t : t;
}

inline hipError_t add_parts(const float *part, int splits, long n0, float *to0, long n1, float *to1, int accumulate, hipStream_t s)
{
    const PartsParams p{part, {to0, to1}, n0 + n1, n0, splits, accumulate};
    if (splits <= 16) hipLaunchKernelGGL(few_parts_kernel, dim3((unsigned)((p.n + 255) / 256)), dim3(256), 0, s, p);
    else if (p.n <= 2048) hipLaunchKernelGGL(parts_kernel<8>, dim3((unsigned)((p.n + 7) / 8)), dim3(kPartsThreads), 0, s, p);
    else hipLaunchKernelGGL(parts_kernel<32>, dim3((unsigned)((p.n + 31) / 32)), dim3(kPartsThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace
}  // namespace esc
