// Layer norm over the channels of each pixel, forward and backward (esc_layernorm_* of include/esc_convattn.h).
//
//   u = (x - mean) r,  r = 1 / sqrt(mean of (x - mean)^2 + eps),  out = weight u + bias
//   a = weight g,  grad_x = r (a - mean(a) - u mean(a u)) + skip,  grad_weight = sum over pixels of g u,  grad_bias = sum over pixels of g
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "esc_convattn.h"
#include "esc_host.hpp"

namespace {

using namespace esc;

constexpr size_t kAlign = 256;
constexpr int kThreads = 256;
constexpr int kLanes = 64, kGroups = kThreads / kLanes;  // of a block: pixels, and groups of channels
constexpr int kMaxSplits = 64;
constexpr int kRun = 1024;  // pixels that a block of the weights' sums takes at a time

struct NormParams {
    const void *x, *grad_out, *skip;
    void *out, *grad_x;
    long x_stride, out_stride, skip_stride, gx_stride;
    const float *weight, *bias;
    float *mean, *rstd;  // [N P] each, or nullptr
    float *part;         // [splits][2][C]
    int N, C, splits;
    long P;
    float eps, inv_c;
};

template <typename E>
__device__ __forceinline__ float value(const E *p)
{
    if constexpr (sizeof(E) == 4) return *p;
    else return __uint_as_float((uint32_t)*p << 16);
}
template <typename E>
__device__ __forceinline__ void put(E *p, float v)
{
    if constexpr (sizeof(E) == 4) *p = v;
    else *p = __builtin_bit_cast(uint16_t, (__bf16)v);
}

// The sum over the block's groups of channels of each pixel's value.
__device__ __forceinline__ float over_groups(float v, float (&s)[kGroups][kLanes])
{
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 6;
    __syncthreads();
    s[group][lane] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) t += s[g][lane];
    return t;
}

// Any number of channels: x is read three times.
template <typename E>
__global__ __launch_bounds__(kThreads) void norm_any_kernel(const NormParams p)
{
    __shared__ float s[kGroups][kLanes];
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 6;
    const long tiles = (p.P + kLanes - 1) / kLanes, all = tiles * p.N;
    for (long tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const long n = tile / tiles, px = (tile - n * tiles) * kLanes + lane, pc = px < p.P ? px : p.P - 1;
        const E *x = static_cast<const E *>(p.x) + n * p.x_stride + pc;
        E *out = static_cast<E *>(p.out) + n * p.out_stride + pc;
        float sum = 0.f;
        for (int c = group; c < p.C; c += kGroups) sum += value(x + c * p.P);
        const float mean = over_groups(sum, s) * p.inv_c;
        sum = 0.f;
        for (int c = group; c < p.C; c += kGroups) {
            const float d = value(x + c * p.P) - mean;
            sum += d * d;
        }
        const float r = 1.f / sqrtf(over_groups(sum, s) * p.inv_c + p.eps);
        if (px < p.P) {
            for (int c = group; c < p.C; c += kGroups) {
                const float u = (value(x + c * p.P) - mean) * r;
                put(out + c * p.P, p.weight != nullptr ? u * p.weight[c] + (p.bias != nullptr ? p.bias[c] : 0.f) : p.bias != nullptr ? u + p.bias[c] : u);
            }
            if (p.mean != nullptr && group == 0) p.mean[n * p.P + px] = mean, p.rstd[n * p.P + px] = r;
        }
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void norm_back_any_kernel(const NormParams p)
{
    __shared__ float s[kGroups][kLanes];
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 6;
    const long tiles = (p.P + kLanes - 1) / kLanes, all = tiles * p.N;
    for (long tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const long n = tile / tiles, px = (tile - n * tiles) * kLanes + lane, pc = px < p.P ? px : p.P - 1;
        const E *x = static_cast<const E *>(p.x) + n * p.x_stride + pc, *g = static_cast<const E *>(p.grad_out) + n * p.out_stride + pc;
        const E *skip = p.skip != nullptr ? static_cast<const E *>(p.skip) + n * p.skip_stride + pc : nullptr;
        E *gx = static_cast<E *>(p.grad_x) + n * p.gx_stride + pc;
        const float mean = p.mean[n * p.P + pc], r = p.rstd[n * p.P + pc];
        float sa = 0.f, sau = 0.f;
        for (int c = group; c < p.C; c += kGroups) {
            const float a = value(g + c * p.P) * (p.weight != nullptr ? p.weight[c] : 1.f), u = (value(x + c * p.P) - mean) * r;
            sa += a, sau += a * u;
        }
        sa = over_groups(sa, s) * p.inv_c, sau = over_groups(sau, s) * p.inv_c;
        if (px >= p.P) continue;
        for (int c = group; c < p.C; c += kGroups) {
            const float a = value(g + c * p.P) * (p.weight != nullptr ? p.weight[c] : 1.f), u = (value(x + c * p.P) - mean) * r;
            const float v = r * (a - sa - u * sau);
            put(gx + c * p.P, skip != nullptr ? v + value(skip + c * p.P) : v);
        }
    }
}

// One channel's sums over a part of the pixels.
template <typename E>
__global__ __launch_bounds__(kThreads) void norm_weights_any_kernel(const NormParams p)
{
    __shared__ float s[2][kThreads];
    const int c = blockIdx.x;
    const long runs = (p.P + kRun - 1) / kRun, all = runs * p.N;
    float sw = 0.f, sb = 0.f;
    for (long run = blockIdx.y; run < all; run += gridDim.y) {
        const long n = run / runs, first = (run - n * runs) * kRun, end = first + kRun < p.P ? first + kRun : p.P;
        const E *x = static_cast<const E *>(p.x) + n * p.x_stride + c * p.P, *g = static_cast<const E *>(p.grad_out) + n * p.out_stride + c * p.P;
        for (long px = first + threadIdx.x; px < end; px += kThreads) {
            const float gv = value(g + px);
            sb += gv, sw += gv * ((value(x + px) - p.mean[n * p.P + px]) * p.rstd[n * p.P + px]);
        }
    }
    s[0][threadIdx.x] = sw, s[1][threadIdx.x] = sb;
    for (int half = kThreads / 2; half > 0; half /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < half) s[0][threadIdx.x] += s[0][threadIdx.x + half], s[1][threadIdx.x] += s[1][threadIdx.x + half];
    }
    if (threadIdx.x == 0) {
        p.part[((size_t)blockIdx.y * 2 + 0) * p.C + c] = s[0][0];
        p.part[((size_t)blockIdx.y * 2 + 1) * p.C + c] = s[1][0];
    }
}

// Adds the parts up, in the order of their numbers.
__global__ __launch_bounds__(kThreads) void norm_parts_kernel(const float *part, int splits, int C, float *weight, float *bias, int accumulate)
{
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= 2 * C) return;
    float t = 0.f;
    for (int k = 0; k < splits; ++k) t += part[(size_t)k * 2 * C + i];
    float *to = i < C ? weight : bias;
    if (to == nullptr) return;
    to += i < C ? i : i - C;
    *to = accumulate ? *to + t : t;
}

esc_status shape(const esc_layernorm *a, long *P)
{
    if (a == nullptr) return ESC_ERR_NULL;
    if (a->N < 1 || a->C < 1 || a->H < 1 || a->W < 1) return ESC_ERR_SHAPE;
    *P = (long)a->H * a->W;
    if (a->C > 65536 || *P >= (1L << 31) || (double)*P * a->N >= 0x1p40) return ESC_ERR_UNSUPPORTED;
    return ESC_OK;
}

size_t saved_size(const esc_layernorm *a, long P) { return round_up((size_t)a->N * P * 8, kAlign); }
int splits_of(const esc_layernorm *a, long P)
{
    return (int)std::min<long>(kMaxSplits, (P + kRun - 1) / kRun * a->N);
}
size_t workspace_size(const esc_layernorm *a, long P) { return round_up((size_t)splits_of(a, P) * 2 * a->C * 4, kAlign); }

}  // namespace

extern "C" {

size_t esc_layernorm_saved_bytes(const esc_layernorm *a)
{
    long P;
    return shape(a, &P) == ESC_OK ? saved_size(a, P) : 0;
}

size_t esc_layernorm_backward_workspace_bytes(const esc_layernorm *a)
{
    long P;
    return shape(a, &P) == ESC_OK ? workspace_size(a, P) : 0;
}

esc_status esc_layernorm_forward(const void *x, esc_dtype dt, const esc_layernorm *a, void *out, void *saved, size_t saved_bytes, void *stream)
{
    long P;
    if (dt != ESC_F32 && dt != ESC_BF16) return ESC_ERR_DTYPE;
    const esc_status st = shape(a, &P);
    if (st != ESC_OK) return st;
    if (x == nullptr || out == nullptr) return ESC_ERR_NULL;
    if (!(a->eps > 0.f) || !isfinite(a->eps)) return ESC_ERR_SHAPE;
    const size_t es = dt == ESC_F32 ? 4 : 2, image = (size_t)a->C * P, vec = (size_t)a->C * 4, sv = saved_size(a, P);
    Images xi, oi;
    if (!images_of(x, a->x_stride, a->N, image, es, &xi) || !images_of(out, a->out_stride, a->N, image, es, &oi)) return ESC_ERR_SHAPE;
    if (((uintptr_t)a->weight | (uintptr_t)a->bias) % 4 != 0) return ESC_ERR_SHAPE;
    if (saved != nullptr && ((uintptr_t)saved % kAlign != 0 || saved_bytes < sv)) return ESC_ERR_WORKSPACE;
    if (meet(oi, xi) || meets(oi, a->weight, vec) || meets(oi, a->bias, vec) || meets(oi, saved, sv) || meets(xi, saved, sv)) return ESC_ERR_ALIAS;
    if (saved != nullptr && ((a->weight != nullptr && overlaps(saved, sv, a->weight, vec)) || (a->bias != nullptr && overlaps(saved, sv, a->bias, vec)))) return ESC_ERR_ALIAS;
    NormParams p{};
    p.x = x, p.out = out, p.x_stride = (long)(xi.stride / es), p.out_stride = (long)(oi.stride / es);
    p.weight = a->weight, p.bias = a->bias, p.N = a->N, p.C = a->C, p.P = P, p.eps = a->eps, p.inv_c = 1.f / (float)a->C;
    if (saved != nullptr) p.mean = static_cast<float *>(saved), p.rstd = p.mean + (size_t)a->N * P;
    const dim3 grid((unsigned)std::min<long>((P + kLanes - 1) / kLanes * a->N, 1 << 20)), block(kThreads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dt == ESC_F32) hipLaunchKernelGGL(norm_any_kernel<float>, grid, block, 0, s, p);
    else hipLaunchKernelGGL(norm_any_kernel<uint16_t>, grid, block, 0, s, p);
    return hipGetLastError() == hipSuccess ? ESC_OK : ESC_ERR_HIP;
}

esc_status esc_layernorm_backward(const void *x, const void *grad_out, const void *grad_skip, esc_dtype dt, const esc_layernorm *a, const void *saved,
                                  size_t saved_bytes, const esc_layernorm_grads *g, int accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    long P;
    if (dt != ESC_F32 && dt != ESC_BF16) return ESC_ERR_DTYPE;
    const esc_status st = shape(a, &P);
    if (st != ESC_OK) return st;
    if (x == nullptr || grad_out == nullptr || saved == nullptr || g == nullptr) return ESC_ERR_NULL;
    if (g->x == nullptr && g->weight == nullptr && g->bias == nullptr) return ESC_ERR_NULL;
    const size_t es = dt == ESC_F32 ? 4 : 2, image = (size_t)a->C * P, vec = (size_t)a->C * 4, sv = saved_size(a, P), wb = workspace_size(a, P);
    Images xi, gi, si{}, gxi{};
    if (!images_of(x, a->x_stride, a->N, image, es, &xi) || !images_of(grad_out, a->out_stride, a->N, image, es, &gi)) return ESC_ERR_SHAPE;
    if (grad_skip != nullptr && !images_of(grad_skip, a->skip_stride, a->N, image, es, &si)) return ESC_ERR_SHAPE;
    if (g->x != nullptr && !images_of(g->x, g->x_stride, a->N, image, es, &gxi)) return ESC_ERR_SHAPE;
    if (((uintptr_t)a->weight | (uintptr_t)g->weight | (uintptr_t)g->bias) % 4 != 0) return ESC_ERR_SHAPE;
    if ((uintptr_t)saved % kAlign != 0 || saved_bytes < sv) return ESC_ERR_WORKSPACE;
    const bool sums = g->weight != nullptr || g->bias != nullptr;
    if (workspace == nullptr || (uintptr_t)workspace % kAlign != 0 || workspace_bytes < wb) return ESC_ERR_WORKSPACE;
    // what is written overlaps nothing else
    struct Flat {
        const void *at;
        size_t bytes;
        bool written;
    } const flat[] = {{a->weight, vec, false}, {saved, sv, false}, {g->weight, vec, true}, {g->bias, vec, true}, {workspace, wb, true}};
    const Images *const read[] = {&xi, &gi, &si};
    for (const Images *r : read)
        if (g->x != nullptr && r->at != nullptr && meet(gxi, *r)) return ESC_ERR_ALIAS;
    for (size_t i = 0; i < sizeof(flat) / sizeof(flat[0]); ++i) {
        if (flat[i].at == nullptr) continue;
        if (g->x != nullptr && meets(gxi, flat[i].at, flat[i].bytes)) return ESC_ERR_ALIAS;
        if (!flat[i].written) continue;
        for (const Images *r : read)
            if (r->at != nullptr && meets(*r, flat[i].at, flat[i].bytes)) return ESC_ERR_ALIAS;
        for (size_t j = 0; j < sizeof(flat) / sizeof(flat[0]); ++j)
            if (j != i && flat[j].at != nullptr && overlaps(flat[i].at, flat[i].bytes, flat[j].at, flat[j].bytes)) return ESC_ERR_ALIAS;
    }
    NormParams p{};
    p.x = x, p.grad_out = grad_out, p.skip = grad_skip, p.grad_x = g->x;
    p.x_stride = (long)(xi.stride / es), p.out_stride = (long)(gi.stride / es), p.skip_stride = (long)(si.stride / es), p.gx_stride = (long)(gxi.stride / es);
    p.weight = a->weight, p.N = a->N, p.C = a->C, p.P = P, p.inv_c = 1.f / (float)a->C;
    p.mean = const_cast<float *>(static_cast<const float *>(saved)), p.rstd = p.mean + (size_t)a->N * P;
    p.part = static_cast<float *>(workspace), p.splits = splits_of(a, P);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 block(kThreads);
    if (g->x != nullptr) {
        const dim3 grid((unsigned)std::min<long>((P + kLanes - 1) / kLanes * a->N, 1 << 20));
        if (dt == ESC_F32) hipLaunchKernelGGL(norm_back_any_kernel<float>, grid, block, 0, s, p);
        else hipLaunchKernelGGL(norm_back_any_kernel<uint16_t>, grid, block, 0, s, p);
        if (hipGetLastError() != hipSuccess) return ESC_ERR_HIP;
    }
    if (sums) {
        const dim3 grid(a->C, p.splits);
        if (dt == ESC_F32) hipLaunchKernelGGL(norm_weights_any_kernel<float>, grid, block, 0, s, p);
        else hipLaunchKernelGGL(norm_weights_any_kernel<uint16_t>, grid, block, 0, s, p);
        if (hipGetLastError() != hipSuccess) return ESC_ERR_HIP;
        hipLaunchKernelGGL(norm_parts_kernel, dim3((2 * a->C + kThreads - 1) / kThreads), block, 0, s, p.part, p.splits, a->C, g->weight, g->bias, accumulate);
        if (hipGetLastError() != hipSuccess) return ESC_ERR_HIP;
    }
    return ESC_OK;
}

}  // extern "C"
