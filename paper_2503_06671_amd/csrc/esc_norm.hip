// Layer norm over the channels of each pixel, forward and backward (esc_layernorm_* of include/esc_convattn.h).
//
//   u = (x - mean) r,  r = 1 / sqrt(mean of (x - mean)^2 + eps),  out = weight u + bias
//   a = weight g,  grad_x = r (a - mean(a) - u mean(a u)) + skip,  grad_weight = sum over pixels of g u,  grad_bias = sum over pixels of g
//
// What bounds it: memory.  x is read once and out written once; the backward pass reads x, g and skip once and writes grad_x.  That takes a pixel's
// channels out of registers: the mean first, then the squares of differences from it (no difference of large sums), then the result.  Planes of one
// channel are contiguous, so neighbouring lanes are neighbouring pixels, four at a time where there are enough, and the channels are
// spread over a wavefront's other lanes and over wavefronts.  One MI355X: 180 x 320 of 192 channels, bf16 10.4 us (44 MB, 4.2 TB/s; a kernel that
// reads x three times 48); 64 x 64 x 64 of 64 channels, bf16 forward 13.9 (4.8 TB/s), backward with skip 26.2 (5.1 TB/s; a copy of 1 GiB 5.1) and 4.6 for the
// parts of the weights' sums; 2 x 339 x 511 of 45, fp32 25.8 and 45; 64 x 64 of 64, fp32 4.4.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "esc_convattn.h"
#include "esc_host.hpp"
#include "esc_parts.hpp"

namespace {

using namespace esc;

constexpr size_t kAlign = 256;
constexpr int kThreads = 256;
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
    long first;          // of a launch's blocks
    float eps, inv_c;
};

template <typename E>
__device__ __forceinline__ float widen(E e)
{
    if constexpr (sizeof(E) == 4) return e;
    else return __uint_as_float((uint32_t)e << 16);
}
template <typename E>
__device__ __forceinline__ float value(const E *p) { return widen(*p); }
template <typename E>
__device__ __forceinline__ void put(E *p, float v)
{
    if constexpr (sizeof(E) == 4) *p = v;
    else *p = __builtin_bit_cast(uint16_t, (__bf16)v);
}

// ---- any number of channels: a block's 1024 threads are LANES pixels of 1024 / LANES groups of channels, and read x as often as they need it ----

constexpr int kAnyThreads = 1024, kAnyAhead = 8;  // (values under way at a time)

// The sums over the block's groups of channels of each pixel's values.
template <int LANES, int Q>
__device__ __forceinline__ void over_groups(float (&v)[Q], float (*s)[kAnyThreads / LANES][LANES])
{
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; ++q) s[q][group][lane] = v[q];
#pragma unroll
    for (int half = kAnyThreads / LANES / 2; half > 0; half /= 2) {
        __syncthreads();
        if (group < half) {
#pragma unroll
            for (int q = 0; q < Q; ++q) s[q][group][lane] += s[q][group + half][lane];
        }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; ++q) v[q] = s[q][0][lane];
}

// f(c, values of N tensors at channel c) for the channels group, group + GROUPS, ...: kAnyAhead of each are asked for at a time.
template <int GROUPS, int N, typename E, typename F>
__device__ __forceinline__ void over_rows(const E *const (&from)[N], int group, int C, long P, F f)
{
    for (int c0 = group; c0 < C; c0 += kAnyAhead * GROUPS) {
        E v[N][kAnyAhead];
#pragma unroll
        for (int u = 0; u < kAnyAhead; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i][u] = from[i][(long)min(c0 + u * GROUPS, C - 1) * P];
#pragma unroll
        for (int u = 0; u < kAnyAhead; ++u) {
            float w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = widen(v[i][u]);
            if (c0 + u * GROUPS < C) f(c0 + u * GROUPS, w);
        }
    }
}

template <typename E, int LANES>
__global__ __launch_bounds__(kAnyThreads) void norm_any_kernel(const NormParams p)
{
    constexpr int kGroups = kAnyThreads / LANES;
    __shared__ float s[1][kGroups][LANES];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const long tiles = (p.P + LANES - 1) / LANES, all = tiles * p.N;
    for (long tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const long n = tile / tiles, px = (tile - n * tiles) * LANES + lane, pc = px < p.P ? px : p.P - 1;
        const E *const x[1] = {static_cast<const E *>(p.x) + n * p.x_stride + pc};
        E *out = static_cast<E *>(p.out) + n * p.out_stride + pc;
        float sum[1] = {0.f};
        over_rows<kGroups>(x, group, p.C, p.P, [&](int, const float (&v)[1]) { sum[0] += v[0]; });
        over_groups<LANES>(sum, s);
        const float mean = sum[0] * p.inv_c;
        sum[0] = 0.f;
        over_rows<kGroups>(x, group, p.C, p.P, [&](int, const float (&v)[1]) { sum[0] += (v[0] - mean) * (v[0] - mean); });
        over_groups<LANES>(sum, s);
        const float r = 1.f / sqrtf(sum[0] * p.inv_c + p.eps);
        if (px < p.P) {
            over_rows<kGroups>(x, group, p.C, p.P, [&](int c, const float (&v)[1]) {
                put(out + c * p.P, ((v[0] - mean) * r) * (p.weight != nullptr ? p.weight[c] : 1.f) + (p.bias != nullptr ? p.bias[c] : 0.f));
            });
            if (p.mean != nullptr && group == 0) p.mean[n * p.P + px] = mean, p.rstd[n * p.P + px] = r;
        }
    }
}

template <typename E, int LANES>
__global__ __launch_bounds__(kAnyThreads) void norm_back_any_kernel(const NormParams p)
{
    constexpr int kGroups = kAnyThreads / LANES;
    __shared__ float s[2][kGroups][LANES];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const long tiles = (p.P + LANES - 1) / LANES, all = tiles * p.N;
    for (long tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const long n = tile / tiles, px = (tile - n * tiles) * LANES + lane, pc = px < p.P ? px : p.P - 1;
        const E *const xg[2] = {static_cast<const E *>(p.x) + n * p.x_stride + pc, static_cast<const E *>(p.grad_out) + n * p.out_stride + pc};
        const E *skip = p.skip != nullptr ? static_cast<const E *>(p.skip) + n * p.skip_stride + pc : nullptr;
        E *gx = static_cast<E *>(p.grad_x) + n * p.gx_stride + pc;
        const float mean = p.mean[n * p.P + pc], r = p.rstd[n * p.P + pc];
        float sum[2] = {0.f, 0.f};
        over_rows<kGroups>(xg, group, p.C, p.P, [&](int c, const float (&v)[2]) {
            const float a = v[1] * (p.weight != nullptr ? p.weight[c] : 1.f);
            sum[0] += a, sum[1] += a * ((v[0] - mean) * r);
        });
        over_groups<LANES>(sum, s);
        const float sa = sum[0] * p.inv_c, sau = sum[1] * p.inv_c;
        if (px >= p.P) continue;
        over_rows<kGroups>(xg, group, p.C, p.P, [&](int c, const float (&v)[2]) {
            const float a = v[1] * (p.weight != nullptr ? p.weight[c] : 1.f), u = (v[0] - mean) * r;
            const float o = r * (a - sa - u * sau);
            put(gx + c * p.P, skip != nullptr ? o + value(skip + c * p.P) : o);
        });
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

// ---- up to 1024 channels: a pixel's channels stay in registers ----
//
// A wavefront's lanes are sixteen times V pixels of four channels; KC such fours and WS wavefronts make up the channels of a tile of 16 V
// pixels, in steps of 4 WS channels.  x is read once, in rows of 16 V pixels, and sums over the channels cross four lanes and, for WS > 1, LDS.

constexpr int kWide = 4;   // V, where there are pixels enough

template <typename E, int V>
struct __attribute__((packed, aligned(sizeof(E)))) Pack {
    E e[V];
};
template <typename E, int V>
__device__ __forceinline__ Pack<E, V> load_pack(const E *p) { return *reinterpret_cast<const Pack<E, V> *>(p); }
template <typename E, int V>
__device__ __forceinline__ void store_pack(E *p, const float (&v)[V])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    Pack<E, V> r;
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < V; ++i) r.e[i] = v[i];
    } else if constexpr (V == 1) {
        r.e[0] = __builtin_bit_cast(uint16_t, (__bf16)v[0]);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const uint32_t two = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[i], v[i + 1]}, bf16x2));
            r.e[i] = (uint16_t)two, r.e[i + 1] = (uint16_t)(two >> 16);
        }
    }
    *reinterpret_cast<Pack<E, V> *>(p) = r;
}

// What is made of these values before is not kept for behind.
template <typename E, int V>
__device__ __forceinline__ void hold(Pack<E, V> &p)
{
    constexpr int kWords = (int)(sizeof(p) + 3) / 4;
    uint32_t w[kWords] = {};
    __builtin_memcpy(w, &p, sizeof(p));
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
    __builtin_memcpy(&p, w, sizeof(p));
}

// The sums over a tile's channels of each of its pixels' values: over a wavefront's four channels, then over WS wavefronts (through `s`, which the
// next call but one may use again).
template <int V, int WS, int Q>
__device__ __forceinline__ void over_channels(float (&v)[Q][V], float (*s)[Q][V][16], int share)
{
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[q][i] += __shfl_xor(v[q][i], 16);
            v[q][i] += __shfl_xor(v[q][i], 32);
        }
    if constexpr (WS > 1) {
        const int lane = threadIdx.x & 63;
        if (lane < 16) {
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int i = 0; i < V; ++i) s[share][q][i][lane] = v[q][i];
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < WS; ++w) t += s[w][q][i][lane & 15];
                v[q][i] = t;
            }
    }
}

template <int WS>
constexpr int kBlock = WS > 4 ? 64 * WS : 256;  // threads: one tile's wavefronts, or four wavefronts
template <int WS>
constexpr int kSets = kBlock<WS> / (64 * WS);   // tiles at a time

// Where a wavefront's lanes are: image, first pixel (the last V pixels instead of some beyond the image), first channel, and that element of an image
// (of the last channel where there is no such one).
struct Place {
    long n, first, want, origin;
    int channel;
    // is there a k-th channel of this lane, and how far it is from the first (0 if there is none)
    template <int WS>
    __device__ __forceinline__ bool has(int k, int C) const { return channel + 4 * WS * k < C; }
    template <int WS>
    __device__ __forceinline__ long row(int k, int C, long P) const { return has<WS>(k, C) ? 4 * WS * k * P : 0; }
};
template <int V, int WS>
__device__ __forceinline__ Place place(long tile, long tiles, long P, int C, int share)
{
    const int lane = threadIdx.x & 63;
    Place r;
    r.n = tile / tiles;
    r.want = (tile - r.n * tiles) * (16 * V) + V * (lane & 15);
    r.first = r.want + V <= P ? r.want : P - V;
    r.channel = (lane >> 4) + 4 * share;
    r.origin = (long)min(r.channel, C - 1) * P + r.first;
    return r;
}

template <typename E, int V, int KC, int WS>
__global__ __launch_bounds__(kBlock<WS>) void norm_kernel(const NormParams p)
{
    __shared__ float s[2][kSets<WS>][WS][1][V][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), set = wave / WS, share = wave % WS;
    const long tiles = (p.P + 16 * V - 1) / (16 * V), all = tiles * p.N;
    const long mine = (p.first + blockIdx.x) * kSets<WS> + set;
    const Place at = place<V, WS>(mine < all ? mine : all - 1, tiles, p.P, p.C, share);  // (a set beyond the last tile does that one again)
    const E *x = static_cast<const E *>(p.x) + at.n * p.x_stride + at.origin;
    E *out = static_cast<E *>(p.out) + at.n * p.out_stride + at.origin;
    Pack<E, V> raw[KC];
    float wv[KC], bv[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) raw[k] = load_pack<E, V>(x + at.row<WS>(k, p.C, p.P));
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        const int c = min(at.channel + 4 * WS * k, p.C - 1);
        wv[k] = p.weight != nullptr ? p.weight[c] : 1.f, bv[k] = p.bias != nullptr ? p.bias[c] : 0.f;
    }
    float mean[1][V], r[1][V], v[KC][V];
#pragma unroll
    for (int i = 0; i < V; ++i) mean[0][i] = r[0][i] = 0.f;
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[k][i] = widen(raw[k].e[i]);
            mean[0][i] += at.has<WS>(k, p.C) ? v[k][i] : 0.f;
        }
    over_channels<V, WS, 1>(mean, s[0][set], share);
#pragma unroll
    for (int i = 0; i < V; ++i) mean[0][i] *= p.inv_c;
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[k][i] -= mean[0][i];
            r[0][i] += at.has<WS>(k, p.C) ? v[k][i] * v[k][i] : 0.f;
        }
    over_channels<V, WS, 1>(r, s[1][set], share);
#pragma unroll
    for (int i = 0; i < V; ++i) r[0][i] = 1.f / sqrtf(r[0][i] * p.inv_c + p.eps);
    if (at.want >= p.P) return;
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        if (!at.has<WS>(k, p.C)) break;
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = (v[k][i] * r[0][i]) * wv[k] + bv[k];
        store_pack<E, V>(out + 4 * WS * k * p.P, o);
    }
    if (p.mean != nullptr && share == 0 && (threadIdx.x & 63) < 16) {
        store_pack<float, V>(p.mean + at.n * p.P + at.first, mean[0]);
        store_pack<float, V>(p.rstd + at.n * p.P + at.first, r[0]);
    }
}

// A block goes through tiles a grid apart, and keeps its channels' sums over the pixels in registers until the end.
template <typename E, int V, int KC, int WS>
__global__ __launch_bounds__(kBlock<WS>) void norm_back_kernel(const NormParams p)
{
    __shared__ float s[2][kSets<WS>][WS][2][V][16];
    __shared__ float sums[kSets<WS>][2][4 * WS * KC];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), set = wave / WS, share = wave % WS, lane = threadIdx.x & 63;
    const long tiles = (p.P + 16 * V - 1) / (16 * V), all = tiles * p.N;
    float wv[KC], gw[KC], gb[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        const int c = (lane >> 4) + 4 * share + 4 * WS * k;
        wv[k] = c < p.C ? p.weight != nullptr ? p.weight[c] : 1.f : 0.f;
        gw[k] = gb[k] = 0.f;
    }
    int turn = 0;
    for (long base = (long)blockIdx.x * kSets<WS>; base < all; base += (long)gridDim.x * kSets<WS>, turn ^= 1) {
        const bool there = base + set < all;
        const Place at = place<V, WS>(there ? base + set : all - 1, tiles, p.P, p.C, share);
        const E *x = static_cast<const E *>(p.x) + at.n * p.x_stride + at.origin, *g = static_cast<const E *>(p.grad_out) + at.n * p.out_stride + at.origin;
        Pack<E, V> xr[KC], gr[KC];
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            const long row = at.row<WS>(k, p.C, p.P);
            xr[k] = load_pack<E, V>(x + row), gr[k] = load_pack<E, V>(g + row);
        }
        const Pack<float, V> mean = load_pack<float, V>(p.mean + at.n * p.P + at.first), r = load_pack<float, V>(p.rstd + at.n * p.P + at.first);
        // a pixel counts once, where this lane was to begin with it
        float counts[V];
#pragma unroll
        for (int i = 0; i < V; ++i) counts[i] = there && at.want < p.P && at.first + i >= at.want ? 1.f : 0.f;
        float t[2][V];
#pragma unroll
        for (int i = 0; i < V; ++i) t[0][i] = t[1][i] = 0.f;
#pragma unroll
        for (int k = 0; k < KC; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool in = at.has<WS>(k, p.C);
                const float gv = in ? widen(gr[k].e[i]) : 0.f, u = (widen(xr[k].e[i]) - mean.e[i]) * r.e[i];
                const float gu = in ? gv * u : 0.f;
                t[0][i] += gv * wv[k], t[1][i] += gu * wv[k];
                gw[k] += counts[i] != 0.f ? gu : 0.f, gb[k] += counts[i] != 0.f ? gv : 0.f;
            }
        over_channels<V, WS, 2>(t, s[turn][set], share);
        // (kept through the sums as they were read, not as what was made of them: half the registers)
#pragma unroll
        for (int k = 0; k < KC; ++k) hold(xr[k]), hold(gr[k]);
        if (p.grad_x != nullptr && there && at.want < p.P) {
            E *gx = static_cast<E *>(p.grad_x) + at.n * p.gx_stride + at.origin;
            const E *skip = p.skip != nullptr ? static_cast<const E *>(p.skip) + at.n * p.skip_stride + at.origin : nullptr;
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                if (!at.has<WS>(k, p.C)) break;
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float u = (widen(xr[k].e[i]) - mean.e[i]) * r.e[i];
                    o[i] = r.e[i] * (widen(gr[k].e[i]) * wv[k] - t[0][i] * p.inv_c - u * (t[1][i] * p.inv_c));
                }
                if (skip != nullptr) {
                    const Pack<E, V> sk = load_pack<E, V>(skip + 4 * WS * k * p.P);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] += widen(sk.e[i]);
                }
                store_pack<E, V>(gx + 4 * WS * k * p.P, o);
            }
        }
    }
    if (p.part == nullptr) return;
    // over the sixteen lanes of a channel's pixels (to the last of them), then over the block's sets of wavefronts
    auto row_sum = [](float v) {
        auto moved = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
        v += moved(v, std::integral_constant<int, 0x111>{});
        v += moved(v, std::integral_constant<int, 0x112>{});
        v += moved(v, std::integral_constant<int, 0x114>{});
        return v + moved(v, std::integral_constant<int, 0x118>{});
    };
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        const float a = row_sum(gw[k]), b = row_sum(gb[k]);
        if ((lane & 15) == 15) {
            const int c = (lane >> 4) + 4 * share + 4 * WS * k;
            sums[set][0][c] = a, sums[set][1][c] = b;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.C; i += kBlock<WS>) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kSets<WS>; ++k) v += sums[k][i < p.C ? 0 : 1][i < p.C ? i : i - p.C];
        p.part[(size_t)blockIdx.x * 2 * p.C + i] = v;
    }
}

// KC and WS for up to 4 WS KC channels.  Few channels a lane leave registers for more wavefronts (backward, 64 x 64 x 64 x 64 bf16: KC 4, WS 4
// 26 us, KC 8, WS 2 33; forward KC 8, WS 2 13.8, KC 16, WS 1 17.3), few wavefronts a tile wait less for one another (forward, 180 x 320 of 192 channels: KC 12, WS 4
// 11.4 us, KC 6, WS 8 13.0), and few empty places are worth either (backward, 339 x 511 of 45 fp32: 48 places 45 us, 64 52).
struct Split {
    int kc, ws;
    constexpr int places() const { return 4 * ws * kc; }
};
constexpr Split kForward[] = {{4, 1}, {8, 1}, {6, 2}, {8, 2}, {6, 4}, {8, 4}, {12, 4}, {16, 4}, {12, 8}, {16, 8}, {12, 16}, {16, 16}};
constexpr Split kBackward[] = {{4, 1}, {4, 2}, {3, 4}, {4, 4}, {3, 8}, {4, 8}, {6, 8}, {8, 8}, {12, 8}, {16, 8}};
template <bool BACK>
constexpr const auto &splits()
{
    if constexpr (BACK) return kBackward;
    else return kForward;
}
template <bool BACK>
constexpr int kSplitCount = (int)(sizeof(splits<BACK>()) / sizeof(Split));

// The number of the split for C channels; the splits' count: more channels than registers hold.
template <bool BACK>
int split_of(int C)
{
    int i = 0;
    while (i < kSplitCount<BACK> && splits<BACK>()[i].places() < C) ++i;
    return i;
}
// pixels of a lane: fewer where sixteen wavefronts have 128 registers each, or a lane has many channels of two tensors
constexpr int wide_of(bool back, Split k) { return (back ? k.kc > 8 : k.ws == 16) ? kWide / 2 : kWide; }

template <typename E, bool BACK, int I = 0>
hipError_t launch_held(NormParams p, int split, int v, long grid, hipStream_t s)
{
    if constexpr (I < kSplitCount<BACK>) {
        if (split != I) return launch_held<E, BACK, I + 1>(p, split, v, grid, s);
        constexpr Split k = splits<BACK>()[I];
        const dim3 block(kBlock<k.ws>);
        constexpr int wide = wide_of(BACK, k);
        if constexpr (BACK) {
            if (v == 1) hipLaunchKernelGGL((norm_back_kernel<E, 1, k.kc, k.ws>), dim3((unsigned)grid), block, 0, s, p);
            else hipLaunchKernelGGL((norm_back_kernel<E, wide, k.kc, k.ws>), dim3((unsigned)grid), block, 0, s, p);
            return hipGetLastError();
        } else {
            return in_launches(grid, kBlock<k.ws>, [&](long first, unsigned blocks) {
                p.first = first;
                if (v == 1) hipLaunchKernelGGL((norm_kernel<E, 1, k.kc, k.ws>), dim3(blocks), block, 0, s, p);
                else hipLaunchKernelGGL((norm_kernel<E, wide, k.kc, k.ws>), dim3(blocks), block, 0, s, p);
                return hipGetLastError();
            });
        }
    } else {
        return hipErrorInvalidValue;
    }
}

// Pixels of a lane: one where more would leave compute units without a tile.
constexpr long kCus = 256;
long tiles_of(long N, long P, int v) { return N * ((P + 16 * v - 1) / (16 * v)); }
template <bool BACK>
int lanes_pixels(long N, long P, Split k)
{
    const int wide = wide_of(BACK, k);
    return P >= wide && tiles_of(N, P, wide) >= kCus ? wide : 1;
}
long sets_of(Split k) { return k.ws < 4 ? 4 / k.ws : 1; }

// Sixteen pixels of a block where 64 would leave compute units without a tile.
template <bool BACK>
hipError_t launch_any(const NormParams &p, bool f32, hipStream_t s)
{
    const long few = (p.P + 63) / 64 * p.N;
    const dim3 block(kAnyThreads), grid((unsigned)std::min<long>(few < kCus ? (p.P + 15) / 16 * p.N : few, 1 << 20));
    const auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, s, p);
        return hipGetLastError();
    };
    if constexpr (BACK) {
        if (few < kCus) return f32 ? launch(norm_back_any_kernel<float, 16>) : launch(norm_back_any_kernel<uint16_t, 16>);
        return f32 ? launch(norm_back_any_kernel<float, 64>) : launch(norm_back_any_kernel<uint16_t, 64>);
    } else {
        if (few < kCus) return f32 ? launch(norm_any_kernel<float, 16>) : launch(norm_any_kernel<uint16_t, 16>);
        return f32 ? launch(norm_any_kernel<float, 64>) : launch(norm_any_kernel<uint16_t, 64>);
    }
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
// Blocks of the backward pass, each with a part of the weights' sums: sixteen wavefronts a compute unit where there are tiles for them.
int splits_of(const esc_layernorm *a, long P)
{
    const int split = split_of<true>(a->C);
    if (split == kSplitCount<true>) return (int)std::min<long>(kMaxSplits, (P + kRun - 1) / kRun * a->N);
    const Split k = kBackward[split];
    return (int)std::min((tiles_of(a->N, P, lanes_pixels<true>(a->N, P, k)) + sets_of(k) - 1) / sets_of(k), kCus * 16 / std::max(4, k.ws));
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
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int split = split_of<false>(a->C);
    if (split < kSplitCount<false>) {
        const Split k = kForward[split];
        const int v = lanes_pixels<false>(a->N, P, k);
        const long blocks = (tiles_of(a->N, P, v) + sets_of(k) - 1) / sets_of(k);
        const hipError_t e = dt == ESC_F32 ? launch_held<float, false>(p, split, v, blocks, s) : launch_held<uint16_t, false>(p, split, v, blocks, s);
        return e == hipSuccess ? ESC_OK : ESC_ERR_HIP;
    }
    return launch_any<false>(p, dt == ESC_F32, s) == hipSuccess ? ESC_OK : ESC_ERR_HIP;
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
    const int split = split_of<true>(a->C);
    if (split < kSplitCount<true>) {
        if (!sums) p.part = nullptr;
        const int v = lanes_pixels<true>(a->N, P, kBackward[split]);
        const hipError_t e = dt == ESC_F32 ? launch_held<float, true>(p, split, v, p.splits, s) : launch_held<uint16_t, true>(p, split, v, p.splits, s);
        if (e != hipSuccess) return ESC_ERR_HIP;
        return !sums || add_parts(p.part, p.splits, a->C, g->weight, a->C, g->bias, accumulate, s) == hipSuccess ? ESC_OK : ESC_ERR_HIP;
    }
    if (g->x != nullptr) {
        if (launch_any<true>(p, dt == ESC_F32, s) != hipSuccess) return ESC_ERR_HIP;
    }
    if (sums) {
        const dim3 grid(a->C, p.splits);
        if (dt == ESC_F32) hipLaunchKernelGGL(norm_weights_any_kernel<float>, grid, block, 0, s, p);
        else hipLaunchKernelGGL(norm_weights_any_kernel<uint16_t>, grid, block, 0, s, p);
        if (hipGetLastError() != hipSuccess) return ESC_ERR_HIP;
        if (add_parts(p.part, p.splits, a->C, g->weight, a->C, g->bias, accumulate, s) != hipSuccess) return ESC_ERR_HIP;
    }
    return ESC_OK;
}

}  // extern "C"
