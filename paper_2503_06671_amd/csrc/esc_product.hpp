// What the point-wise product's kernels share (esc_product.hip: products of any size, weights' gradients, host side; esc_product_strip.hip: products
// whose input channels stay in registers).
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "esc_terms.hpp"

namespace esc {

struct ProductParams {
    const void *x;         // K planes an image
    const void *extra;     // M planes an image: the residual, or grad_out, or nullptr
    void *out;             // M planes an image
    long x_stride, extra_stride, out_stride;  // elements
    const float *w, *b;
    int K, M, w_ld, act;
    long P, pixels;        // of an image, of all
    long tiles;            // of an image (or of all, where tiles pass images' borders)
    bool across;           // tiles pass images' borders
};

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr long kCus = 256;

struct bf16s {
    uint16_t bits;
};
template <typename T>
constexpr bool kWide = sizeof(T) == 4;

__device__ __forceinline__ uint32_t pack2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2)); }

// N terms of two values, a word of two for each: three are exact, by truncation; two, and one, are the nearest.
template <int N>
__device__ __forceinline__ void terms_of(float a, float b, uint32_t (&t)[N])
{
    if constexpr (N == 3) {
        split_bf16(a, b, t);
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            t[q] = pack2(a, b);
            if (q + 1 < N) a -= __uint_as_float(t[q] << 16), b -= __uint_as_float(t[q] & 0xffff0000u);
        }
    }
}

// Behind the last product: an ordinary instruction may read a product's result twelve issue slots later.
__device__ __forceinline__ void settle()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15");
    __builtin_amdgcn_sched_barrier(0);
}

template <typename T>
__device__ __forceinline__ float widen(T v)
{
    if constexpr (kWide<T>) return v;
    else return __uint_as_float((uint32_t)v.bits << 16);
}
// Two neighbours at any address their type allows.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Two {
    T a, b;
};

enum : int { kNone = 0, kGelu = 1, kSilu = 2 };

// e = erfc(|v| / sqrt 2) as 2^-(t P(t)), t = |v| (esc_gelu.hpp has the polynomial's derivation)
__device__ __forceinline__ float erfc_of(float t)
{
    float q = fmaf(2.834909764715121e-06f, t, -3.937766086892225e-05f);
    q = fmaf(q, t, 0.0001861801283666864f);
    q = fmaf(q, t, 0.0001369366073049605f);
    q = fmaf(q, t, -0.0070634204894304276f);
    q = fmaf(q, t, 0.052496179938316345f);
    q = fmaf(q, t, 0.4592081904411316f);
    q = fmaf(q, t, 1.1511051654815674f);
    return __builtin_amdgcn_exp2f(-q * t);
}
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504f)); }

__device__ __forceinline__ float activation(int act, float v)
{
    if (act == kGelu) {
        const float h = 0.5f * v;
        return fmaf(fabsf(h), 1.f - erfc_of(fabsf(v)), h);
    }
    return act == kSilu ? v * sigmoid(v) : v;
}
__device__ __forceinline__ float slope(int act, float v)
{
    if (act == kGelu) {
        // Phi(v) + v phi(v)
        const float e = 0.5f * erfc_of(fabsf(v));
        return fmaf(v * 0.3989422804f, __builtin_amdgcn_exp2f(v * v * -0.7213475204f), v >= 0.f ? 1.f - e : e);
    }
    if (act == kSilu) {
        const float s = sigmoid(v);
        return s * fmaf(v, 1.f - s, 1.f);
    }
    return 1.f;
}

// What the kernels' sums become: act(v) for all of them, the choice made once for a wavefront.
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N])
{
    if (act == kGelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activation(kGelu, v[i]);
    } else if (act == kSilu) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activation(kSilu, v[i]);
    }
}
template <int N>
__device__ __forceinline__ void slopes(int act, float (&v)[N])
{
    if (act == kGelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = slope(kGelu, v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = slope(kSilu, v[i]);
    }
}
// kForward: out = act(pre) + extra.  kSlope: out = extra act'(pre), fp32.
enum : int { kForward = 0, kSlope = 1 };

// Which eighths of the grid the dies get: consecutive pieces on one die.
__device__ __forceinline__ unsigned piece_of(unsigned block, unsigned blocks)
{
    const unsigned each = blocks / 8u, rest = blocks % 8u, die = block % 8u;
    return die * each + (die < rest ? die : rest) + block / 8u;
}

}  // namespace

// The products there are: forward; gp = grad_out act'(pre), fp32; grad_x = W^T g, of g in the storage type or of gp held in fp32 with bf16 storage.
enum : int { kForwardF32, kForwardBf16, kSlopeF32, kSlopeBf16, kBackF32, kBackBf16, kBackGp };

// Whether esc_product_strip.hip takes a product.
__attribute__((visibility("hidden"))) bool strip_fits(int kind, const ProductParams &p, long N);
__attribute__((visibility("hidden"))) hipError_t launch_strip(int kind, const ProductParams &p, long N, hipStream_t s);

}  // namespace esc
