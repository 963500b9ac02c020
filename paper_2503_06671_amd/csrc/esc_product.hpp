// What the point-wise product's kernels share (esc_product.hip: products of any size, weights' gradients, host side; esc_product_strip.hip: products
// whose input channels stay in registers).
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "esc_gelu.hpp"
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
    long tiles;            // of pixels, of an image (or of all, where they pass images' borders)
    unsigned first;        // a launch's first block
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
enum : int { kNone = 0, kGelu = 1, kSilu = 2 };

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504f)); }

__device__ __forceinline__ float activation(int act, float v)
{
    if (act == kGelu) return ffn_gelu(v);
    return act == kSilu ? v * sigmoid(v) : v;
}
__device__ __forceinline__ float slope(int act, float v)
{
    if (act == kGelu) {
        // Phi(v) + v phi(v)
        const float e = 0.5f * erfc_root2(fabsf(v));
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
// kForward: out = act(pre).  kResidual: out = act(pre) + extra.  kSlope: out = extra act'(pre), fp32.
enum : int { kForward = 0, kSlope = 1, kResidual = 2 };

// ---- accesses to an image's planes by 32-bit offsets ----

typedef __amdgpu_buffer_rsrc_t Rsrc;
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kRawBuffer = 0x00020000;     // raw buffer (no stride, no swizzle), 32-bit data format
constexpr unsigned kBeyond = 0x80000000u;  // an offset beyond every resource (an image of a tensor is < 2 GiB)
constexpr int kSchedNoVmem = 0x38f;        // a scheduling barrier for accesses to memory alone
constexpr int kSchedNoVmemNoMfma = 0x386;  // a scheduling barrier for accesses to memory and matrix instructions
constexpr size_t kMostImage = (size_t)1 << 31;
constexpr long kMostPlane = 1L << 24;      // pixels: 31 planes' offset beside kBeyond does not pass 32 bits

__device__ __forceinline__ Rsrc resource(const void *at, long bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, (int)bytes, kRawBuffer);
}

// NT neighbouring elements of a lane, as words.
template <typename T, int NT>
struct Raw {
    static constexpr int kWords = NT * (int)sizeof(T) == 8 ? 2 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ float value(int t) const
    {
        if constexpr (kWide<T>) return __uint_as_float(w[t]);
        else return __uint_as_float(t == 0 ? w[0] << 16 : w[0] & 0xffff0000u);
    }
};
template <typename T, int NT>
__device__ __forceinline__ Raw<T, NT> load(Rsrc r, unsigned voff, unsigned soff)
{
    Raw<T, NT> v;
    if constexpr (Raw<T, NT>::kWords == 2) {
        const u32x2 two = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)voff, (int)soff, 0));
        v.w[0] = two.x, v.w[1] = two.y;
    } else if constexpr (NT * sizeof(T) == 4) {
        v.w[0] = (unsigned)__builtin_amdgcn_raw_buffer_load_b32(r, (int)voff, (int)soff, 0);
    } else {
        v.w[0] = (unsigned)__builtin_amdgcn_raw_buffer_load_b16(r, (int)voff, (int)soff, 0);
    }
    return v;
}
template <typename T, int NT>
__device__ __forceinline__ void store(Rsrc r, unsigned voff, unsigned soff, float a, float b)
{
    if constexpr (NT * sizeof(T) == 8) {
        typedef decltype(__builtin_amdgcn_raw_buffer_load_b64(r, 0, 0, 0)) B64;
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(B64, u32x2{__float_as_uint(a), __float_as_uint(b)}), r, (int)voff, (int)soff, 0);
    } else if constexpr (kWide<T>) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(a), r, (int)voff, (int)soff, 0);
    } else if constexpr (NT == 2) {
        __builtin_amdgcn_raw_buffer_store_b32(pack2(a, b), r, (int)voff, (int)soff, 0);
    } else {
        __builtin_amdgcn_raw_buffer_store_b16((unsigned short)pack2(a, a), r, (int)voff, (int)soff, 0);
    }
}

// N matrix instructions, with ordinary ones between them: a wavefront's next instruction waits for the matrix unit only if it is one for it.
template <int N>
__device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
    }
}

// ---- weights: runs of four channels of one output, zeros beyond K and M ----

// Four weights of output m from channel k on.  `four`: K is a multiple of four, a run is inside or outside as a whole.
__device__ __forceinline__ void load_weights(Rsrc rw, int M, int K, int ld, bool four, int m, int k, float (&w)[4])
{
    if (four) {
        const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(m < M && k < K ? 4u * ((unsigned)m * (unsigned)ld + (unsigned)k) : kBeyond), 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __uint_as_float(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = __uint_as_float((unsigned)__builtin_amdgcn_raw_buffer_load_b32(rw, (int)(m < M && k + e < K ? 4u * ((unsigned)m * (unsigned)ld + (unsigned)(k + e)) : kBeyond), 0, 0));
    }
}
// The same where w's rows are the channels.  K0 of k is the wavefront's, the rest a lane's.
__device__ __forceinline__ void load_weights_across(Rsrc rw, int M, int K, int ld, int m, int k0, int k1, float (&w)[4])
{
    const unsigned at = m < M ? 4u * ((unsigned)k1 * (unsigned)ld + (unsigned)m) : kBeyond;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        w[e] = __uint_as_float((unsigned)__builtin_amdgcn_raw_buffer_load_b32(rw, (int)(k0 + k1 + e < K ? at : kBeyond), (int)(k0 + e < K ? 4u * ((unsigned)(k0 + e) * (unsigned)ld) : 0u), 0));
}

// Which eighths of a launch the dies get: consecutive pieces on one die.
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

// grad_x of a product with an activation, gp on the way: gp = grad_out act'(b + w x), fp32, kept where gp is not nullptr, and grad_x = W^T gp.
struct BackParams {
    const void *x, *grad_out;
    float *gp;
    void *grad_x;
    long x_stride, g_stride, gp_stride, gx_stride;  // elements
    const float *w, *b;
    int K, M, act;
    long P;
    unsigned tiles_of_image;
    unsigned first;        // a launch's first block
};
__attribute__((visibility("hidden"))) bool back_fits(bool f32, int K, int M, long P, long N);
__attribute__((visibility("hidden"))) hipError_t launch_back(bool f32, const BackParams &p, long N, hipStream_t s);

}  // namespace esc
