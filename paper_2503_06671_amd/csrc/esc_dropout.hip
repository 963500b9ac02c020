// Dropout with the residual added, its mask drawn from a counter-based generator (esc_dropout_* of include/esc_convattn.h).
//
//   out[i] = residual[i] + ( draw(unit(i)) >= q ? x[i] * 65536 / (65536 - q) : 0 )
//
// draw(u) is a 16-bit part of block u / 8 of Philox4x32 with ten rounds: eight draws a block, so that a thread that takes eight
// consecutive elements runs the generator once (some 110 instructions for eight elements, a quarter of what the vector units could do in the time).  Whole planes
// and images are spans of blocks of their own: one draw a block, and what is dropped is not read.
//
// What bounds it: memory.  One MI355X, 64 x 64 x 64 of 64 channels, bf16: elements with residual 16.8 us (101 MB, 6.0 TB/s: part of it from the last-level
// cache), the gradient 12.7; 4 x 64 x 64 of 192, fp32, whole images 6.6.  (Loads of eight elements behind conditions, which the compiler took apart: 23.7,
// 16.7 and 8.6.)
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "esc_convattn.h"
#include "esc_host.hpp"

namespace {

using namespace esc;

constexpr int kThreads = 256;
constexpr int kChunk = 8;      // elements of a block of draws, and of a thread's access
constexpr int kUnroll = 2;     // chunks a thread has under way
constexpr int kPart = kThreads * kUnroll;
constexpr long kSmallPlane = 512;  // planes below this many elements are not spans of their own

enum : int { kPerElement = 0, kPerSpan = 1, kPerPlane = 2 };

struct DropParams {
    const void *x, *residual;
    void *out;
    long x_stride, residual_stride, out_stride;  // elements from image to image
    const long long *offset_device;
    uint64_t seed, offset;
    long spans, span;     // how many runs of elements, and how long they are
    long spans_of_image;  // (an image is so many)
    long units_of_span;   // per plane: planes of an image
    long parts;           // blocks' pieces of a span
    uint32_t q, plane;
    float scale;
};

struct Words {
    uint32_t w[4];
};

// Ten rounds on the counter (n, offset) with the key `seed`.
__device__ __forceinline__ Words philox(uint64_t n, uint64_t offset, uint64_t seed)
{
    uint32_t x0 = (uint32_t)n, x1 = (uint32_t)(n >> 32), x2 = (uint32_t)offset, x3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
        x0 = (uint32_t)(b >> 32) ^ x1 ^ k0, x1 = (uint32_t)b;
        x2 = (uint32_t)(a >> 32) ^ x3 ^ k1, x3 = (uint32_t)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return Words{{x0, x1, x2, x3}};
}
__device__ __forceinline__ uint32_t draw_of(const Words &w, int j) { return (j & 1) ? w.w[j >> 1] >> 16 : w.w[j >> 1] & 0xffffu; }
// (for an index that is not known at compile time)
__device__ __forceinline__ uint32_t draw_at(const Words &w, uint32_t j)
{
    const uint32_t lo = (j & 2) ? w.w[1] : w.w[0], hi = (j & 2) ? w.w[3] : w.w[2], v = (j & 4) ? hi : lo;
    return (j & 1) ? v >> 16 : v & 0xffffu;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

typedef u32x4 Loose4 __attribute__((aligned(4)));
typedef u32x4 Loose2 __attribute__((aligned(2)));

// Eight neighbouring elements at any address their type allows: all of them (WHOLE), or those from `first` to `last`.
template <typename E>
struct Eight {
    static constexpr int kWords = kChunk * (int)sizeof(E) / 16;
    typedef typename std::conditional<sizeof(E) == 4, Loose4, Loose2>::type Loose;
    u32x4 w[kWords];
    template <bool WHOLE>
    __device__ __forceinline__ void load(const E *p, int first, int last)
    {
        if constexpr (WHOLE) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const Loose *>(p)[i];
        } else {
            E e[kChunk];
#pragma unroll
            for (int j = 0; j < kChunk; ++j) e[j] = j >= first && j < last ? p[j] : E(0);
            __builtin_memcpy(w, e, sizeof(w));
        }
    }
    template <bool WHOLE>
    __device__ __forceinline__ void store(E *p, int first, int last) const
    {
        if constexpr (WHOLE) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) reinterpret_cast<Loose *>(p)[i] = w[i];
        } else {
            E e[kChunk];
            __builtin_memcpy(e, w, sizeof(w));
#pragma unroll
            for (int j = 0; j < kChunk; ++j)
                if (j >= first && j < last) p[j] = e[j];
        }
    }
    __device__ __forceinline__ float value(int j) const
    {
        if constexpr (sizeof(E) == 4) return __uint_as_float(w[j >> 2][j & 3]);
        else return __uint_as_float((j & 1) ? w[0][j >> 1] & 0xffff0000u : w[0][j >> 1] << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[kChunk])
    {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            if constexpr (sizeof(E) == 4) w[j >> 2][j & 3] = __float_as_uint(v[j]);
            else if ((j & 1) == 0) w[0][j >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[j], v[j + 1]}, bf16x2));
        }
    }
};

// A block's part of a span: kUnroll chunks a thread.  WHOLE: all of them lie in the span.
template <typename E, int KIND, bool RES, bool WHOLE>
__device__ __forceinline__ void part_of_span(const DropParams &p, uint64_t offset, long span, long part, const E *x, const E *res, E *out, int shift)
{
    const long base = span * p.span / kChunk;
    bool all = true;
    if constexpr (KIND == kPerSpan) {
        if (p.q != 0) all = draw_at(philox((uint64_t)span >> 3, offset, p.seed), (uint32_t)span & 7) >= p.q;
    }
    Eight<E> v[kUnroll], r[kUnroll];
    int first[kUnroll], last[kUnroll];
    long at[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        at[u] = (part * kPart + u * kThreads + (long)threadIdx.x) * kChunk - shift;
        first[u] = at[u] < 0 ? (int)-at[u] : 0;
        last[u] = (int)(at[u] >= p.span ? 0 : p.span - at[u] < kChunk ? p.span - at[u] : kChunk);
        if (!WHOLE && last[u] <= 0) continue;
        if (KIND != kPerSpan || all) v[u].template load<WHOLE>(x + at[u], first[u], last[u]);
        if constexpr (RES) r[u].template load<WHOLE>(res + at[u], first[u], last[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        if (!WHOLE && last[u] <= 0) continue;
        bool keep[kChunk];
        if constexpr (KIND == kPerElement) {
            const Words w = philox((uint64_t)(base + (at[u] + shift) / kChunk), offset, p.seed);
#pragma unroll
            for (int j = 0; j < kChunk; ++j) keep[j] = draw_of(w, j) >= p.q;
        } else if constexpr (KIND == kPerSpan) {
#pragma unroll
            for (int j = 0; j < kChunk; ++j) keep[j] = all;
        } else {
            // (a span is an image of fewer than 2^31 elements)
            uint64_t held = ~(uint64_t)0;
            Words w{};
            uint32_t plane = (uint32_t)at[u] / p.plane, left = p.plane - ((uint32_t)at[u] - plane * p.plane);
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
                const uint64_t unit = (uint64_t)span * (uint64_t)p.units_of_span + plane;
                if (unit >> 3 != held) held = unit >> 3, w = philox(held, offset, p.seed);
                keep[j] = draw_at(w, (uint32_t)unit & 7) >= p.q;
                if (--left == 0) ++plane, left = p.plane;
            }
        }
        float o[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            o[j] = keep[j] ? v[u].value(j) * p.scale : 0.f;
            if constexpr (RES) o[j] = o[j] + r[u].value(j);
        }
        Eight<E> to;
        to.set(o);
        to.template store<WHOLE>(out + at[u], first[u], last[u]);
    }
}

template <typename E, int KIND, bool RES>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const DropParams p)
{
    const uint64_t offset = p.offset + (p.offset_device != nullptr ? (uint64_t)*p.offset_device : 0);
    const long blocks = p.spans * p.parts;
    for (long block = blockIdx.x; block < blocks; block += gridDim.x) {
        const long span = block / p.parts, part = block - span * p.parts;
        const long image = span / p.spans_of_image, inside = (span - image * p.spans_of_image) * p.span;
        const E *x = static_cast<const E *>(p.x) + image * p.x_stride + inside;
        const E *res = RES ? static_cast<const E *>(p.residual) + image * p.residual_stride + inside : nullptr;
        E *out = static_cast<E *>(p.out) + image * p.out_stride + inside;
        // chunks begin at multiples of eight of the elements' numbers where these are the draws' too
        const int shift = KIND == kPerElement ? (int)(span * p.span & (kChunk - 1)) : 0;
        const long begin = part * kPart * kChunk - shift;
        if (begin >= 0 && begin + kPart * kChunk <= p.span) part_of_span<E, KIND, RES, true>(p, offset, span, part, x, res, out, shift);
        else part_of_span<E, KIND, RES, false>(p, offset, span, part, x, res, out, shift);
    }
}

template <typename E, bool RES>
hipError_t launch(const DropParams &p, int kind, hipStream_t s)
{
    const dim3 grid((unsigned)std::min<long>(p.spans * p.parts, 1 << 20)), block(kThreads);
    if (kind == kPerElement) hipLaunchKernelGGL((dropout_kernel<E, kPerElement, RES>), grid, block, 0, s, p);
    else if (kind == kPerSpan) hipLaunchKernelGGL((dropout_kernel<E, kPerSpan, RES>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((dropout_kernel<E, kPerPlane, RES>), grid, block, 0, s, p);
    return hipGetLastError();
}

// From `in` (and the residual) to `out`, whose strides are given.
esc_status dropout(const void *in, long in_stride, const void *residual, long residual_stride, void *out, long out_stride, esc_dtype dt, const esc_dropout *a,
                   void *stream)
{
    if (a == nullptr) return ESC_ERR_NULL;
    if (dt != ESC_F32 && dt != ESC_BF16) return ESC_ERR_DTYPE;
    if (a->N < 1 || a->C < 1 || a->H < 1 || a->W < 1) return ESC_ERR_SHAPE;
    if (a->over != ESC_DROPOUT_ELEMENT && a->over != ESC_DROPOUT_PLANE && a->over != ESC_DROPOUT_IMAGE) return ESC_ERR_SHAPE;
    if (!(a->p >= 0.0 && a->p < 1.0)) return ESC_ERR_SHAPE;
    const long plane = (long)a->H * a->W;
    if (plane >= (1L << 31)) return ESC_ERR_UNSUPPORTED;
    if ((double)a->N * (double)a->C * (double)plane >= 0x1p48) return ESC_ERR_UNSUPPORTED;
    const uint32_t q = (uint32_t)floor(a->p * 65536.0 + 0.5);
    if (q > 65535) return ESC_ERR_UNSUPPORTED;
    if (in == nullptr || out == nullptr) return ESC_ERR_NULL;
    const size_t es = dt == ESC_F32 ? 4 : 2;
    const long image = (long)a->C * plane;
    Images xi, ri, oi;
    if (!images_of(in, in_stride, a->N, image, es, &xi) || !images_of(out, out_stride, a->N, image, es, &oi)) return ESC_ERR_SHAPE;
    if (residual != nullptr && !images_of(residual, residual_stride, a->N, image, es, &ri)) return ESC_ERR_SHAPE;
    if ((uintptr_t)a->offset_device % 8 != 0) return ESC_ERR_SHAPE;
    if (meet(oi, xi) || (residual != nullptr && meet(oi, ri)) || meets(oi, a->offset_device, 8)) return ESC_ERR_ALIAS;
    DropParams p{};
    p.x = in, p.residual = residual, p.out = out;
    p.x_stride = (long)(xi.stride / es), p.out_stride = (long)(oi.stride / es), p.residual_stride = residual != nullptr ? (long)(ri.stride / es) : 0;
    p.offset_device = a->offset_device, p.seed = a->seed, p.offset = a->offset;
    p.q = q, p.scale = (float)(65536.0 / (65536.0 - (double)q)), p.plane = (uint32_t)plane;
    int kind;
    if (a->over == ESC_DROPOUT_ELEMENT) {
        const bool flat = a->N == 1 || (p.x_stride == image && p.out_stride == image && (residual == nullptr || p.residual_stride == image));
        kind = kPerElement, p.spans = flat ? 1 : a->N, p.span = flat ? a->N * image : image, p.spans_of_image = 1;
    } else if (a->over == ESC_DROPOUT_IMAGE) {
        kind = kPerSpan, p.spans = a->N, p.span = image, p.spans_of_image = 1;
    } else if (plane >= kSmallPlane || image >= (1L << 31)) {
        kind = kPerSpan, p.spans = (long)a->N * a->C, p.span = plane, p.spans_of_image = a->C;
    } else {
        kind = kPerPlane, p.spans = a->N, p.span = image, p.spans_of_image = 1, p.units_of_span = a->C;
    }
    // (a chunk more than the elements fill: a span need not begin where a chunk does)
    p.parts = ((p.span + kChunk - 1) / kChunk + 1 + kPart - 1) / kPart;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (dt == ESC_F32) e = residual != nullptr ? launch<float, true>(p, kind, s) : launch<float, false>(p, kind, s);
    else e = residual != nullptr ? launch<uint16_t, true>(p, kind, s) : launch<uint16_t, false>(p, kind, s);
    return e == hipSuccess ? ESC_OK : ESC_ERR_HIP;
}

}  // namespace

extern "C" {

esc_status esc_dropout_forward(const void *x, const void *residual, esc_dtype dt, const esc_dropout *a, void *out, void *stream)
{
    return a == nullptr ? ESC_ERR_NULL : dropout(x, a->x_stride, residual, a->residual_stride, out, a->out_stride, dt, a, stream);
}

esc_status esc_dropout_backward(const void *grad_out, esc_dtype dt, const esc_dropout *a, void *grad_x, void *stream)
{
    return a == nullptr ? ESC_ERR_NULL : dropout(grad_out, a->out_stride, nullptr, 0, grad_x, a->x_stride, dt, a, stream);
}

}  // extern "C"
