// Point-wise products of any width with bias, activation and residual in their epilogue, and their gradients
// (esc_pointwise_* of include/esc_convattn.h).
//
//   forward    out[m, q] = act(b[m] + sum_k w[m, k] x[k, q]) + residual[m, q]          q: the pixels of all images
//   backward   pre = b + w x, gp = grad_out act'(pre);  grad_x[k, q] = sum_m w[m, k] gp[m, q];  grad_w[m, k] = sum_q gp[m, q] x[k, q];
//              grad_b[m] = sum_q gp[m, q]
//
// All are matrix products on v_mfma_f32_32x32x16_bf16 of terms of the values: an fp32 value is three bf16 terms (its top eight
// mantissa bits, the next eight, the rest: exact), a product of two such values the six products of terms whose orders add up to
// two at most (the rest lies below 2^-21 of it).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "esc_convattn.h"
#include "esc_host.hpp"
#include "esc_parts.hpp"
#include "esc_product.hpp"

namespace {

using namespace esc;

constexpr size_t kAlign = 256;
// ---- out = act(w x + b) + residual, and the products of the same form in the backward pass ----

// A block's tile is 32 MT WM outputs x 64 WP pixels; a wavefront has 32 MT outputs of 64 pixels.  Two neighbouring pixels are a
// lane's in two column blocks: columns of even pixels, then those of odd ones.  Operands lie in LDS as units of eight
// consecutive channels (k) of one pixel or output, a unit 16 bytes, [term][k / 8][place].
template <typename TI, typename TO, typename TE, int TX, int TW, int MT, int WM, int WP, bool TRANS, int MODE>
struct Product {
    static constexpr int kTop = TX > TW ? TX : TW;               // products of terms whose orders add up to less
    static constexpr int kStage = TX == 3 ? 16 : 32;             // channels of a stage
    static constexpr int kEights = kStage / 8;
    static constexpr int BM = 32 * MT * WM, BP = 64 * WP;
    static constexpr int kHalf = BP / 2 + 4;                     // places from even to odd pixels (four: other banks)
    static constexpr int kXPitch = BP / 2 + kHalf;
    static constexpr int kWPitch = BM + (TRANS ? 0 : 8 / kEights);
    static constexpr int kXUnits = TX * kEights * kXPitch, kWUnits = TW * kEights * kWPitch;
    static constexpr int kBuffer = kXUnits + kWUnits;
    static constexpr int kAt = kWide<TI> ? 1 : 2;                // pixels of a load
    static constexpr int kXLoads = kEights * BP / kAt, kXEach = (kXLoads + kThreads - 1) / kThreads;
    static constexpr int kWLoads = kEights * BM, kWEach = (kWLoads + kThreads - 1) / kThreads;
    static constexpr size_t kLds = (size_t)2 * kBuffer * 16 + BM * 4;
};

extern __shared__ __align__(16) u32x4 product_lds[];

template <typename TI, typename TO, typename TE, int TX, int TW, int MT, int WM, int WP, bool TRANS, int MODE>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(const ProductParams p)
{
    using C = Product<TI, TO, TE, TX, TW, MT, WM, WP, TRANS, MODE>;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, wm = wave % WM, wp = wave / WM;
    const int K = p.K, M = p.M, stages = (K + C::kStage - 1) / C::kStage;
    const long P = p.P;
    const unsigned groups = (unsigned)(M + C::BM - 1) / C::BM;
    const unsigned piece = piece_of(blockIdx.x, gridDim.x), tile = piece / groups;
    const int m0 = (int)(piece - tile * groups) * C::BM;
    const long image = p.across ? 0 : tile / p.tiles;
    const long q0 = ((long)tile - image * p.tiles) * C::BP;   // the tile's first pixel, of its image or of all

    // where pixel q0 + i is: its image and its place there.  What lies beyond the last pixel is the last pair again, computed and stored
    // with the same bits, or, in tiles that pass images' borders, the last pixel, not stored.
    auto place = [&](int i, long &n, long &at) {
        if (p.across) {
            const long q = min(q0 + i, p.pixels - 1);
            n = q / P, at = q - n * P;
        } else {
            n = image, at = min(q0 + (i & ~1), P - 2) + (i & 1);
        }
    };

    // ---- this thread's share of a stage's loads: eight channels of kAt pixels, eight weights of a row ----
    const TI *xp[C::kXEach][C::kAt];
    int xk[C::kXEach], xto[C::kXEach];
#pragma unroll
    for (int i = 0; i < C::kXEach; ++i) {
        const int u = tid + i * kThreads, unit = u % (C::BP / C::kAt);
        xk[i] = __builtin_amdgcn_readfirstlane(u / (C::BP / C::kAt));
        const int px = unit * C::kAt;
#pragma unroll
        for (int j = 0; j < C::kAt; ++j) {
            long n, at;
            place(px + j, n, at);
            xp[i][j] = static_cast<const TI *>(p.x) + n * p.x_stride + at;
        }
        xto[i] = xk[i] * C::kXPitch + (px >> 1) + (px & 1) * C::kHalf;
    }
    TI xr[C::kXEach][C::kAt][8];
    float wr[C::kWEach][8];
    auto fetch = [&](int st) {
#pragma unroll
        for (int i = 0; i < C::kXEach; ++i) {
            if (C::kXLoads % kThreads != 0 && xk[i] >= C::kEights) continue;
            const int k0 = st * C::kStage + 8 * xk[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const long row = (long)min(k0 + e, K - 1) * P;
                if constexpr (C::kAt == 2) {
                    if (p.across) {
                        xr[i][0][e] = xp[i][0][row], xr[i][1][e] = xp[i][1][row];
                    } else {
                        const Two<TI> t = *reinterpret_cast<const Two<TI> *>(xp[i][0] + row);
                        xr[i][0][e] = t.a, xr[i][1][e] = t.b;
                    }
                } else {
                    xr[i][0][e] = xp[i][0][row];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < C::kWEach; ++i) {
            const int u = tid + i * kThreads;
            const int k8 = TRANS ? u / C::BM : u % C::kEights, row = TRANS ? u % C::BM : u / C::kEights;
            const int m = m0 + row, k = st * C::kStage + 8 * k8;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                wr[i][e] = (m < M && k + e < K && k8 < C::kEights && row < C::BM) ? (TRANS ? p.w[(size_t)(k + e) * p.w_ld + m] : p.w[(size_t)m * p.w_ld + k + e]) : 0.f;
        }
    };
    auto put = [&](int st) {
        u32x4 *xs = product_lds + (st & 1) * C::kBuffer, *ws = xs + C::kXUnits;
#pragma unroll
        for (int i = 0; i < C::kXEach; ++i) {
            if (C::kXLoads % kThreads != 0 && xk[i] >= C::kEights) continue;
            const int in = K - (st * C::kStage + 8 * xk[i]);   // how many of the eight there are
#pragma unroll
            for (int j = 0; j < C::kAt; ++j) {
                uint32_t t[4][TX];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    terms_of<TX>(2 * e < in ? widen(xr[i][j][2 * e]) : 0.f, 2 * e + 1 < in ? widen(xr[i][j][2 * e + 1]) : 0.f, t[e]);
#pragma unroll
                for (int q = 0; q < TX; ++q) xs[q * C::kEights * C::kXPitch + xto[i] + j * C::kHalf] = u32x4{t[0][q], t[1][q], t[2][q], t[3][q]};
            }
        }
#pragma unroll
        for (int i = 0; i < C::kWEach; ++i) {
            const int u = tid + i * kThreads;
            const int k8 = TRANS ? u / C::BM : u % C::kEights, row = TRANS ? u % C::BM : u / C::kEights;
            if (C::kWLoads % kThreads != 0 && u >= C::kWLoads) continue;
            uint32_t t[4][TW];
#pragma unroll
            for (int e = 0; e < 4; ++e) terms_of<TW>(wr[i][2 * e], wr[i][2 * e + 1], t[e]);
#pragma unroll
            for (int q = 0; q < TW; ++q) ws[(q * C::kEights + k8) * C::kWPitch + row] = u32x4{t[0][q], t[1][q], t[2][q], t[3][q]};
        }
    };

    float *bias = reinterpret_cast<float *>(product_lds + 2 * C::kBuffer);
    if (tid < C::BM) bias[tid] = p.b != nullptr && m0 + tid < M ? p.b[m0 + tid] : 0.f;
    static_assert(C::BM <= kThreads, "a thread for each output's bias");

    f32x16 acc[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[mt][t][i] = 0.f;

    fetch(0);
    put(0);
    __syncthreads();
    for (int st = 0; st < stages; ++st) {
        if (st + 1 < stages) fetch(st + 1);
        const u32x4 *xs = product_lds + (st & 1) * C::kBuffer, *ws = xs + C::kXUnits;
#pragma unroll
        for (int c = 0; c < C::kEights / 2; ++c) {
            u32x4 a[MT][TW], b[2][TX];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int q = 0; q < TX; ++q) b[t][q] = xs[(q * C::kEights + 2 * c + half) * C::kXPitch + t * C::kHalf + 32 * wp + l32];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int q = 0; q < TW; ++q) a[mt][q] = ws[(q * C::kEights + 2 * c + half) * C::kWPitch + 32 * (MT * wm + mt) + l32];
            // small terms first; neighbouring instructions on different sums
#pragma unroll
            for (int qw = TW - 1; qw >= 0; --qw)
#pragma unroll
                for (int qx = TX - 1; qx >= 0; --qx) {
                    if (qw + qx >= C::kTop) continue;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            acc[mt][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[mt][qw]), __builtin_bit_cast(bf16x8, b[t][qx]),
                                                                                 acc[mt][t], 0, 0, 0);
                }
        }
        if (st + 1 < stages) put(st + 1);
        __syncthreads();
    }
    settle();

    // ---- lane l has outputs m0 + 32 (MT wm + mt) + 8 (i / 4) + 4 half + i % 4 of the pixels of places l32 of its two column blocks ----
    const int px = 64 * wp + 2 * l32;
    long n0, n1, at0, at1;
    place(px, n0, at0);
    place(px + 1, n1, at1);
    const bool in0 = !p.across || q0 + px < p.pixels, in1 = !p.across || q0 + px + 1 < p.pixels;
    TO *o0 = static_cast<TO *>(p.out) + n0 * p.out_stride + at0, *o1 = static_cast<TO *>(p.out) + n1 * p.out_stride + at1;
    const TE *e0 = static_cast<const TE *>(p.extra) + n0 * p.extra_stride + at0, *e1 = static_cast<const TE *>(p.extra) + n1 * p.extra_stride + at1;
    auto finish = [&](float v, float e) {
        if constexpr (MODE == kSlope) return e * slope(p.act, v);
        else return p.extra != nullptr ? activation(p.act, v) + e : activation(p.act, v);
    };
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = 32 * (MT * wm + mt) + 8 * (i >> 2) + 4 * half + (i & 3), m = m0 + row;
            const float v0 = acc[mt][0][i] + bias[row], v1 = acc[mt][1][i] + bias[row];
            if (m >= M) continue;
            const long off = (long)m * P;
            if (p.across) {
                if (in0) {
                    const float r = finish(v0, p.extra != nullptr ? widen(e0[off]) : 0.f);
                    if constexpr (kWide<TO>) o0[off] = r;
                    else o0[off].bits = (uint16_t)pack2(r, r);
                }
                if (in1) {
                    const float r = finish(v1, p.extra != nullptr ? widen(e1[off]) : 0.f);
                    if constexpr (kWide<TO>) o1[off] = r;
                    else o1[off].bits = (uint16_t)pack2(r, r);
                }
            } else {
                float x0 = 0.f, x1 = 0.f;
                if (p.extra != nullptr) {
                    const Two<TE> e = *reinterpret_cast<const Two<TE> *>(e0 + off);
                    x0 = widen(e.a), x1 = widen(e.b);
                }
                const float r0 = finish(v0, x0), r1 = finish(v1, x1);
                Two<TO> r;
                if constexpr (kWide<TO>) {
                    r.a = r0, r.b = r1;
                } else {
                    const uint32_t two = pack2(r0, r1);
                    r.a.bits = (uint16_t)two, r.b.bits = (uint16_t)(two >> 16);
                }
                *reinterpret_cast<Two<TO> *>(o0 + off) = r;
            }
        }
}

template <typename TI, typename TO, typename TE, int TX, int TW, int MT, int WM, int WP, bool TRANS, int MODE>
hipError_t launch_product_as(ProductParams p, long N, hipStream_t s)
{
    using C = Product<TI, TO, TE, TX, TW, MT, WM, WP, TRANS, MODE>;
    const long groups = (p.M + C::BM - 1) / C::BM, apart = N * ((p.P + C::BP - 1) / C::BP), together = (p.pixels + C::BP - 1) / C::BP;
    // small images share tiles (single pixels have no pair to load at once)
    p.across = N > 1 ? p.P < 2 || 4 * together < 3 * apart : p.P < 2;
    p.tiles = p.across ? together : apart / N;
    const long grid = (p.across ? together : apart) * groups;
    if (grid >= (1L << 31)) return hipErrorInvalidValue;
    const auto kernel = product_kernel<TI, TO, TE, TX, TW, MT, WM, WP, TRANS, MODE>;
    if (C::kLds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), C::kLds, s, p);
    return hipGetLastError();
}

template <typename TI, typename TO, typename TE, int TX, int TW, bool TRANS, int MODE>
hipError_t launch_product(const ProductParams &p, long N, hipStream_t s)
{
    if (p.M > 64) return launch_product_as<TI, TO, TE, TX, TW, 2, 2, 2, TRANS, MODE>(p, N, s);
    return launch_product_as<TI, TO, TE, TX, TW, 2, 1, 4, TRANS, MODE>(p, N, s);
}

hipError_t launch_any(int kind, const ProductParams &p, long N, hipStream_t s)
{
    if (strip_fits(kind, p, N)) return launch_strip(kind, p, N, s);
    switch (kind) {
    case kForwardF32: return launch_product<float, float, float, 3, 3, false, kForward>(p, N, s);
    case kForwardBf16: return launch_product<bf16s, bf16s, bf16s, 1, 2, false, kForward>(p, N, s);
    case kSlopeF32: return launch_product<float, float, float, 3, 3, false, kSlope>(p, N, s);
    // (weights in three terms with bf16 storage too: what is left of them goes into every pixel's gradient)
    case kSlopeBf16: return launch_product<bf16s, float, bf16s, 1, 3, false, kSlope>(p, N, s);
    case kBackF32: return launch_product<float, float, float, 3, 3, true, kForward>(p, N, s);
    case kBackBf16: return launch_product<bf16s, bf16s, bf16s, 1, 2, true, kForward>(p, N, s);
    case kBackGp: return launch_product<float, bf16s, bf16s, 2, 2, true, kForward>(p, N, s);
    default: return hipErrorInvalidValue;
    }
}

// ---- grad_w[m, k] = sum over pixels of g[m, q] x[k, q], grad_b[m] = sum over pixels of g[m, q] ----

constexpr int kSide = 64;     // of a block's tile of grad_w; a wavefront has 32 x 32
constexpr int kPixels = 32;   // of a stage

struct WeightParams {
    const void *g, *x;
    long g_stride, x_stride;
    float *part, *part_b;     // [splits][M][K], [splits][M], or nullptr
    int K, M, splits;
    long P, pixels;
};

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight {
    T e[8];
};

template <typename TG, typename TI, int QG, int QX>
__global__ __launch_bounds__(kThreads, 2) void product_weights_kernel(const WeightParams p)
{
    constexpr int kTop = QG > QX ? QG : QX, kPitch = kSide + 2, kEights = kPixels / 8;
    __shared__ u32x4 s[2][(QG + QX) * kEights * kPitch];
    __shared__ float s_b[kThreads];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, wm = wave & 1, wk = wave >> 1;
    const int across = (p.K + kSide - 1) / kSide;
    const int m0 = (int)blockIdx.x / across * kSide, k0 = (int)blockIdx.x % across * kSide;
    const long stages = (p.pixels + kPixels - 1) / kPixels;
    const long first = stages * blockIdx.y / p.splits, end = stages * (blockIdx.y + 1) / p.splits;
    const int row = tid >> 2, e8 = tid & 3;  // this thread's unit of both operands: eight pixels of a row
    const int gm = min(m0 + row, p.M - 1), xk = min(k0 + row, p.K - 1);
    TG gr[8];
    TI xr[8];
    int in = 0;
    auto fetch = [&](long st) {
        const long q = st * kPixels, n = q / p.P, at = q - n * p.P;
        if (at + kPixels <= p.P) {  // (the same for the block)
            const Eight<TG> a = *reinterpret_cast<const Eight<TG> *>(static_cast<const TG *>(p.g) + n * p.g_stride + gm * p.P + at + 8 * e8);
            const Eight<TI> b = *reinterpret_cast<const Eight<TI> *>(static_cast<const TI *>(p.x) + n * p.x_stride + xk * p.P + at + 8 * e8);
#pragma unroll
            for (int j = 0; j < 8; ++j) gr[j] = a.e[j], xr[j] = b.e[j];
            in = 8;
        } else {
            const long mine = q + 8 * e8;
            in = (int)(p.pixels - mine < 0 ? 0 : p.pixels - mine < 8 ? p.pixels - mine : 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const long one = min(mine + j, p.pixels - 1), i = one / p.P, a = one - i * p.P;
                gr[j] = static_cast<const TG *>(p.g)[i * p.g_stride + gm * p.P + a];
                xr[j] = static_cast<const TI *>(p.x)[i * p.x_stride + xk * p.P + a];
            }
        }
    };
    float sum_b = 0.f;
    auto put = [&](int buffer) {
        uint32_t t[4][QG], u[4][QX];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a0 = 2 * j < in ? widen(gr[2 * j]) : 0.f, a1 = 2 * j + 1 < in ? widen(gr[2 * j + 1]) : 0.f;
            const float b0 = 2 * j < in ? widen(xr[2 * j]) : 0.f, b1 = 2 * j + 1 < in ? widen(xr[2 * j + 1]) : 0.f;
            sum_b += a0 + a1;
            terms_of<QG>(a0, a1, t[j]);
            terms_of<QX>(b0, b1, u[j]);
        }
#pragma unroll
        for (int q = 0; q < QG; ++q) s[buffer][(q * kEights + e8) * kPitch + row] = u32x4{t[0][q], t[1][q], t[2][q], t[3][q]};
#pragma unroll
        for (int q = 0; q < QX; ++q) s[buffer][((QG + q) * kEights + e8) * kPitch + row] = u32x4{u[0][q], u[1][q], u[2][q], u[3][q]};
    };
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    if (first < end) {
        fetch(first);
        put(0);
    }
    __syncthreads();
    for (long st = first; st < end; ++st) {
        const int buffer = (int)(st - first) & 1;
        if (st + 1 < end) fetch(st + 1);
#pragma unroll
        for (int c = 0; c < kEights / 2; ++c) {
            u32x4 a[QG], b[QX];
#pragma unroll
            for (int q = 0; q < QG; ++q) a[q] = s[buffer][(q * kEights + 2 * c + half) * kPitch + 32 * wm + l32];
#pragma unroll
            for (int q = 0; q < QX; ++q) b[q] = s[buffer][((QG + q) * kEights + 2 * c + half) * kPitch + 32 * wk + l32];
#pragma unroll
            for (int i = QG - 1; i >= 0; --i)
#pragma unroll
                for (int j = QX - 1; j >= 0; --j)
                    if (i + j < kTop)
                        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, b[j]), acc, 0, 0, 0);
        }
        if (st + 1 < end) put(buffer ^ 1);
        __syncthreads();
    }
    settle();
    if (p.part != nullptr) {
        const int k = k0 + 32 * wk + l32;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int m = m0 + 32 * wm + 8 * (i >> 2) + 4 * half + (i & 3);
            const float v = acc[i];
            if (m < p.M && k < p.K) p.part[((size_t)blockIdx.y * p.M + m) * p.K + k] = v;
        }
    }
    if (p.part_b != nullptr && k0 == 0) {
        s_b[tid] = sum_b;
        __syncthreads();
        if (tid < kSide && m0 + tid < p.M) p.part_b[(size_t)blockIdx.y * p.M + m0 + tid] = (s_b[4 * tid] + s_b[4 * tid + 1]) + (s_b[4 * tid + 2] + s_b[4 * tid + 3]);
    }
}

template <typename TG, typename TI, int QG, int QX>
hipError_t launch_weights(const WeightParams &p, hipStream_t s)
{
    const unsigned tiles = (unsigned)(((p.M + kSide - 1) / kSide) * ((p.K + kSide - 1) / kSide));
    hipLaunchKernelGGL((product_weights_kernel<TG, TI, QG, QX>), dim3(tiles, p.splits), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

// ---- host side ----

esc_status shape(const esc_pointwise *a, long *P)
{
    if (a == nullptr) return ESC_ERR_NULL;
    if (a->N < 1 || a->K < 1 || a->M < 1 || a->H < 1 || a->W < 1) return ESC_ERR_SHAPE;
    if (a->act != ESC_ACT_NONE && a->act != ESC_ACT_GELU && a->act != ESC_ACT_SILU) return ESC_ERR_SHAPE;
    *P = (long)a->H * a->W;
    if (a->K > 65536 || a->M > 65536 || *P >= (1L << 31) || (double)*P * a->N >= 0x1p40) return ESC_ERR_UNSUPPORTED;
    return ESC_OK;
}

// blocks for the whole card a few times over, 16 stages each at least
int splits_of(const esc_pointwise *a, long P)
{
    const long tiles = (long)((a->M + kSide - 1) / kSide) * ((a->K + kSide - 1) / kSide), stages = ((long)a->N * P + kPixels - 1) / kPixels;
    return (int)std::max<long>(1, std::min((4 * kCus + tiles - 1) / tiles, stages / 16));
}

struct Scratch {
    size_t gp, part, part_b, total;
};
Scratch scratch(const esc_pointwise *a, long P)
{
    Scratch s;
    const size_t splits = (size_t)splits_of(a, P);
    s.gp = 0;
    s.part = a->act != ESC_ACT_NONE ? round_up((size_t)a->N * P * a->M * 4, kAlign) : 0;
    s.part_b = s.part + round_up(splits * a->M * a->K * 4, kAlign);
    s.total = s.part_b + round_up(splits * a->M * 4, kAlign);
    return s;
}

}  // namespace

extern "C" {

size_t esc_pointwise_backward_workspace_bytes(const esc_pointwise *a, esc_dtype dt)
{
    long P;
    return (dt == ESC_F32 || dt == ESC_BF16) && shape(a, &P) == ESC_OK ? scratch(a, P).total : 0;
}

esc_status esc_pointwise_forward(const void *x, const void *residual, esc_dtype dt, const esc_pointwise *a, void *out, void *stream)
{
    long P;
    if (dt != ESC_F32 && dt != ESC_BF16) return ESC_ERR_DTYPE;
    const esc_status st = shape(a, &P);
    if (st != ESC_OK) return st;
    if (x == nullptr || out == nullptr || a->w == nullptr) return ESC_ERR_NULL;
    const size_t es = dt == ESC_F32 ? 4 : 2, wb = (size_t)a->M * a->K * 4;
    Images xi, oi, ri{};
    if (!images_of(x, a->x_stride, a->N, (size_t)a->K * P, es, &xi) || !images_of(out, a->out_stride, a->N, (size_t)a->M * P, es, &oi)) return ESC_ERR_SHAPE;
    if (residual != nullptr && !images_of(residual, a->residual_stride, a->N, (size_t)a->M * P, es, &ri)) return ESC_ERR_SHAPE;
    if (((uintptr_t)a->w | (uintptr_t)a->b) % 4 != 0) return ESC_ERR_SHAPE;
    if (meet(oi, xi) || (residual != nullptr && meet(oi, ri)) || meets(oi, a->w, wb) || meets(oi, a->b, (size_t)a->M * 4)) return ESC_ERR_ALIAS;
    ProductParams p{};
    p.x = x, p.extra = residual, p.out = out;
    p.x_stride = (long)(xi.stride / es), p.out_stride = (long)(oi.stride / es), p.extra_stride = (long)(ri.stride / es);
    p.w = a->w, p.b = a->b, p.K = a->K, p.M = a->M, p.w_ld = a->K, p.act = (int)a->act, p.P = P, p.pixels = P * a->N;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = launch_any(dt == ESC_F32 ? kForwardF32 : kForwardBf16, p, a->N, s);
    return e == hipSuccess ? ESC_OK : ESC_ERR_HIP;
}

esc_status esc_pointwise_backward(const void *x, const void *grad_out, esc_dtype dt, const esc_pointwise *a, const esc_pointwise_grads *g, int accumulate,
                                  void *workspace, size_t workspace_bytes, void *stream)
{
    long P;
    if (dt != ESC_F32 && dt != ESC_BF16) return ESC_ERR_DTYPE;
    const esc_status st = shape(a, &P);
    if (st != ESC_OK) return st;
    if (x == nullptr || grad_out == nullptr || a->w == nullptr || g == nullptr) return ESC_ERR_NULL;
    if (g->x == nullptr && g->w == nullptr && g->b == nullptr) return ESC_ERR_NULL;
    const bool f32 = dt == ESC_F32;
    const size_t es = f32 ? 4 : 2, wb = (size_t)a->M * a->K * 4, vb = (size_t)a->M * 4;
    Images xi, gi, gxi{};
    if (!images_of(x, a->x_stride, a->N, (size_t)a->K * P, es, &xi) || !images_of(grad_out, a->out_stride, a->N, (size_t)a->M * P, es, &gi)) return ESC_ERR_SHAPE;
    if (g->x != nullptr && !images_of(g->x, g->x_stride, a->N, (size_t)a->K * P, es, &gxi)) return ESC_ERR_SHAPE;
    if (((uintptr_t)a->w | (uintptr_t)a->b | (uintptr_t)g->w | (uintptr_t)g->b) % 4 != 0) return ESC_ERR_SHAPE;
    const Scratch sc = scratch(a, P);
    if (workspace == nullptr || (uintptr_t)workspace % kAlign != 0 || workspace_bytes < sc.total) return ESC_ERR_WORKSPACE;
    // what is written overlaps nothing else
    const struct {
        const void *at;
        size_t bytes;
        bool written;
    } flat[] = {{a->w, wb, false}, {a->b, vb, false}, {g->w, wb, true}, {g->b, vb, true}, {workspace, sc.total, true}};
    const int n = (int)(sizeof(flat) / sizeof(flat[0]));
    if (g->x != nullptr && (meet(gxi, xi) || meet(gxi, gi))) return ESC_ERR_ALIAS;
    for (int i = 0; i < n; ++i) {
        if (flat[i].at == nullptr) continue;
        if (g->x != nullptr && meets(gxi, flat[i].at, flat[i].bytes)) return ESC_ERR_ALIAS;
        if (!flat[i].written) continue;
        if (meets(xi, flat[i].at, flat[i].bytes) || meets(gi, flat[i].at, flat[i].bytes)) return ESC_ERR_ALIAS;
        for (int j = 0; j < n; ++j)
            if (j != i && flat[j].at != nullptr && overlaps(flat[i].at, flat[i].bytes, flat[j].at, flat[j].bytes)) return ESC_ERR_ALIAS;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool act = a->act != ESC_ACT_NONE;
    char *mem = static_cast<char *>(workspace);
    const long x_stride = (long)(xi.stride / es), g_stride = (long)(gi.stride / es);
    if (act) {  // gp, fp32
        ProductParams p{};
        p.x = x, p.extra = grad_out, p.out = mem;
        p.x_stride = x_stride, p.extra_stride = g_stride, p.out_stride = (long)a->M * P;
        p.w = a->w, p.b = a->b, p.K = a->K, p.M = a->M, p.w_ld = a->K, p.act = (int)a->act, p.P = P, p.pixels = P * a->N;
        const hipError_t e = launch_any(f32 ? kSlopeF32 : kSlopeBf16, p, a->N, s);
        if (e != hipSuccess) return ESC_ERR_HIP;
    }
    if (g->x != nullptr) {
        ProductParams p{};
        p.x = act ? mem : grad_out, p.out = g->x;
        p.x_stride = act ? (long)a->M * P : g_stride, p.out_stride = (long)(gxi.stride / es);
        p.w = a->w, p.K = a->M, p.M = a->K, p.w_ld = a->K, p.act = kNone, p.P = P, p.pixels = P * a->N;
        const hipError_t e = launch_any(f32 ? kBackF32 : act ? kBackGp : kBackBf16, p, a->N, s);
        if (e != hipSuccess) return ESC_ERR_HIP;
    }
    if (g->w != nullptr || g->b != nullptr) {
        WeightParams p{};
        p.g = act ? mem : grad_out, p.x = x, p.g_stride = act ? (long)a->M * P : g_stride, p.x_stride = x_stride;
        p.part = g->w != nullptr ? reinterpret_cast<float *>(mem + sc.part) : nullptr;
        p.part_b = g->b != nullptr ? reinterpret_cast<float *>(mem + sc.part_b) : nullptr;
        p.K = a->K, p.M = a->M, p.splits = splits_of(a, P), p.P = P, p.pixels = P * a->N;
        const hipError_t e = f32 ? launch_weights<float, float, 3, 3>(p, s) : act ? launch_weights<float, bf16s, 3, 1>(p, s) : launch_weights<bf16s, bf16s, 1, 1>(p, s);
        if (e != hipSuccess) return ESC_ERR_HIP;
        if (g->w != nullptr && add_parts(p.part, p.splits, (long)a->M * a->K, g->w, 0, nullptr, accumulate, s) != hipSuccess) return ESC_ERR_HIP;
        if (g->b != nullptr && add_parts(p.part_b, p.splits, a->M, g->b, 0, nullptr, accumulate, s) != hipSuccess) return ESC_ERR_HIP;
    }
    return ESC_OK;
}

}  // extern "C"
