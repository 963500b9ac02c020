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
//
// Which kernel: up to 192 input channels (fp32 160) strip_kernel, and for gp and grad_x in one launch up to 128 (fp32 64) strip_back_kernel
// (esc_product_strip.hip), bound by memory; wider ones product_kernel, bound by the matrix and vector units; few pixels and outputs with many channels
// product_thin_kernel, bound by latency; grad_w product_weights_kernel.  One MI355X, 16 x 64 x 64, 640 to 1280 channels, gelu, bf16 (107 GFLOP a
// product), medians of 80 calls in a row (the first ten of a process are a sixth slower): forward 250 us (two products of terms, 860 TFLOP/s of those;
// 8192^3 in a library 1229), gp 343 (three, 940), grad_x 311 (three, 1040), grad_w 343 (three, 940).
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

// A wavefront owns 32 MT outputs of 32 NT pixels, a block four such runs of pixels: 128 outputs x 256 pixels where there is work enough.  (Both operands
// through LDS, tiles of 128 x 128: 1050 us for the forward pass above; weights read four bytes at a time, 16 lines an access: 481.)  Its input channels come in stages of 32, one or two stages ahead, straight into
// the registers of the right operand (esc_product_strip.hip); the weights pass LDS, split into terms there by the block a stage ahead, two buffers, one barrier a
// stage: units of eight consecutive channels of one output, [term][eighth of the stage][output].
//
// ACROSS: tiles pass images' borders (small images), or offsets take more than 32 bits: pixels by pointers of their own, one by one.
template <int MT, int TW>
struct Streamed {
    static constexpr int kPitch = 32 * MT + 2;   // (two: other banks for the eighths of a row, which neighbouring threads write)
    static constexpr int kBuffer = TW * 4 * kPitch;
    static constexpr size_t kLds = (size_t)2 * kBuffer * 16 + 32 * MT * 4;
};
extern __shared__ __align__(16) u32x4 product_lds[];

template <typename TI, typename TO, typename TE, int TX, int TW, int MT, int NT, bool TRANS, int MODE, bool ACROSS>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(const ProductParams p)
{
    using C = Streamed<MT, TW>;
    constexpr int kTop = TX > TW ? TX : TW;      // products of terms whose orders add up to less
    constexpr int kRuns = 256 * MT, kEach = kRuns / kThreads;  // runs of four weights of a stage, of a thread
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int K = p.K, M = p.M, stages = (K + 31) / 32;
    const unsigned groups = (unsigned)(M + 32 * MT - 1) / (32u * MT);
    const unsigned piece = p.first + piece_of(blockIdx.x, gridDim.x), tile = piece / groups;
    const int m0 = (int)(piece - tile * groups) * 32 * MT;
    const unsigned mine = 32u * NT * (unsigned)wave + NT * (unsigned)l32;   // this lane's first pixel, of the tile

    // ---- where the pixels are ----
    const long image = ACROSS ? 0 : tile / p.tiles;
    long pn[NT], pat[NT];   // ACROSS: each pixel's image, and its place there
    bool there[NT];
    unsigned pxc = 0;       // else the first one's place (a lane whose pixels reach beyond the plane takes its last ones again: the same bits are stored)
    if constexpr (ACROSS) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const long q = (long)tile * (128 * NT) + mine + t, in = min(q, p.pixels - 1);
            there[t] = q < p.pixels, pn[t] = in / p.P, pat[t] = in - pn[t] * p.P;
        }
    } else {
        const unsigned px = (unsigned)(tile - image * p.tiles) * (128u * NT) + mine, P = (unsigned)p.P;
        pxc = px + NT <= P ? px : P - NT;
    }

    // ---- channels of a stage: 32 st + 16 c + 8 half + j of this lane's pixels ----
    typedef Raw<TI, ACROSS ? 1 : NT> X;
    constexpr int kLoads = ACROSS ? NT : 1;
    constexpr int kAhead = kWide<TI> ? 1 : 2;   // stages that are asked for ahead: four bytes an element take the registers, and products the time
    const unsigned ib = (unsigned)p.P * (unsigned)sizeof(TI);
    const Rsrc rx = resource(static_cast<const TI *>(p.x) + image * p.x_stride, ACROSS ? 0 : (long)K * ib);
    const unsigned in_off = 8u * (unsigned)half * ib + pxc * (unsigned)sizeof(TI);
    auto xfetch = [&](int st, int c, X (&r)[8][kLoads]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = 32 * st + 16 * c + j, mine = k + 8 * half;
            if constexpr (ACROSS) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const TI v = static_cast<const TI *>(p.x)[pn[t] * p.x_stride + (long)min(mine, K - 1) * p.P + pat[t]];
                    if constexpr (kWide<TI>) r[j][t].w[0] = mine < K ? __float_as_uint(v) : 0u;
                    else r[j][t].w[0] = mine < K ? v.bits : 0u;
                }
            } else {
                r[j][0] = load<TI, NT>(rx, mine < K ? in_off : kBeyond, k < K ? (unsigned)k * ib : 0u);
            }
        }
    };

    // ---- weights of a stage ----
    const Rsrc rw = resource(p.w, 4L * K * M);
    const bool four = (K & 3) == 0;
    float wr[kEach][4];
    // (a row's runs, neighbours in memory, by neighbouring threads; TRANS: a channel's outputs)
    auto run_of = [&](int i, int &row, int &k4) {
        const int u = tid + i * kThreads;
        row = TRANS ? u % (32 * MT) : u >> 3, k4 = TRANS ? u / (32 * MT) : u & 7;
    };
    auto wfetch = [&](int st) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            int row, k4;
            run_of(i, row, k4);
            // (64 outputs and more: a wavefront's threads have one run of channels; 32: two)
            if constexpr (TRANS && MT == 1) load_weights_across(rw, M, K, p.w_ld, m0 + row, 32 * st + 8 * (__builtin_amdgcn_readfirstlane(k4) >> 1), 4 * (k4 & 1), wr[i]);
            else if constexpr (TRANS) load_weights_across(rw, M, K, p.w_ld, m0 + row, 32 * st + 4 * __builtin_amdgcn_readfirstlane(k4), 0, wr[i]);
            else load_weights(rw, M, K, p.w_ld, four, m0 + row, 32 * st + 4 * k4, wr[i]);
        }
    };
    auto wput = [&](int i, int st) {   // the i-th run
        u32x2 *ws = reinterpret_cast<u32x2 *>(product_lds + (st & 1) * C::kBuffer);
        int row, k4;
        run_of(i, row, k4);
        uint32_t t[2][TW];
        terms_of<TW>(wr[i][0], wr[i][1], t[0]);
        terms_of<TW>(wr[i][2], wr[i][3], t[1]);
#pragma unroll
        for (int q = 0; q < TW; ++q) ws[2 * ((q * 4 + (k4 >> 1)) * C::kPitch + row) + (k4 & 1)] = u32x2{t[0][q], t[1][q]};
    };

    // what is asked for stays in the order it is written in, and in front of the products that follow: at a wait for some of it the rest stays under way
    auto order = [] { __builtin_amdgcn_sched_barrier(kSchedNoVmemNoMfma); };
    X raw[kAhead][2][8][kLoads];
    wfetch(0);
    order();
#pragma unroll
    for (int d = 0; d < kAhead; ++d)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            xfetch(d, c, raw[d][c]);
            order();
        }
    float *bias = reinterpret_cast<float *>(product_lds + 2 * C::kBuffer);
    if (tid < 32 * MT) bias[tid] = p.b != nullptr && m0 + tid < M ? p.b[m0 + tid] : 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) wput(i, 0);
    f32x16 acc[MT][NT];
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[mt][t][i] = bias[32 * mt + 4 * half + 8 * (i >> 2) + (i & 3)];

    // a quarter of the right operand of sixteen channels: the terms of two of each lane's eight
    auto split = [&](const X (&raw)[8][kLoads], int e, u32x4 (&to)[NT][TX]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            constexpr bool one = kLoads > 1;
            const X &v0 = raw[2 * e][one ? t : 0], &v1 = raw[2 * e + 1][one ? t : 0];
            if constexpr (!kWide<TI> && TX == 1 && !ACROSS) {
                to[t][0][e] = __builtin_amdgcn_perm(v1.w[0], v0.w[0], t == 0 ? 0x05040100u : 0x07060302u);
            } else {
                uint32_t q[TX];
                terms_of<TX>(v0.value(one ? 0 : t), v1.value(one ? 0 : t), q);
#pragma unroll
                for (int i = 0; i < TX; ++i) to[t][i][e] = q[i];
            }
        }
    };
    // A stage's products in steps of 32 outputs and sixteen channels, each with the next one's weights asked for ahead and, between its matrix instructions, a
    // share of what is to be split: the second sixteen channels in the first MT steps, the next stage's weights in the others.
    auto body = [&](int st, X (&raw)[2][8][kLoads]) {
        static_assert(kEach == MT, "a run for each of the second sixteen channels' steps");
        const u32x4 *ws = product_lds + (st & 1) * C::kBuffer + half * C::kPitch + l32;
        auto weights_of = [&](int step, u32x4 (&a)[TW]) {
#pragma unroll
            for (int q = 0; q < TW; ++q) a[q] = ws[(q * 4 + 2 * (step / MT)) * C::kPitch + 32 * (step % MT)];
        };
        u32x4 b[2][NT][TX], next[TW];
        weights_of(0, next);
        wfetch(st + 1);
        order();
#pragma unroll
        for (int e = 0; e < 4; ++e) split(raw[0], e, b[0]);
        order();
        xfetch(st + kAhead, 0, raw[0]);
        order();
#pragma unroll
        for (int step = 0; step < 2 * MT; ++step) {
            const int c = step / MT, mt = step % MT;
            u32x4 a[TW];
#pragma unroll
            for (int q = 0; q < TW; ++q) a[q] = next[q];
            if (step + 1 < 2 * MT) weights_of(step + 1, next);
            // small terms first; neighbouring instructions on different sums
#pragma unroll
            for (int qw = TW - 1; qw >= 0; --qw)
#pragma unroll
                for (int qx = TX - 1; qx >= 0; --qx) {
                    if (qw + qx >= kTop) continue;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[mt][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[qw]), __builtin_bit_cast(bf16x8, b[c][t][qx]), acc[mt][t], 0, 0, 0);
                }
            if (c == 0) {
#pragma unroll
                for (int e = 4 * mt / MT; e < 4 * (mt + 1) / MT; ++e) split(raw[1], e, b[1]);
            } else {
                wput(mt, st + 1);
            }
            interleave<NT * (kTop == 1 ? 1 : TX == 1 || TW == 1 ? kTop : kTop * (kTop + 1) / 2)>();
            __builtin_amdgcn_sched_barrier(0);
            if (step == MT - 1) {
                xfetch(st + kAhead, 1, raw[1]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
    };
    // (beyond the last stage loads bring nothing, and zeros are put)
    int st = 0;
    for (; st + 1 < stages; st += 2) {
        body(st, raw[0]);
        body(st + 1, raw[kAhead - 1]);
    }
    if (st < stages) body(st, raw[0]);
    settle();

    // ---- lane l has outputs m0 + 32 mt + 8 (i / 4) + 4 half + i % 4 in element i of its pixels' sums ----
    auto row_of = [](int i) { return 8 * (i >> 2) + (i & 3); };
    const unsigned ob = (unsigned)p.P * (unsigned)sizeof(TO), eb = (unsigned)p.P * (unsigned)sizeof(TE);
    constexpr bool has = MODE != kForward;
    const Rsrc ro = resource(static_cast<TO *>(p.out) + image * p.out_stride, ACROSS ? 0 : (long)M * ob);
    const Rsrc re = resource(has ? static_cast<const TE *>(p.extra) + image * p.extra_stride : nullptr, ACROSS || !has ? 0 : (long)M * eb);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int left = M - (m0 + 32 * mt) - 4 * half;
        float v[NT * 16], e[NT * 16];
        if constexpr (has && ACROSS) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    e[16 * t + i] = widen(static_cast<const TE *>(p.extra)[pn[t] * p.extra_stride + (long)min(m0 + 32 * mt + 4 * half + row_of(i), M - 1) * p.P + pat[t]]);
        } else if constexpr (has) {
            const unsigned off = (unsigned)(m0 + 32 * mt + 4 * half) * eb + pxc * (unsigned)sizeof(TE);
            Raw<TE, NT> ex[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) ex[i] = load<TE, NT>(re, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * eb);
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t) e[16 * t + i] = ex[i].value(t);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[16 * t + i] = acc[mt][t][i];
        if constexpr (MODE == kSlope) {
            slopes(p.act, v);
#pragma unroll
            for (int i = 0; i < NT * 16; ++i) v[i] *= e[i];
        } else {
            activate(p.act, v);
            if constexpr (MODE == kResidual) {
#pragma unroll
                for (int i = 0; i < NT * 16; ++i) v[i] += e[i];
            }
        }
        if constexpr (ACROSS) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (there[t] && row_of(i) < left) {
                        TO *to = static_cast<TO *>(p.out) + pn[t] * p.out_stride + (long)(m0 + 32 * mt + 4 * half + row_of(i)) * p.P + pat[t];
                        if constexpr (kWide<TO>) *to = v[16 * t + i];
                        else to->bits = (uint16_t)pack2(v[16 * t + i], 0.f);
                    }
        } else {
            const unsigned off = (unsigned)(m0 + 32 * mt + 4 * half) * ob + pxc * (unsigned)sizeof(TO);
#pragma unroll
            for (int i = 0; i < 16; ++i) store<TO, NT>(ro, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * ob, v[i], v[16 * (NT - 1) + i]);
        }
    }
}

template <typename TI, typename TO, typename TE, int TX, int TW, int MT, int NT, bool TRANS, int MODE, bool ACROSS>
hipError_t launch_as(ProductParams p, long N, hipStream_t s)
{
    using C = Streamed<MT, TW>;
    p.tiles = ((ACROSS ? p.pixels : p.P) + 128 * NT - 1) / (128 * NT);
    const long grid = p.tiles * (ACROSS ? 1 : N) * ((p.M + 32 * MT - 1) / (32 * MT));
    const auto kernel = product_kernel<TI, TO, TE, TX, TW, MT, NT, TRANS, MODE, ACROSS>;
    static_assert(C::kLds <= 64 * 1024, "");
    return in_launches(grid, kThreads, [&](long first, unsigned blocks) {
        p.first = (unsigned)first;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), C::kLds, s, p);
        return hipGetLastError();
    });
}

template <typename TI, typename TO, typename TE, int TX, int TW, bool TRANS, int MODE>
hipError_t launch_product(const ProductParams &p, long N, hipStream_t s)
{
    // small images share tiles; their pixels, and those of images beyond 2 GiB, go one by one
    const size_t widest = std::max(std::max(p.K * sizeof(TI), p.M * sizeof(TO)), p.M * sizeof(TE)) * (size_t)p.P;
    if (widest >= kMostImage || p.P > kMostPlane || p.P < 2 || (N > 1 && p.P < 96)) return launch_as<TI, TO, TE, TX, TW, 2, 1, TRANS, MODE, true>(p, N, s);
    const auto blocks = [&](int mt, int nt) { return N * ((p.P + 128 * nt - 1) / (128 * nt)) * ((p.M + 32 * mt - 1) / (32 * mt)); };
    // as much for a wavefront as leaves every compute unit two blocks (and, with three terms of both, registers)
    if constexpr (TX != 3)
        if (p.M > 64 && blocks(4, 2) >= 2 * kCus) return launch_as<TI, TO, TE, TX, TW, 4, 2, TRANS, MODE, false>(p, N, s);
    if (p.M <= 32) {
        // (gp of that many pixels has its grad_x in the same launch: back_fits)
        if constexpr (!(kWide<TI> && !kWide<TO>))
            if (blocks(1, 2) >= 2 * kCus) return launch_as<TI, TO, TE, TX, TW, 1, 2, TRANS, MODE, false>(p, N, s);
        return launch_as<TI, TO, TE, TX, TW, 1, 1, TRANS, MODE, false>(p, N, s);
    }
    if (blocks(2, 2) >= 2 * kCus) return launch_as<TI, TO, TE, TX, TW, 2, 2, TRANS, MODE, false>(p, N, s);
    return launch_as<TI, TO, TE, TX, TW, 2, 1, TRANS, MODE, false>(p, N, s);
}

// ---- few pixels and outputs, many channels: a block's eight wavefronts share one tile of 32 outputs and 32 pixels and take every eighth sixteen of its channels
// each, both operands straight from memory; their sums are added in LDS ----

constexpr int kThinWaves = 8, kThinAhead = 4;   // sixteens that are under way at a time

template <typename TI, typename TO, typename TE, int TX, int TW, bool TRANS, int MODE>
__global__ __launch_bounds__(64 * kThinWaves) void product_thin_kernel(const ProductParams p)
{
    constexpr int kTop = TX > TW ? TX : TW;
    __shared__ float sums[kThinWaves][16][64];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5, K = p.K, M = p.M, sixteens = (K + 15) / 16;
    const unsigned groups = (unsigned)(M + 31) / 32u, piece = piece_of(blockIdx.x, gridDim.x), tile = piece / groups;
    const int m0 = (int)(piece - tile * groups) * 32;
    const long q = (long)tile * 32 + l32, in = min(q, p.pixels - 1), n = in / p.P, at = in - n * p.P;
    const TI *const x = static_cast<const TI *>(p.x) + n * p.x_stride + at;
    const Rsrc rw = resource(p.w, 4L * K * M);
    const bool four = (K & 3) == 0;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    for (int c0 = wave; c0 < sixteens; c0 += kThinWaves * kThinAhead) {
        TI xr[kThinAhead][8];
        float wr[kThinAhead][8];
#pragma unroll
        for (int u = 0; u < kThinAhead; ++u) {
            // (a sixteen beyond the last brings zeros)
            const int k = 16 * (c0 + kThinWaves * u) + 8 * half;
#pragma unroll
            for (int j = 0; j < 8; ++j) xr[u][j] = x[(long)min(k + j, K - 1) * p.P];
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                float w[4];
                if constexpr (TRANS) load_weights_across(rw, M, K, p.w_ld, m0 + l32, 16 * (c0 + kThinWaves * u) + j, 8 * half, w);
                else load_weights(rw, M, K, p.w_ld, four, m0 + l32, k + j, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) wr[u][j + e] = w[e];
            }
        }
#pragma unroll
        for (int u = 0; u < kThinAhead; ++u) {
            const int left = K - (16 * (c0 + kThinWaves * u) + 8 * half);
            u32x4 a[TW], b[TX];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t ta[TW], tb[TX];
                terms_of<TW>(wr[u][2 * e], wr[u][2 * e + 1], ta);
                terms_of<TX>(2 * e < left ? widen(xr[u][2 * e]) : 0.f, 2 * e + 1 < left ? widen(xr[u][2 * e + 1]) : 0.f, tb);
#pragma unroll
                for (int i = 0; i < TW; ++i) a[i][e] = ta[i];
#pragma unroll
                for (int i = 0; i < TX; ++i) b[i][e] = tb[i];
            }
#pragma unroll
            for (int qw = TW - 1; qw >= 0; --qw)
#pragma unroll
                for (int qx = TX - 1; qx >= 0; --qx)
                    if (qw + qx < kTop)
                        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[qw]), __builtin_bit_cast(bf16x8, b[qx]), acc, 0, 0, 0);
        }
    }
    settle();
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    const bool has = p.extra != nullptr;
    constexpr int kMine = 16 / kThinWaves;
    float v[kMine], e[kMine];
    int row[kMine];
#pragma unroll
    for (int r = 0; r < kMine; ++r) {
        const int i = kMine * wave + r;
        row[r] = m0 + 8 * (i >> 2) + 4 * half + (i & 3);
        e[r] = has ? widen(static_cast<const TE *>(p.extra)[n * p.extra_stride + (long)min(row[r], M - 1) * p.P + at]) : 0.f;
        v[r] = p.b != nullptr ? p.b[min(row[r], M - 1)] : 0.f;
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kThinWaves; ++w) t += sums[w][i][lane];
        v[r] += t;
    }
    if constexpr (MODE == kSlope) {
        slopes(p.act, v);
#pragma unroll
        for (int r = 0; r < kMine; ++r) v[r] *= e[r];
    } else {
        activate(p.act, v);
#pragma unroll
        for (int r = 0; r < kMine; ++r) v[r] += e[r];
    }
    if (q >= p.pixels) return;
#pragma unroll
    for (int r = 0; r < kMine; ++r)
        if (row[r] < M) {
            TO *to = static_cast<TO *>(p.out) + n * p.out_stride + (long)row[r] * p.P + at;
            if constexpr (kWide<TO>) *to = v[r];
            else to->bits = (uint16_t)pack2(v[r], 0.f);
        }
}

template <typename TI, typename TO, typename TE, int TX, int TW, bool TRANS, int MODE>
hipError_t launch_thin(const ProductParams &p, hipStream_t s)
{
    const long grid = (p.pixels + 31) / 32 * ((p.M + 31) / 32);
    hipLaunchKernelGGL((product_thin_kernel<TI, TO, TE, TX, TW, TRANS, MODE>), dim3((unsigned)grid), dim3(64 * kThinWaves), 0, s, p);
    return hipGetLastError();
}

// Where the other kernels would leave most compute units without a block, and a block with a long way through the channels.
bool thin_fits(const ProductParams &p) { return p.K >= 128 && (p.pixels + 127) / 128 * ((p.M + 63) / 64) < kCus / 2; }

hipError_t launch_any(int kind, const ProductParams &p, long N, hipStream_t s)
{
    if (thin_fits(p)) {
        switch (kind) {
        case kForwardF32: return launch_thin<float, float, float, 3, 3, false, kForward>(p, s);
        case kForwardBf16: return launch_thin<bf16s, bf16s, bf16s, 1, 2, false, kForward>(p, s);
        case kSlopeF32: return launch_thin<float, float, float, 3, 3, false, kSlope>(p, s);
        case kSlopeBf16: return launch_thin<bf16s, float, bf16s, 1, 3, false, kSlope>(p, s);
        case kBackF32: return launch_thin<float, float, float, 3, 3, true, kForward>(p, s);
        case kBackBf16: return launch_thin<bf16s, bf16s, bf16s, 1, 2, true, kForward>(p, s);
        case kBackGp: return launch_thin<float, bf16s, bf16s, 2, 2, true, kForward>(p, s);
        default: return hipErrorInvalidValue;
        }
    }
    if (strip_fits(kind, p, N)) return launch_strip(kind, p, N, s);
    switch (kind) {
    case kForwardF32: return p.extra != nullptr ? launch_product<float, float, float, 3, 3, false, kResidual>(p, N, s) : launch_product<float, float, float, 3, 3, false, kForward>(p, N, s);
    case kForwardBf16: return p.extra != nullptr ? launch_product<bf16s, bf16s, bf16s, 1, 2, false, kResidual>(p, N, s) : launch_product<bf16s, bf16s, bf16s, 1, 2, false, kForward>(p, N, s);
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

constexpr int kPixels = 32;   // of a stage

struct WeightParams {
    const void *g, *x;
    long g_stride, x_stride;
    float *part;              // [splits][M K of grad_w where that is wanted, then M of grad_b where that is]
    bool has_w, has_b;
    int K, M, splits, tiles, across;   // (tiles of grad_w, and those side by side)
    long P, pixels;
};

// A run of pixels of one row, 16 bytes of it.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Run {
    static constexpr int kCount = 16 / (int)sizeof(T);
    T e[kCount];
};

// One operand of a block's tile: ROWS rows, staged as units of eight consecutive pixels, [term][eighth of the stage][row].
template <typename T, int Q, int ROWS>
struct Staged {
    typedef Run<T> R;
    static constexpr int kEights = kPixels / 8, kPitch = ROWS + 2, kUnits = Q * kEights * kPitch;
    static constexpr int kRunsOfRow = kPixels / R::kCount, kEach = ROWS * kRunsOfRow / kThreads;
    R r[kEach];
    __device__ __forceinline__ static int row_of(int i) { return ((int)threadIdx.x + i * kThreads) / kRunsOfRow; }
    __device__ __forceinline__ static int run_of(int i) { return ((int)threadIdx.x + i * kThreads) % kRunsOfRow; }
    // Rows first, first + 1, ... (the last one's again beyond it) of a stage that lies in one image, `at` its first pixel there.
    __device__ __forceinline__ void whole(const T *image, long P, long at, int first, int rows)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            r[i] = *reinterpret_cast<const R *>(image + (long)min(first + row_of(i), rows - 1) * P + at + R::kCount * run_of(i));
    }
    // The same of a stage that begins with pixel `at` of image n and passes the image's border or, `left` pixels on, the last image's: pixel by pixel,
    // zeros beyond the last.
    __device__ __forceinline__ void scattered(const T *base, long stride, long P, long left, long n, long at, int first, int rows)
    {
        static_assert(kThreads % kRunsOfRow == 0, "a thread's runs are of the same pixels");
        const int mine = R::kCount * run_of(0);
        long pn = n, pat = at + mine;
        while (pat >= P) pat -= P, ++pn;
#pragma unroll
        for (int j = 0; j < R::kCount; ++j) {
            const bool in = mine + j < left;
            const T *const pixel = base + (in ? pn * stride + pat : n * stride + at);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const T v = pixel[(long)min(first + row_of(i), rows - 1) * P];
                r[i].e[j] = in ? v : T{};
            }
            if (++pat == P) pat = 0, ++pn;
        }
    }
    __device__ __forceinline__ void put(u32x4 *lds, float *sums) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if constexpr (R::kCount == 4) {
                uint32_t t[2][Q];
                terms_of<Q>(widen(r[i].e[0]), widen(r[i].e[1]), t[0]);
                terms_of<Q>(widen(r[i].e[2]), widen(r[i].e[3]), t[1]);
#pragma unroll
                for (int q = 0; q < Q; ++q)
                    reinterpret_cast<uint2 *>(lds + (q * kEights + (run_of(i) >> 1)) * kPitch + row_of(i))[run_of(i) & 1] = uint2{t[0][q], t[1][q]};
                if (sums != nullptr) sums[i] += (widen(r[i].e[0]) + widen(r[i].e[1])) + (widen(r[i].e[2]) + widen(r[i].e[3]));
            } else {
                static_assert(R::kCount == 4 || Q == 1, "two bytes an element are a term each");
                lds[run_of(i) * kPitch + row_of(i)] = __builtin_bit_cast(u32x4, r[i]);
                if (sums != nullptr) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) sums[i] += widen(r[i].e[j]) + widen(r[i].e[j + 1]);
                }
            }
        }
    }
};

// A block's tile of grad_w is 64 MT x 64 KT, a wavefront's 32 MT x 32 KT.
//
// Products of the first terms have sums of their own, `acc`, those of the others `low`: the matrix unit cuts off what lies far below the sum that it
// adds to, always downwards, and over the thousands of additions of a long share that leans to one side.  (One sum for all, 31 x 3 gradients over
// 4096 x 4096 pixels, fp32, normal values: all of them too low, 3.9e-5 of their 2-norm, now 1.3e-6; 1024 x 1024: 2.3e-6, now 3.0e-7.  The times are the
// same, both builds in turn: 16 x 64 x 64 of 640 to 1280 channels fp32 666 and 664 us; the whole backward pass of 64 to 128 channels, 64 x 64 x 64,
// gelu, bf16 101 both.)
template <typename TG, typename TI, int QG, int QX, int MT, int KT>
__global__ __launch_bounds__(kThreads, 2) void product_weights_kernel(const WeightParams p)
{
    constexpr int kTop = QG > QX ? QG : QX, BM = 64 * MT, BK = 64 * KT;
    typedef Staged<TG, QG, BM> G;
    typedef Staged<TI, QX, BK> X;
    __shared__ u32x4 s[2][G::kUnits + X::kUnits];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, wm = wave & 1, wk = wave >> 1;
    // the tiles of a split, which read the same pixels, follow one another on one die
    const unsigned piece = piece_of(blockIdx.x, gridDim.x), split = piece / (unsigned)p.tiles;
    const int tile = (int)(piece - split * (unsigned)p.tiles), m0 = tile / p.across * BM, k0 = tile % p.across * BK;
    const long stages = (p.pixels + kPixels - 1) / kPixels;
    const long first = stages * split / p.splits, end = stages * (split + 1) / p.splits;
    const TG *const gp = static_cast<const TG *>(p.g);
    const TI *const xp = static_cast<const TI *>(p.x);
    G g;
    X x;
    // the stage that is fetched next: its first pixel, of all images' and of its image
    long q = first * kPixels, n = q / p.P, at = q - n * p.P;
    auto fetch = [&] {
        if (at + kPixels <= p.P) {  // (the same for the block)
            g.whole(gp + n * p.g_stride, p.P, at, m0, p.M);
            x.whole(xp + n * p.x_stride, p.P, at, k0, p.K);
        } else {
            g.scattered(gp, p.g_stride, p.P, p.pixels - q, n, at, m0, p.M);
            x.scattered(xp, p.x_stride, p.P, p.pixels - q, n, at, k0, p.K);
        }
        q += kPixels, at += kPixels;
        if (at >= p.P) {
            const long images = at / p.P;
            n += images, at -= images * p.P;
        }
    };
    const bool has_b = p.has_b && k0 == 0;
    const size_t of_w = p.has_w ? (size_t)p.M * p.K : 0;
    float *const part = p.part + split * (of_w + (p.has_b ? p.M : 0));
    float sums[G::kEach];
#pragma unroll
    for (int i = 0; i < G::kEach; ++i) sums[i] = 0.f;
    auto put = [&](int buffer) {
        g.put(s[buffer], has_b ? sums : nullptr);
        x.put(s[buffer] + G::kUnits, nullptr);
    };
    f32x16 acc[MT][KT], low[MT][KT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = low[i][j][e] = 0.f;
    if (first < end) {
        fetch();
        put(0);
    }
    __syncthreads();
    for (long st = first; st < end; ++st) {
        const int buffer = (int)(st - first) & 1;
        if (st + 1 < end) fetch();
        const u32x4 *gs = s[buffer] + 32 * MT * wm + l32, *xs = s[buffer] + G::kUnits + 32 * KT * wk + l32;
#pragma unroll
        for (int c = 0; c < kPixels / 16; ++c) {
            u32x4 a[MT][QG], b[KT][QX];
#pragma unroll
            for (int j = 0; j < KT; ++j)
#pragma unroll
                for (int q = 0; q < QX; ++q) b[j][q] = xs[(q * X::kEights + 2 * c + half) * X::kPitch + 32 * j];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < QG; ++q) a[i][q] = gs[(q * G::kEights + 2 * c + half) * G::kPitch + 32 * i];
#pragma unroll
            for (int qg = QG - 1; qg >= 0; --qg)
#pragma unroll
                for (int qx = QX - 1; qx >= 0; --qx) {
                    if (qg + qx >= kTop) continue;
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int j = 0; j < KT; ++j) {
                            f32x16 &to = qg + qx > 0 ? low[i][j] : acc[i][j];
                            to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i][qg]), __builtin_bit_cast(bf16x8, b[j][qx]), to, 0, 0, 0);
                        }
                }
        }
        if (st + 1 < end) put(buffer ^ 1);
        __syncthreads();
    }
    settle();
    if (p.has_w) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                const int k = k0 + 32 * (KT * wk + j) + l32;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int m = m0 + 32 * (MT * wm + t) + 8 * (i >> 2) + 4 * half + (i & 3);
                    const float v = acc[t][j][i] + low[t][j][i];
                    if (m < p.M && k < p.K) part[(size_t)m * p.K + k] = v;
                }
            }
    }
    if (has_b) {
        // a row's runs are neighbouring threads'
        float *const all = reinterpret_cast<float *>(s[0]);
#pragma unroll
        for (int i = 0; i < G::kEach; ++i) all[tid + i * kThreads] = sums[i];
        __syncthreads();
        if (tid < BM && m0 + tid < p.M) {
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < G::kRunsOfRow; ++j) t += all[tid * G::kRunsOfRow + j];
            part[of_w + m0 + tid] = t;
        }
    }
}

// A block's sides of grad_w in 64s: 128 where there are more than 64 channels, but one of them alone where six terms take all the LDS.
struct Sides {
    int mt, kt;
};
Sides sides_of(int M, int K, bool f32)
{
    const int mt = M > 64 ? 2 : 1;
    return Sides{mt, K > 64 && !(f32 && mt == 2) ? 2 : 1};
}

template <typename TG, typename TI, int QG, int QX>
hipError_t launch_weights(WeightParams p, hipStream_t s)
{
    const auto [mt, kt] = sides_of(p.M, p.K, kWide<TI>);
    p.across = (p.K + 64 * kt - 1) / (64 * kt), p.tiles = p.across * ((p.M + 64 * mt - 1) / (64 * mt));
    const dim3 grid((unsigned)p.tiles * (unsigned)p.splits), block(kThreads);
    if constexpr (!kWide<TI>) {
        if (mt == 2 && kt == 2) {
            hipLaunchKernelGGL((product_weights_kernel<TG, TI, QG, QX, 2, 2>), grid, block, 0, s, p);
            return hipGetLastError();
        }
    }
    if (mt == 2) hipLaunchKernelGGL((product_weights_kernel<TG, TI, QG, QX, 2, 1>), grid, block, 0, s, p);
    else if (kt == 2) hipLaunchKernelGGL((product_weights_kernel<TG, TI, QG, QX, 1, 2>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((product_weights_kernel<TG, TI, QG, QX, 1, 1>), grid, block, 0, s, p);
    return hipGetLastError();
}

// ---- host side ----

esc_status shape(const esc_pointwise *a, long *P)
{
    if (a == nullptr) return ESC_ERR_NULL;
    if (a->N < 1 || a->K < 1 || a->M < 1 || a->H < 1 || a->W < 1) return ESC_ERR_SHAPE;
    if (a->act != ESC_ACT_NONE && a->act != ESC_ACT_GELU && a->act != ESC_ACT_SILU) return ESC_ERR_SHAPE;
    *P = (long)a->H * a->W;
    if (a->K > 65536 || a->M > 65536 || (long)a->K * a->M >= (1L << 29) || *P >= (1L << 31) || (double)*P * a->N >= 0x1p40) return ESC_ERR_UNSUPPORTED;
    // (the smallest pieces of either product, numbered in 32 bits: 128 pixels of an image, or of all images where these are small, and 32 channels)
    const long tiles = a->N == 1 || *P >= 96 ? a->N * ((*P + 127) / 128) : (a->N * *P + 127) / 128;
    if (tiles * ((std::max(a->K, a->M) + 31) / 32) >= (1L << 31)) return ESC_ERR_UNSUPPORTED;
    return ESC_OK;
}

// Shares of the pixels: two blocks a compute unit and no more (11 shares of 50 tiles, a round of 38 blocks behind one of 512: 560 us, 10 shares 390), two stages
// each at least.
int splits_of(const esc_pointwise *a, long P, bool f32)
{
    const Sides side = sides_of(a->M, a->K, f32);
    const long mt = 64 * side.mt, kt = 64 * side.kt;
    const long tiles = ((a->M + mt - 1) / mt) * ((a->K + kt - 1) / kt), stages = ((long)a->N * P + kPixels - 1) / kPixels;
    return (int)std::max<long>(1, std::min(2 * kCus / tiles, stages / 2));
}

struct Scratch {
    size_t gp, part, total;
};
Scratch scratch(const esc_pointwise *a, long P, bool f32)
{
    Scratch s;
    const size_t splits = (size_t)splits_of(a, P, f32);
    s.gp = 0;
    s.part = a->act != ESC_ACT_NONE ? round_up((size_t)a->N * P * a->M * 4, kAlign) : 0;
    s.total = s.part + round_up(splits * a->M * ((size_t)a->K + 1) * 4, kAlign);
    return s;
}

}  // namespace

extern "C" {

size_t esc_pointwise_backward_workspace_bytes(const esc_pointwise *a, esc_dtype dt)
{
    long P;
    return (dt == ESC_F32 || dt == ESC_BF16) && shape(a, &P) == ESC_OK ? scratch(a, P, dt == ESC_F32).total : 0;
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
    const Scratch sc = scratch(a, P, f32);
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
    const bool sums = g->w != nullptr || g->b != nullptr;
    const bool joint = act && g->x != nullptr && back_fits(f32, a->K, a->M, P, a->N);
    if (joint) {
        BackParams p{};
        p.x = x, p.grad_out = grad_out, p.gp = sums ? reinterpret_cast<float *>(mem) : nullptr, p.grad_x = g->x;
        p.x_stride = x_stride, p.g_stride = g_stride, p.gp_stride = (long)a->M * P, p.gx_stride = (long)(gxi.stride / es);
        p.w = a->w, p.b = a->b, p.K = a->K, p.M = a->M, p.act = (int)a->act, p.P = P;
        if (launch_back(f32, p, a->N, s) != hipSuccess) return ESC_ERR_HIP;
    } else if (act) {  // gp, fp32
        ProductParams p{};
        p.x = x, p.extra = grad_out, p.out = mem;
        p.x_stride = x_stride, p.extra_stride = g_stride, p.out_stride = (long)a->M * P;
        p.w = a->w, p.b = a->b, p.K = a->K, p.M = a->M, p.w_ld = a->K, p.act = (int)a->act, p.P = P, p.pixels = P * a->N;
        const hipError_t e = launch_any(f32 ? kSlopeF32 : kSlopeBf16, p, a->N, s);
        if (e != hipSuccess) return ESC_ERR_HIP;
    }
    if (g->x != nullptr && !joint) {
        ProductParams p{};
        p.x = act ? mem : grad_out, p.out = g->x;
        p.x_stride = act ? (long)a->M * P : g_stride, p.out_stride = (long)(gxi.stride / es);
        p.w = a->w, p.K = a->M, p.M = a->K, p.w_ld = a->K, p.act = kNone, p.P = P, p.pixels = P * a->N;
        const hipError_t e = launch_any(f32 ? kBackF32 : act ? kBackGp : kBackBf16, p, a->N, s);
        if (e != hipSuccess) return ESC_ERR_HIP;
    }
    if (sums) {
        WeightParams p{};
        p.g = act ? mem : grad_out, p.x = x, p.g_stride = act ? (long)a->M * P : g_stride, p.x_stride = x_stride;
        p.part = reinterpret_cast<float *>(mem + sc.part), p.has_w = g->w != nullptr, p.has_b = g->b != nullptr;
        p.K = p.has_w ? a->K : 1, p.M = a->M, p.splits = splits_of(a, P, f32), p.P = P, p.pixels = P * a->N;
        const hipError_t e = f32 ? launch_weights<float, float, 3, 3>(p, s) : act ? launch_weights<float, bf16s, 3, 1>(p, s) : launch_weights<bf16s, bf16s, 1, 1>(p, s);
        if (e != hipSuccess) return ESC_ERR_HIP;
        if (add_parts(p.part, p.splits, p.has_w ? (long)a->M * a->K : 0, g->w, p.has_b ? a->M : 0, g->b, accumulate, s) != hipSuccess) return ESC_ERR_HIP;
    }
    return ESC_OK;
}

}  // extern "C"
