// Point-wise products whose input channels are few enough to stay in registers (esc_product.hpp).
//
// A wavefront owns 32 NT pixels and has all K input channels of them in registers as the right operand of v_mfma_f32_32x32x16_bf16: a lane holds
// eight consecutive channels of its pixel for each sixteen, as eight loads of channel rows bring them (32 lanes on a run of 32 NT pixels), split into
// terms once.  The weights pass LDS in chunks of 32 outputs, two buffers, one barrier a chunk; behind a chunk's products stand its
// activation, residual and stores, while other wavefronts multiply.  x is read once where one block takes all outputs.
//
// What bounds it: memory, for as many channels as the vector units' share (splitting, activation) hides behind.  MI355X, over several cards:
// 339 x 511, 64 to 64 channels with residual, fp32 23.2 us where the last-level cache holds its inputs, 28 to 32 with others in each call (133 MB, 4.2
// to 4.8 TB/s); 64 x 64 x 64, 64 to 128, gelu, bf16 forward 29 to 34 (101 MB: one round of blocks, whose reading and writing do not overlap), gp and
// grad_x 60 to 71 (268 MB, 3.8 to 4.5 TB/s; as two kernels 84); 180 x 320, 192 to 576, bf16 30 to 35 (730 to 850 TFLOP/s of products of terms); a
// kernel that stages both operands in LDS: 57, 97, 290 and 150.
#include "esc_host.hpp"
#include "esc_product.hpp"

#include <algorithm>
#include <type_traits>

namespace esc {
namespace {

// Weights of a chunk in LDS: units of eight consecutive channels of one output, [term][eighth][output], eighths a unit further apart than outputs
// take (other banks for a thread's neighbours, who write other eighths of the same output).
constexpr int kPitch = 33;

template <int KC, int TW>
struct StripLds {
    static constexpr int kUnits = KC * TW * 2 * kPitch;
    static constexpr size_t kBytes = (size_t)2 * kUnits * 16 + 2 * 32 * 4;
};
extern __shared__ __align__(16) u32x4 strip_lds[];

// A wavefront's pixels as right operands: channel 16 c + 8 half + j of its lanes' NT pixels, whose first channel's place (of this half) is `off`.  Four
// sixteens are on their way while the four before them are split; `meanwhile` is done behind the first.
template <typename T, int TX, int KC, int NT, typename F>
__device__ __forceinline__ void load_operands(Rsrc rx, unsigned off, unsigned plane, int K, u32x4 (&b)[KC][NT][TX], F meanwhile)
{
    constexpr int kGroup = KC < 4 ? KC : 4;
    const int half = ((int)threadIdx.x & 63) >> 5;
    Raw<T, NT> r[2][kGroup][8];
    auto ask = [&](int g) {
#pragma unroll
        for (int c = 0; c < kGroup; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = 16 * (kGroup * g + c) + j;
                if (kGroup * g + c < KC) r[g & 1][c][j] = load<T, NT>(rx, k + 8 * half < K ? off : kBeyond, k < K ? (unsigned)k * plane : 0u);
            }
        __builtin_amdgcn_sched_barrier(kSchedNoVmem);
    };
    auto split = [&](int g) {
#pragma unroll
        for (int c = 0; c < kGroup; ++c) {
            if (kGroup * g + c >= KC) break;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const Raw<T, NT> &v0 = r[g & 1][c][2 * e], &v1 = r[g & 1][c][2 * e + 1];
                    u32x4 (&to)[TX] = b[kGroup * g + c][t];
                    if constexpr (!kWide<T> && TX == 1) {
                        to[0][e] = __builtin_amdgcn_perm(v1.w[0], v0.w[0], t == 0 ? 0x05040100u : 0x07060302u);
                    } else {
                        uint32_t q[TX];
                        terms_of<TX>(v0.value(t), v1.value(t), q);
#pragma unroll
                        for (int i = 0; i < TX; ++i) to[i][e] = q[i];
                    }
                }
        }
    };
    constexpr int kAll = (KC + kGroup - 1) / kGroup;
    ask(0);
    if constexpr (kAll > 1) ask(1);
    meanwhile();
#pragma unroll
    for (int g = 0; g < kAll; ++g) {
        split(g);
        if (g + 2 < kAll) ask(g + 2);
    }
}

struct StripParams : ProductParams {
    int each;   // chunks of 32 outputs a block
    unsigned parts;
    unsigned tiles_of_image;
};

// blocks of a compute unit, by what the operands leave of the registers
constexpr int strip_blocks(int words, bool more) { return words <= 32 && !more ? 4 : words < 48 ? 3 : 2; }

template <typename TI, typename TO, typename TE, int TX, int TW, int KC, int NT, bool TRANS, int MODE>
__global__ __launch_bounds__(kThreads, strip_blocks(4 * KC * NT * TX, MODE != kForward || TRANS)) void strip_kernel(const StripParams p)
{
    constexpr int kTop = TX > TW ? TX : TW;      // products of terms whose orders add up to less
    constexpr int kRuns = 128 * KC, kEach = kRuns / kThreads;  // runs of four weights of a chunk, of a thread
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int K = p.K, M = p.M;
    const unsigned P = (unsigned)p.P;
    const unsigned piece = p.first + piece_of(blockIdx.x, gridDim.x), tile = piece / p.parts, n = tile / p.tiles_of_image;
    const int c0 = (int)(piece - tile * p.parts) * p.each, c1 = min(c0 + p.each, (M + 31) / 32);
    const unsigned px = (tile - n * p.tiles_of_image) * (128u * NT) + 32u * NT * (unsigned)wave + NT * (unsigned)l32;
    // (a lane whose pixels reach beyond the plane takes the plane's last ones again: the same bits are stored)
    const unsigned pxc = px + NT <= P ? px : P - NT;

    // ---- weights ----
    const Rsrc rw = resource(p.w, 4L * K * M);
    const bool four = (K & 3) == 0;
    float wr[kEach][4];
    float br = 0.f;
    // (a row's runs, neighbours in memory, by neighbouring threads; TRANS: a channel's outputs)
    auto run_of = [&](int i, int &row, int &k4) {
        const int u = tid + i * kThreads;
        row = TRANS ? u & 31 : u / (4 * KC), k4 = TRANS ? u >> 5 : u % (4 * KC);
    };
    auto wfetch = [&](int chunk) {
        br = p.b != nullptr && tid < 32 ? p.b[min(32 * chunk + tid, M - 1)] : 0.f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            int row, k4;
            run_of(i, row, k4);
            if constexpr (TRANS) load_weights_across(rw, M, K, p.w_ld, 32 * chunk + row, 8 * (__builtin_amdgcn_readfirstlane(k4) >> 1), 4 * (k4 & 1), wr[i]);
            else load_weights(rw, M, K, p.w_ld, four, 32 * chunk + row, 4 * k4, wr[i]);
        }
    };
    auto wput = [&](int buffer) {
        u32x2 *ws = reinterpret_cast<u32x2 *>(strip_lds + buffer * StripLds<KC, TW>::kUnits);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            int row, k4;
            run_of(i, row, k4);
            uint32_t t[2][TW];
            terms_of<TW>(wr[i][0], wr[i][1], t[0]);
            terms_of<TW>(wr[i][2], wr[i][3], t[1]);
#pragma unroll
            for (int q = 0; q < TW; ++q) ws[2 * ((q * 2 * KC + (k4 >> 1)) * kPitch + row) + (k4 & 1)] = u32x2{t[0][q], t[1][q]};
        }
        float *bias = reinterpret_cast<float *>(strip_lds + 2 * StripLds<KC, TW>::kUnits) + 32 * buffer;
        if (tid < 32) bias[tid] = br;
    };
    wfetch(c0);

    // ---- the pixels' channels: channel 16 c + 8 half + j ----
    const unsigned ib = P * (unsigned)sizeof(TI);
    const Rsrc rx = resource(static_cast<const TI *>(p.x) + (size_t)n * p.x_stride, (long)K * ib);
    const unsigned in_off = 8u * (unsigned)half * ib + pxc * (unsigned)sizeof(TI);
    u32x4 b[KC][NT][TX];
    load_operands<TI, TX, KC, NT>(rx, in_off, ib, K, b, [&] { wput(0); });
    __syncthreads();

    const unsigned ob = P * (unsigned)sizeof(TO), eb = P * (unsigned)sizeof(TE);
    const Rsrc ro = resource(static_cast<TO *>(p.out) + (size_t)n * p.out_stride, (long)M * ob);
    const Rsrc re = resource(MODE != kForward ? static_cast<const TE *>(p.extra) + (size_t)n * p.extra_stride : nullptr, MODE != kForward ? (long)M * eb : 0);
    // lane l has outputs 32 chunk + 8 (i / 4) + 4 half + i % 4 in element i of its pixels' sums
    auto row_of = [](int i) { return 8 * (i >> 2) + (i & 3); };
    for (int chunk = c0; chunk < c1; ++chunk) {
        const int buffer = (chunk - c0) & 1, left = M - 32 * chunk - 4 * half;
        if (chunk + 1 < c1) wfetch(chunk + 1);
        Raw<TE, NT> ex[16];
        if constexpr (MODE != kForward) {
            const unsigned off = (unsigned)(32 * chunk + 4 * half) * eb + pxc * (unsigned)sizeof(TE);
#pragma unroll
            for (int i = 0; i < 16; ++i) ex[i] = load<TE, NT>(re, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * eb);
        }
        f32x16 acc[NT];
        const float *bias = reinterpret_cast<const float *>(strip_lds + 2 * StripLds<KC, TW>::kUnits) + 32 * buffer;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(bias + 8 * g + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t][4 * g + e] = v[e];
        }
        const u32x4 *ws = strip_lds + buffer * StripLds<KC, TW>::kUnits + half * kPitch + l32;
        // (the next sixteen channels' weights are asked for ahead of these ones' products, and no others: they would take registers)
        u32x4 next[TW];
#pragma unroll
        for (int q = 0; q < TW; ++q) next[q] = ws[q * 2 * KC * kPitch];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            u32x4 a[TW];
#pragma unroll
            for (int q = 0; q < TW; ++q) a[q] = next[q];
            if (c + 1 < KC) {
#pragma unroll
                for (int q = 0; q < TW; ++q) next[q] = ws[(q * 2 * KC + 2 * (c + 1)) * kPitch];
            }
            // small terms first; neighbouring instructions on different sums
#pragma unroll
            for (int qw = TW - 1; qw >= 0; --qw)
#pragma unroll
                for (int qx = TX - 1; qx >= 0; --qx) {
                    if (qw + qx >= kTop) continue;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[qw]), __builtin_bit_cast(bf16x8, b[c][t][qx]), acc[t], 0, 0, 0);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        settle();
        float v[NT * 16];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[16 * t + i] = acc[t][i];
        if constexpr (MODE == kSlope) {
            slopes(p.act, v);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) v[16 * t + i] *= ex[i].value(t);
        } else {
            activate(p.act, v);
            if constexpr (MODE == kResidual) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[16 * t + i] += ex[i].value(t);
            }
        }
        const unsigned off = (unsigned)(32 * chunk + 4 * half) * ob + pxc * (unsigned)sizeof(TO);
#pragma unroll
        for (int i = 0; i < 16; ++i) store<TO, NT>(ro, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * ob, v[i], v[16 * (NT - 1) + i]);
        if (chunk + 1 < c1) wput(buffer ^ 1);
        __syncthreads();
    }
}

// ---- grad_x = W^T ( grad_out act'(b + W x) ) ----
//
// A chunk's 32 outputs gp of a wavefront's pixels, as the first product leaves them in a lane (rows 8 g + 4 half + r of its pixel), are the right operand of
// the second as they lie there, the channels of W^T staged in that order; its sums, grad_x of all K channels, stay in registers over the chunks.  gp never has to
// be read back for it.
template <int KC, int TF, int TB>
struct BackLds {
    static constexpr int kBuffers = KC <= 4 ? 2 : 1;
    static constexpr int kRows = 16 * KC, kPitchT = kRows + 1;
    static constexpr int kForwardUnits = KC * TF * 2 * kPitch, kUnits = kForwardUnits + 2 * TB * 2 * kPitchT;
    static constexpr size_t kBytes = (size_t)kBuffers * (kUnits * 16 + 32 * 4);
};

// TX, TF: terms of x and W in the first product; TG, TB: of gp and W in the second.
template <typename T, int TX, int TF, int TG, int TB, int KC, int NT>
__global__ __launch_bounds__(kThreads, 2) void strip_back_kernel(const BackParams p)
{
    typedef BackLds<KC, TF, TB> L;
    constexpr int kTopF = TX > TF ? TX : TF, kTopB = TG > TB ? TG : TB, KT = KC / 2;
    constexpr int kEach = 128 * KC / kThreads;                                  // runs of four weights of a chunk, of a thread
    constexpr int kUnitsT = L::kRows * 4, kEachT = (kUnitsT + kThreads - 1) / kThreads;  // eights of outputs of a channel, of a thread
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int K = p.K, M = p.M, chunks = (M + 31) / 32;
    const unsigned P = (unsigned)p.P;
    const unsigned tile = p.first + piece_of(blockIdx.x, gridDim.x), n = tile / p.tiles_of_image;
    const unsigned px = (tile - n * p.tiles_of_image) * (128u * NT) + 32u * NT * (unsigned)wave + NT * (unsigned)l32;
    const unsigned pxc = px + NT <= P ? px : P - NT;

    const Rsrc rw = resource(p.w, 4L * K * M);
    const bool four = (K & 3) == 0;
    float wr[kEach][4], tr[kEachT][8], br = 0.f;
    auto wfetch = [&](int chunk) {
        br = p.b != nullptr && tid < 32 && 32 * chunk + tid < M ? p.b[32 * chunk + tid] : 0.f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = tid + i * kThreads;
            load_weights(rw, M, K, K, four, 32 * chunk + u / (4 * KC), 4 * (u % (4 * KC)), wr[i]);
        }
#pragma unroll
        for (int i = 0; i < kEachT; ++i) {
            const int u = tid + i * kThreads, row = u % L::kRows, part = u / L::kRows;   // part: sixteen 2, half of it
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int m = 32 * chunk + 16 * (part >> 1) + 8 * (j >> 2) + 4 * (part & 1) + (j & 3);
                tr[i][j] = __uint_as_float((unsigned)__builtin_amdgcn_raw_buffer_load_b32(rw, (int)(m < M && row < K && part < 4 ? 4u * ((unsigned)m * (unsigned)K + (unsigned)row) : kBeyond), 0, 0));
            }
        }
    };
    auto wput = [&](int buffer) {
        u32x4 *const base = strip_lds + buffer * L::kUnits;
        u32x2 *ws = reinterpret_cast<u32x2 *>(base);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = tid + i * kThreads, row = u / (4 * KC), k4 = u % (4 * KC);
            uint32_t t[2][TF];
            terms_of<TF>(wr[i][0], wr[i][1], t[0]);
            terms_of<TF>(wr[i][2], wr[i][3], t[1]);
#pragma unroll
            for (int q = 0; q < TF; ++q) ws[2 * ((q * 2 * KC + (k4 >> 1)) * kPitch + row) + (k4 & 1)] = u32x2{t[0][q], t[1][q]};
        }
        u32x4 *const ts = base + L::kForwardUnits;
#pragma unroll
        for (int i = 0; i < kEachT; ++i) {
            const int u = tid + i * kThreads, row = u % L::kRows, part = u / L::kRows;
            if (kUnitsT % kThreads != 0 && u >= kUnitsT) break;
            uint32_t t[4][TB];
#pragma unroll
            for (int e = 0; e < 4; ++e) terms_of<TB>(tr[i][2 * e], tr[i][2 * e + 1], t[e]);
#pragma unroll
            for (int q = 0; q < TB; ++q) ts[(((part >> 1) * TB + q) * 2 + (part & 1)) * L::kPitchT + row] = u32x4{t[0][q], t[1][q], t[2][q], t[3][q]};
        }
        if (tid < 32) reinterpret_cast<float *>(strip_lds + L::kBuffers * L::kUnits)[32 * buffer + tid] = br;
    };
    wfetch(0);

    const unsigned ib = P * (unsigned)sizeof(T), fb = P * 4u;
    const unsigned first = pxc * (unsigned)sizeof(T);
    u32x4 b[KC][NT][TX];
    {
        const Rsrc rx = resource(static_cast<const T *>(p.x) + (size_t)n * p.x_stride, (long)K * ib);
        load_operands<T, TX, KC, NT>(rx, 8u * (unsigned)half * ib + first, ib, K, b, [&] { wput(0); });
    }
    __syncthreads();

    const Rsrc rg = resource(static_cast<const T *>(p.grad_out) + (size_t)n * p.g_stride, (long)M * ib);
    const Rsrc rp = resource(p.gp != nullptr ? p.gp + (size_t)n * p.gp_stride : nullptr, p.gp != nullptr ? (long)M * fb : 0);
    auto row_of = [](int i) { return 8 * (i >> 2) + (i & 3); };
    f32x16 gx[KT][NT];
#pragma unroll
    for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) gx[k][t][i] = 0.f;
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int buffer = L::kBuffers == 2 ? chunk & 1 : 0, left = M - 32 * chunk - 4 * half;
        if (chunk + 1 < chunks) wfetch(chunk + 1);
        Raw<T, NT> ex[16];
        {
            const unsigned off = (unsigned)(32 * chunk + 4 * half) * ib + first;
#pragma unroll
            for (int i = 0; i < 16; ++i) ex[i] = load<T, NT>(rg, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * ib);
        }
        f32x16 acc[NT];
        const float *bias = reinterpret_cast<const float *>(strip_lds + L::kBuffers * L::kUnits) + 32 * buffer;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(bias + 8 * g + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t][4 * g + e] = v[e];
        }
        const u32x4 *ws = strip_lds + buffer * L::kUnits + half * kPitch + l32;
        u32x4 next[TF];
#pragma unroll
        for (int q = 0; q < TF; ++q) next[q] = ws[q * 2 * KC * kPitch];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            u32x4 a[TF];
#pragma unroll
            for (int q = 0; q < TF; ++q) a[q] = next[q];
            if (c + 1 < KC) {
#pragma unroll
                for (int q = 0; q < TF; ++q) next[q] = ws[(q * 2 * KC + 2 * (c + 1)) * kPitch];
            }
#pragma unroll
            for (int qw = TF - 1; qw >= 0; --qw)
#pragma unroll
                for (int qx = TX - 1; qx >= 0; --qx) {
                    if (qw + qx >= kTopF) continue;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[qw]), __builtin_bit_cast(bf16x8, b[c][t][qx]), acc[t], 0, 0, 0);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        settle();
        float v[NT * 16];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[16 * t + i] = acc[t][i];
        slopes(p.act, v);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[16 * t + i] *= ex[i].value(t);
        if (p.gp != nullptr) {
            const unsigned off = (unsigned)(32 * chunk + 4 * half) * fb + pxc * 4u;
#pragma unroll
            for (int i = 0; i < 16; ++i) store<float, NT>(rp, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * fb, v[i], v[16 * (NT - 1) + i]);
        }
        const u32x4 *ts = strip_lds + buffer * L::kUnits + L::kForwardUnits + half * L::kPitchT + l32;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            u32x4 g[NT][TG];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t q[TG];
                    terms_of<TG>(v[16 * t + 8 * c + 2 * e], v[16 * t + 8 * c + 2 * e + 1], q);
#pragma unroll
                    for (int i = 0; i < TG; ++i) g[t][i][e] = q[i];
                }
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                u32x4 a[TB];
#pragma unroll
                for (int q = 0; q < TB; ++q) a[q] = ts[(c * TB + q) * 2 * L::kPitchT + 32 * k];
#pragma unroll
                for (int qw = TB - 1; qw >= 0; --qw)
#pragma unroll
                    for (int qg = TG - 1; qg >= 0; --qg) {
                        if (qw + qg >= kTopB) continue;
#pragma unroll
                        for (int t = 0; t < NT; ++t)
                            gx[k][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[qw]), __builtin_bit_cast(bf16x8, g[t][qg]), gx[k][t], 0, 0, 0);
                    }
            }
        }
        if (chunk + 1 < chunks) {
            if constexpr (L::kBuffers == 1) __syncthreads();   // everyone has finished with this chunk's weights
            wput(L::kBuffers == 2 ? buffer ^ 1 : 0);
        }
        __syncthreads();
    }
    settle();
    const Rsrc ro = resource(static_cast<T *>(p.grad_x) + (size_t)n * p.gx_stride, (long)K * ib);
#pragma unroll
    for (int k = 0; k < KT; ++k) {
        const int left = K - 32 * k - 4 * half;
        const unsigned off = (unsigned)(32 * k + 4 * half) * ib + first;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v0 = gx[k][0][i], v1 = gx[k][NT - 1][i];
            store<T, NT>(ro, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * ib, v0, v1);
        }
    }
}

template <typename TI, typename TO, typename TE, int TX, int TW, int KC, int NT, bool TRANS, int MODE>
hipError_t launch_as(const ProductParams &q, long N, hipStream_t s)
{
    const long tiles = (q.P + 128 * NT - 1) / (128 * NT), all = tiles * N;
    const int chunks = (q.M + 31) / 32;
    // The outputs are shared out over blocks where pixels alone leave compute units without the blocks they hold, or the last round of blocks short:
    // the fewest chunks on the longest way, a block's beginning and its reading of x counted as two.
    constexpr long kPlaces = kCus * strip_blocks(4 * KC * NT * TX, MODE != kForward || TRANS);
    long parts = 1, best = 0;
    for (int k = 1; k <= chunks; ++k) {
        const long way = (all * k + kPlaces - 1) / kPlaces * ((chunks + k - 1) / k + 2);
        if (best == 0 || way < best) parts = k, best = way;
    }
    StripParams p;
    static_cast<ProductParams &>(p) = q;
    p.each = (int)((chunks + parts - 1) / parts);
    p.parts = (unsigned)((chunks + p.each - 1) / p.each);
    p.tiles_of_image = (unsigned)tiles;
    const auto kernel = strip_kernel<TI, TO, TE, TX, TW, KC, NT, TRANS, MODE>;
    constexpr size_t lds = StripLds<KC, TW>::kBytes;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    return in_launches(all * p.parts, kThreads, [&](long first, unsigned blocks) {
        p.first = (unsigned)first;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), lds, s, p);
        return hipGetLastError();
    });
}

// Two pixels a lane where the registers hold their channels and every compute unit has two blocks, of a third of the outputs at least.
template <typename TI, typename TO, typename TE, int TX, int TW, int KC, bool TRANS, int MODE>
hipError_t launch_nt(const ProductParams &p, long N, hipStream_t s)
{
    if constexpr (KC * TX <= 12 && !(KC == 12 && MODE == kResidual))
        if (p.P >= 2 && N * ((p.P + 255) / 256) * std::min(3, (p.M + 31) / 32) >= 2 * kCus) return launch_as<TI, TO, TE, TX, TW, KC, 2, TRANS, MODE>(p, N, s);
    return launch_as<TI, TO, TE, TX, TW, KC, 1, TRANS, MODE>(p, N, s);
}
template <typename TI, typename TO, typename TE, int TX, int TW, bool TRANS, int MODE>
hipError_t launch_kc(const ProductParams &p, long N, hipStream_t s)
{
    const int k = (p.K + 15) / 16;
    if (k <= 2) return launch_nt<TI, TO, TE, TX, TW, 2, TRANS, MODE>(p, N, s);
    if (k <= 4) return launch_nt<TI, TO, TE, TX, TW, 4, TRANS, MODE>(p, N, s);
    if (k <= 8) return launch_nt<TI, TO, TE, TX, TW, 8, TRANS, MODE>(p, N, s);
    return launch_nt<TI, TO, TE, TX, TW, TX == 3 ? 10 : 12, TRANS, MODE>(p, N, s);
}

template <typename T, int TX, int TF, int TG, int TB, int KC, int NT>
hipError_t launch_back_as(BackParams p, long N, hipStream_t s)
{
    p.tiles_of_image = (unsigned)((p.P + 128 * NT - 1) / (128 * NT));
    constexpr size_t lds = BackLds<KC, TF, TB>::kBytes;
    static_assert(lds <= 64 * 1024, "");
    return in_launches(p.tiles_of_image * N, kThreads, [&](long first, unsigned blocks) {
        p.first = (unsigned)first;
        hipLaunchKernelGGL((strip_back_kernel<T, TX, TF, TG, TB, KC, NT>), dim3(blocks), dim3(kThreads), lds, s, p);
        return hipGetLastError();
    });
}
// what the registers hold, with bf16 storage and with fp32
constexpr int kMostK[2] = {192, 160}, kBackMostK[2] = {128, 64};

}  // namespace

bool back_fits(bool f32, int K, int M, long P, long N)
{
    if (K > kBackMostK[f32] || (size_t)std::max(K, M) * P * 4 >= kMostImage || P > kMostPlane || !(N == 1 || P >= 96)) return false;
    // (a block goes through all outputs: few pixels are better shared out over two launches.  5 x 50 x 61, 96 to 45, fp32: two launches 14.0 us, one 15.7)
    return N * ((P + 127) / 128) >= kCus;
}

hipError_t launch_back(bool f32, const BackParams &p, long N, hipStream_t s)
{
    const int k = (p.K + 15) / 16;
    if (f32) {
        if (k <= 2) return launch_back_as<float, 3, 3, 3, 3, 2, 1>(p, N, s);
        return launch_back_as<float, 3, 3, 3, 3, 4, 1>(p, N, s);
    }
    const bool two = p.P >= 2 && N * ((p.P + 255) / 256) >= 2 * kCus;
    if (k <= 2) return two ? launch_back_as<bf16s, 1, 3, 2, 2, 2, 2>(p, N, s) : launch_back_as<bf16s, 1, 3, 2, 2, 2, 1>(p, N, s);
    if (k <= 4) return two ? launch_back_as<bf16s, 1, 3, 2, 2, 4, 2>(p, N, s) : launch_back_as<bf16s, 1, 3, 2, 2, 4, 1>(p, N, s);
    return launch_back_as<bf16s, 1, 3, 2, 2, 8, 1>(p, N, s);
}

bool strip_fits(int kind, const ProductParams &p, long N)
{
    const size_t in = kind == kForwardBf16 || kind == kSlopeBf16 || kind == kBackBf16 ? 2 : 4, out = kind == kForwardBf16 || kind == kBackBf16 || kind == kBackGp ? 2 : 4;
    // (the slope's other input is no wider than what it writes)
    if (p.K > kMostK[kind == kForwardF32 || kind == kSlopeF32 || kind == kBackF32] || (size_t)p.K * p.P * in >= kMostImage || (size_t)p.M * p.P * out >= kMostImage || p.P > kMostPlane) return false;
    // small images fill too little of a block's pixels
    return N == 1 || p.P >= 96;
}

hipError_t launch_strip(int kind, const ProductParams &p, long N, hipStream_t s)
{
    switch (kind) {
    case kForwardF32: return p.extra != nullptr ? launch_kc<float, float, float, 3, 3, false, kResidual>(p, N, s) : launch_kc<float, float, float, 3, 3, false, kForward>(p, N, s);
    case kForwardBf16: return p.extra != nullptr ? launch_kc<bf16s, bf16s, bf16s, 1, 2, false, kResidual>(p, N, s) : launch_kc<bf16s, bf16s, bf16s, 1, 2, false, kForward>(p, N, s);
    case kSlopeF32: return launch_kc<float, float, float, 3, 3, false, kSlope>(p, N, s);
    case kSlopeBf16: return launch_kc<bf16s, float, bf16s, 1, 3, false, kSlope>(p, N, s);
    case kBackF32: return launch_kc<float, float, float, 3, 3, true, kForward>(p, N, s);
    case kBackBf16: return launch_kc<bf16s, bf16s, bf16s, 1, 2, true, kForward>(p, N, s);
    case kBackGp: return launch_kc<float, bf16s, bf16s, 2, 2, true, kForward>(p, N, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace esc
