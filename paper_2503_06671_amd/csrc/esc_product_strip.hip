// Point-wise products whose input channels are few enough to stay in registers (esc_product.hpp).
//
// A wavefront owns 32 NT pixels and has all K input channels of them in registers as the right operand of v_mfma_f32_32x32x16_bf16: a lane holds
// eight consecutive channels of its pixel for each sixteen, as eight loads of channel rows bring them (32 lanes on a run of 32 NT pixels), split into
// terms once.  The weights pass LDS in chunks of 32 outputs, two buffers, one barrier a chunk; behind a chunk's products stand its
// activation, residual and stores, while other wavefronts multiply.  x is read once where one block takes all outputs.
#include "esc_product.hpp"

#include <algorithm>
#include <type_traits>

namespace esc {
namespace {

typedef __amdgpu_buffer_rsrc_t Rsrc;
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kRawBuffer = 0x00020000;     // raw buffer (no stride, no swizzle), 32-bit data format
constexpr unsigned kBeyond = 0x80000000u;  // an offset beyond every resource (an image of a tensor is < 2 GiB)
constexpr size_t kMostImage = (size_t)1 << 31;

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

// Weights of a chunk in LDS: units of eight consecutive channels of one output, [channels / 16][term][half of the sixteen][output], halves a unit
// further apart than outputs take (other banks for a thread's neighbours, who write other eighths of the same output).
constexpr int kPitch = 33;

template <int KC, int TW>
struct StripLds {
    static constexpr int kUnits = KC * TW * 2 * kPitch;
    static constexpr size_t kBytes = (size_t)2 * kUnits * 16 + 2 * 32 * 4;
};
extern __shared__ __align__(16) u32x4 strip_lds[];

struct StripParams : ProductParams {
    int each;   // chunks of 32 outputs a block
    unsigned parts;
    unsigned tiles_of_image;
};

template <typename TI, typename TO, typename TE, int TX, int TW, int KC, int NT, bool TRANS, int MODE>
__global__ __launch_bounds__(kThreads, 2) void strip_kernel(const StripParams p)
{
    constexpr int kTop = TX > TW ? TX : TW;      // products of terms whose orders add up to less
    constexpr int kUnits = 64 * KC, kEach = (kUnits + kThreads - 1) / kThreads;  // runs of eight weights of a chunk, of a thread
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int K = p.K, M = p.M;
    const unsigned P = (unsigned)p.P;
    const unsigned piece = piece_of(blockIdx.x, gridDim.x), tile = piece / p.parts, n = tile / p.tiles_of_image;
    const int c0 = (int)(piece - tile * p.parts) * p.each, c1 = min(c0 + p.each, (M + 31) / 32);
    const unsigned px = (tile - n * p.tiles_of_image) * (128u * NT) + 32u * NT * (unsigned)wave + NT * (unsigned)l32;
    // (a lane whose pixels reach beyond the plane takes the plane's last ones again: the same bits are stored)
    const unsigned pxc = px + NT <= P ? px : P - NT;

    // ---- weights ----
    struct __attribute__((packed, aligned(4))) W4 {
        float v[4];
    };
    const bool k8 = (K & 7) == 0;   // a run of eight is inside or outside as a whole
    float wr[kEach][8];
    float br = 0.f;
    auto wfetch = [&](int chunk) {
        br = p.b != nullptr && tid < 32 ? p.b[min(32 * chunk + tid, M - 1)] : 0.f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = tid + i * kThreads;
            const int row = TRANS ? u & 31 : u / (2 * KC), e8 = TRANS ? u >> 5 : u % (2 * KC);
            const int m = 32 * chunk + row, k = 8 * e8;
            if constexpr (TRANS) {
                const float *s = p.w + min(m, M - 1);
#pragma unroll
                for (int e = 0; e < 8; ++e) wr[i][e] = s[(size_t)min(k + e, K - 1) * p.w_ld];
            } else if (k8) {
                const float *s = p.w + (m < M && k < K ? (size_t)m * p.w_ld + k : 0);
                const W4 a = *reinterpret_cast<const W4 *>(s), b = *reinterpret_cast<const W4 *>(s + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) wr[i][e] = a.v[e], wr[i][4 + e] = b.v[e];
            } else {
                const float *s = p.w + (size_t)min(m, M - 1) * p.w_ld;
#pragma unroll
                for (int e = 0; e < 8; ++e) wr[i][e] = s[min(k + e, K - 1)];
            }
        }
    };
    auto wput = [&](int chunk, int buffer) {
        u32x4 *ws = strip_lds + buffer * StripLds<KC, TW>::kUnits;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int u = tid + i * kThreads;
            if (kUnits % kThreads != 0 && u >= kUnits) break;
            const int row = TRANS ? u & 31 : u / (2 * KC), e8 = TRANS ? u >> 5 : u % (2 * KC);
            const int in = 32 * chunk + row < M ? K - 8 * e8 : 0;   // how many of the eight there are
            uint32_t t[4][TW];
#pragma unroll
            for (int e = 0; e < 4; ++e) terms_of<TW>(2 * e < in ? wr[i][2 * e] : 0.f, 2 * e + 1 < in ? wr[i][2 * e + 1] : 0.f, t[e]);
#pragma unroll
            for (int q = 0; q < TW; ++q) ws[(((e8 >> 1) * TW + q) * 2 + (e8 & 1)) * kPitch + row] = u32x4{t[0][q], t[1][q], t[2][q], t[3][q]};
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
    {
        Raw<TI, NT> r[KC][8];
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = 16 * c + 8 * half + j < K;
                r[c][j] = load<TI, NT>(rx, in ? in_off : kBeyond, 16 * c + j < K ? (unsigned)(16 * c + j) * ib : 0u);
            }
        wput(c0, 0);
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (!kWide<TI> && TX == 1) {
                    b[c][0][0][e] = __builtin_amdgcn_perm(r[c][2 * e + 1].w[0], r[c][2 * e].w[0], 0x05040100u);
                    if constexpr (NT == 2) b[c][1][0][e] = __builtin_amdgcn_perm(r[c][2 * e + 1].w[0], r[c][2 * e].w[0], 0x07060302u);
                } else {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        uint32_t q[TX];
                        terms_of<TX>(r[c][2 * e].value(t), r[c][2 * e + 1].value(t), q);
#pragma unroll
                        for (int i = 0; i < TX; ++i) b[c][t][i][e] = q[i];
                    }
                }
            }
    }
    __syncthreads();

    const unsigned ob = P * (unsigned)sizeof(TO), eb = P * (unsigned)sizeof(TE);
    const Rsrc ro = resource(static_cast<TO *>(p.out) + (size_t)n * p.out_stride, (long)M * ob);
    const Rsrc re = resource(p.extra != nullptr ? static_cast<const TE *>(p.extra) + (size_t)n * p.extra_stride : nullptr, p.extra != nullptr ? (long)M * eb : 0);
    // lane l has outputs 32 chunk + 8 (i / 4) + 4 half + i % 4 in element i of its pixels' sums
    auto row_of = [](int i) { return 8 * (i >> 2) + (i & 3); };
    for (int chunk = c0; chunk < c1; ++chunk) {
        const int buffer = (chunk - c0) & 1, left = M - 32 * chunk - 4 * half;
        if (chunk + 1 < c1) wfetch(chunk + 1);
        Raw<TE, NT> ex[16];
        if (p.extra != nullptr) {
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
        for (int q = 0; q < TW; ++q) next[q] = ws[q * 2 * kPitch];
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            u32x4 a[TW];
#pragma unroll
            for (int q = 0; q < TW; ++q) a[q] = next[q];
            if (c + 1 < KC) {
#pragma unroll
                for (int q = 0; q < TW; ++q) next[q] = ws[((c + 1) * TW + q) * 2 * kPitch];
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
            if (p.extra != nullptr) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[16 * t + i] += ex[i].value(t);
            }
        }
        const unsigned off = (unsigned)(32 * chunk + 4 * half) * ob + pxc * (unsigned)sizeof(TO);
#pragma unroll
        for (int i = 0; i < 16; ++i) store<TO, NT>(ro, row_of(i) < left ? off : kBeyond, (unsigned)row_of(i) * ob, v[i], v[16 * (NT - 1) + i]);
        if (chunk + 1 < c1) wput(chunk + 1, buffer ^ 1);
        __syncthreads();
    }
}

template <typename TI, typename TO, typename TE, int TX, int TW, int KC, int NT, bool TRANS, int MODE>
hipError_t launch_as(const ProductParams &q, long N, hipStream_t s)
{
    const long tiles = (q.P + 128 * NT - 1) / (128 * NT), all = tiles * N;
    const int chunks = (q.M + 31) / 32;
    // where pixels alone do not give each compute unit two blocks, the outputs are shared out too
    const long parts = std::max<long>(1, std::min<long>(chunks, (2 * kCus + all - 1) / all));
    StripParams p;
    static_cast<ProductParams &>(p) = q;
    p.each = (int)((chunks + parts - 1) / parts);
    p.parts = (unsigned)((chunks + p.each - 1) / p.each);
    p.tiles_of_image = (unsigned)tiles;
    if (all * p.parts >= (1L << 31)) return hipErrorInvalidValue;
    const auto kernel = strip_kernel<TI, TO, TE, TX, TW, KC, NT, TRANS, MODE>;
    constexpr size_t lds = StripLds<KC, TW>::kBytes;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)(all * p.parts)), dim3(kThreads), lds, s, p);
    return hipGetLastError();
}

// Two pixels a lane where the registers hold their channels and every compute unit has two blocks.
template <typename TI, typename TO, typename TE, int TX, int TW, int KC, bool TRANS, int MODE>
hipError_t launch_nt(const ProductParams &p, long N, hipStream_t s)
{
    if constexpr (KC * TX <= 16)
        if (p.P >= 2 && N * ((p.P + 255) / 256) >= 2 * kCus) return launch_as<TI, TO, TE, TX, TW, KC, 2, TRANS, MODE>(p, N, s);
    return launch_as<TI, TO, TE, TX, TW, KC, 1, TRANS, MODE>(p, N, s);
}
template <typename TI, typename TO, typename TE, int TX, int TW, bool TRANS, int MODE>
hipError_t launch_kc(const ProductParams &p, long N, hipStream_t s)
{
    const int k = (p.K + 15) / 16;
    if (k <= 2) return launch_nt<TI, TO, TE, TX, TW, 2, TRANS, MODE>(p, N, s);
    if (k <= 4) return launch_nt<TI, TO, TE, TX, TW, 4, TRANS, MODE>(p, N, s);
    if (k <= 8) return launch_nt<TI, TO, TE, TX, TW, 8, TRANS, MODE>(p, N, s);
    return launch_nt<TI, TO, TE, TX, TW, 12, TRANS, MODE>(p, N, s);
}

}  // namespace

bool strip_fits(int kind, const ProductParams &p, long N)
{
    const size_t in = kind == kForwardBf16 || kind == kSlopeBf16 || kind == kBackBf16 ? 2 : 4, out = kind == kForwardBf16 || kind == kBackBf16 || kind == kBackGp ? 2 : 4;
    // (the slope's other input is no wider than what it writes)
    if (p.K > 192 || (size_t)p.K * p.P * in >= kMostImage || (size_t)p.M * p.P * out >= kMostImage) return false;
    // small images fill too little of a block's pixels
    return N == 1 || p.P >= 96;
}

hipError_t launch_strip(int kind, const ProductParams &p, long N, hipStream_t s)
{
    switch (kind) {
    case kForwardF32: return launch_kc<float, float, float, 3, 3, false, kForward>(p, N, s);
    case kForwardBf16: return launch_kc<bf16s, bf16s, bf16s, 1, 2, false, kForward>(p, N, s);
    case kSlopeF32: return launch_kc<float, float, float, 3, 3, false, kSlope>(p, N, s);
    case kSlopeBf16: return launch_kc<bf16s, float, bf16s, 1, 3, false, kSlope>(p, N, s);
    case kBackF32: return launch_kc<float, float, float, 3, 3, true, kForward>(p, N, s);
    case kBackBf16: return launch_kc<bf16s, bf16s, bf16s, 1, 2, true, kForward>(p, N, s);
    case kBackGp: return launch_kc<float, bf16s, bf16s, 2, 2, true, kForward>(p, N, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace esc
