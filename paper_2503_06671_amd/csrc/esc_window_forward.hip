// Window attention, forward: out = softmax(scale q.k + bias) v over the keys of a window, in one pass over the keys with a running
// maximum and sum.
//
// A wavefront has 64 queries (two tiles of 32), a block up to four wavefronts, and goes through the window's keys TK at a time,
// staged in LDS.  Scores are formed transposed (keys down, queries across: S^T = K Q^T), so that a lane holds 16 keys of ONE query:
// maximum and sum need no exchange but between the two halves of the wavefront, and the exponentials are, as they lie in registers,
// the right operand of the next product O^T = V^T P^T.  The bias is the product's starting value.
#include "esc_window.hpp"

namespace esc {
namespace {

// SAVE: the backward pass follows.  Its delta = sum over the channels of out * dout stands for sum over the keys of p * dp, and what it is off goes into every
// term of the bias' gradient, an fp32 result: with bf16 storage the exponentials are then two bf16 terms (with one the bias' gradient
// was 9e-5 off, with two 4e-7).
template <typename T, int DP, bool SAVE>
__global__ __launch_bounds__(256) void window_forward_kernel(const WindowParams p)
{
    using G = WinGeom<T, DP>;
    extern __shared__ __align__(16) char lds[];
    char *rm = lds, *cm = rm + G::RM_BYTES;
    int *off = reinterpret_cast<int *>(cm + G::CM_BYTES);
    uint8_t *bits = reinterpret_cast<uint8_t *>(off + G::TK / 4);
    float *table = reinterpret_cast<float *>(bits + G::TK / 4);

    const int unit = unit_of(p.units);
    if (unit < 0) return;
    const int block = unit % p.blocks, head = unit / p.blocks % p.heads, wi = unit / p.blocks / p.heads;
    const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
    const int q0 = block * p.waves * kWinWaveTokens;
    if (q0 >= w.L) return;
    const int centre = (p.wh - 1) * p.tw + p.ww - 1;
    const TableRange range = table_range(q0, min(q0 + p.waves * kWinWaveTokens, w.L), w.h, w.wp, p.tw, centre, -1);
    stage_table(p, table, range, head);

    const long hw = (long)p.H * p.W;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int kvh = head / (p.heads / p.kv_heads);
    const T *q = static_cast<const T *>(p.q) + w.n * p.qs + head * (long)p.d * hw;
    const T *k = static_cast<const T *>(p.k) + w.n * p.ks + kvh * (long)p.d * hw;
    const T *v = static_cast<const T *>(p.v) + w.n * p.vs + kvh * (long)p.d * hw;

    Fragment<T, DP> own[2];
    long pixel[2];
    bool ok[2], there[2];
    int place[2];  // in the table, of the offset to the key that has off = 0
    float top[2], sum[2];
    wf32x16 acc[2][G::DT];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int t = q0 + wave * kWinWaveTokens + u * 32 + (lane & 31), tc = min(t, w.L - 1);
        const int y = tc / w.wp, x = tc - y * w.wp;
        there[u] = t < w.L && x < w.w;
        ok[u] = there[u] && seen(p, w, y, x);
        pixel[u] = (long)(w.y0 + y) * p.W + w.x0 + x;
        place[u] = centre - (y * p.tw + x) - range.base;
        own[u] = own_fragment<T, DP>(p, q + pixel[u], ok[u]);
        top[u] = -__builtin_inff(), sum[u] = 0.f;
#pragma unroll
        for (int b = 0; b < G::DT; ++b) acc[u][b] = wf32x16{};
    }
    const bool busy = q0 + wave * kWinWaveTokens < w.L;  // (the same for the wavefront)

    for (int t0 = 0; t0 < w.L; t0 += G::TK) {
        __syncthreads();
        stage<T, DP, true, false>(p, w, k, t0, rm, nullptr, threadIdx.x, blockDim.x);
        stage<T, DP, false, true>(p, w, v, t0, nullptr, cm, threadIdx.x, blockDim.x);
        stage_tokens<G::TK>(p, w, t0, off, bits);
        __syncthreads();
        if (!busy) continue;
        for (int tile = 0; tile < G::TK / 32 && t0 + tile * 32 < w.L; ++tile) {
            const wu32x2 nibbles = *reinterpret_cast<const wu32x2 *>(bits + tile * 8);
            const bool whole = __builtin_amdgcn_readfirstlane((int)((nibbles.x & nibbles.y) == 0x0f0f0f0fu));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                wf32x16 s;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const float *from = table + place[u] + off[tile * 8 + 2 * a + half];
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[4 * a + j] = from[j];
                }
                s = score<T, DP>(rm, tile, own[u], s);
                if (!whole) {
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const uint32_t b = (a < 2 ? nibbles.x : nibbles.y) >> (16 * (a & 1) + 8 * half);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[4 * a + j] = (b >> j & 1) != 0 ? s[4 * a + j] : -__builtin_inff();
                    }
                }
                float m = s[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
                m = fmaxf(m, other_half(m));
                const float old = top[u], next = fmaxf(old, m), from = next == -__builtin_inff() ? 0.f : next;
                const float shift = from * p.log2_scale;
                float shrink;
                if (__builtin_expect(!__any(__builtin_fabsf(shift) > kLargeShift), 1)) {
                    shrink = old == -__builtin_inff() ? 0.f : exp2_of(old * p.log2_scale - shift);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], p.log2_scale, -shift);
                } else {
                    shrink = exp2_of((old - from) * p.log2_scale);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = (s[i] - from) * p.log2_scale;
                }
                top[u] = next;
                float add = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[i] = exp2_of(s[i]);
                    add += s[i];
                }
                sum[u] = __builtin_fmaf(sum[u], shrink, add);
#pragma unroll
                for (int b = 0; b < G::DT; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[u][b][i] *= shrink;
                accumulate<T, DP>(cm, tile, pack<G::F32 ? 3 : SAVE ? 2 : 1>(s), acc[u]);
            }
        }
    }
    if (!busy) return;
    T *out = static_cast<T *>(p.out) + ((long)w.n * p.heads + head) * p.d * hw;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const float all = sum[u] + other_half(sum[u]);
        if (!there[u]) continue;
        const bool some = ok[u] && !(all == 0.f);
        const float over = some ? 1.f / all : 0.f;
        const long pix = ((long)w.n * p.heads + head) * hw + pixel[u];
        if (SAVE && half == 0) {
            p.top[pix] = some && top[u] != -__builtin_inff() ? top[u] : 0.f;
            p.log_sum[pix] = some ? __builtin_log2f(all) : __builtin_inff();
        }
#pragma unroll
        for (int b = 0; b < G::DT; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = b * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (c < p.d) {
                    const float o = some ? acc[u][b][i] * over : 0.f;
                    const T r = narrow<T>(o);
                    out[c * hw + pixel[u]] = r;
                    if constexpr (SAVE && !G::F32) static_cast<T *>(p.rest)[((long)w.n * p.heads + head) * p.d * hw + c * hw + pixel[u]] = to_bf16(o - widen(r));
                }
            }
    }
}

template <typename T, int DP>
size_t lds_of(int len)
{
    using G = WinGeom<T, DP>;
    return G::RM_BYTES + G::CM_BYTES + (G::TK / 4) * 5 + (size_t)len * 4;
}

template <typename T, int DP, bool SAVE>
hipError_t launch_one(const WindowParams &p, hipStream_t s)
{
    const size_t lds = lds_of<T, DP>(p.len);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&window_forward_kernel<T, DP, SAVE>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((window_forward_kernel<T, DP, SAVE>), dim3((unsigned)((p.units + 7) / 8 * 8)), dim3(64 * p.waves), lds, s, p);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch(const WindowParams &p, hipStream_t s)
{
    return p.top != nullptr ? launch_one<T, DP, true>(p, s) : launch_one<T, DP, false>(p, s);
}

}  // namespace

size_t window_forward_lds(bool f32, int dp, int len)
{
    if (f32) return dp == 16 ? lds_of<float, 16>(len) : dp == 32 ? lds_of<float, 32>(len) : lds_of<float, 64>(len);
    return dp == 16 ? lds_of<uint16_t, 16>(len) : dp == 32 ? lds_of<uint16_t, 32>(len) : lds_of<uint16_t, 64>(len);
}

hipError_t launch_window_forward(const WindowParams &p, bool f32, int dp, hipStream_t s)
{
    if (f32) return dp == 16 ? launch<float, 16>(p, s) : dp == 32 ? launch<float, 32>(p, s) : launch<float, 64>(p, s);
    return dp == 16 ? launch<uint16_t, 16>(p, s) : dp == 32 ? launch<uint16_t, 32>(p, s) : launch<uint16_t, 64>(p, s);
}

}  // namespace esc
