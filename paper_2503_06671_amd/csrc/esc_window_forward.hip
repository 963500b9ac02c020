// Window attention, forward: out = softmax(scale q.k + bias) v over the keys of a window, in one pass over the keys with a running
// maximum and sum.
//
// A wavefront has one or two tiles of 32 queries, a block up to eight wavefronts, and goes through the window's keys TK at a time,
// staged in LDS in two buffers.  Scores are formed transposed (keys down, queries across: S^T = K Q^T), so that a lane holds 16 keys of ONE query:
// maximum and sum need no exchange but between the two halves of the wavefront, and the exponentials are, as they lie in registers,
// the right operand of the next product O^T = V^T P^T.  The bias is the product's starting value.  The running maximum is followed only
// where a score exceeds it by more than kSlack: the exponentials then reach 2^kSlack, and most tiles rescale nothing.
//
// Calls with fewer tiles than the chip has room for take one tile a wavefront and let up to four wavefronts (no more than a chunk has tiles) share a
// tile's keys; their sums are joined in LDS at the end.
//
// What bounds it: the issue of vector instructions (16 exponentials and as many multiplications, maxima, sums and conversions for a lane of a tile of
// 32 x 32 pairs, beside three to six products in bf16) where there are wavefronts enough: 87 % of the slots for 64 maps of 64 x 64, 78 % in windows of 13; the
// products' share of the matrix units' time is 12 to 24 % with bf16 storage, 32 % with fp32.  At 180 x 320 the two rounds of blocks, the second of them
// short, leave 60 % (bf16) and 49 % (fp32) of the slots used.  Measured, one MI355X: 180 x 320, 4 heads of 16, windows of 32 x 32: bf16 88 us, fp32 151 us;
// 6 heads of 32, windows of 48, bf16: 298 us; 3 x 339 x 511, 6 heads of 8 that share 2 keys, windows of 13, bf16: 350 us; a map of 64 x 64 alone, fp32: 29 us.
#include "esc_window.hpp"

namespace esc {
namespace {

// What exponentials relative to the score `old` are times, relative to `next`.
__device__ __forceinline__ float rescale(const WindowParams &p, float old, float next)
{
    return exp2_of(__builtin_fmaf(old - next, p.log2_scale, shift_rest(next, p.log2_scale) - shift_rest(old, p.log2_scale)));
}

// The exponentials in the second product, with bf16 storage: two bf16 terms, which leave the result off by its own rounding alone (0.0017 of its norm;
// with one term 0.0023, for 71 us instead of 88 at 180 x 320, windows of 32, and 245 instead of 298 in windows of 48).
// SAVE: the backward pass follows.  Its delta = sum over the channels of out * dout stands for sum over the keys of p * dp, and what it is off goes into every
// term of the bias' gradient, an fp32 result: with bf16 storage the exponentials are then three bf16 terms, and what rounding took from
// the result is kept (off by, of the bias' gradient's norm, for windows of 2 to 60 tokens: 1e-4 with one term, 0.5e-6 to 3.6e-6 with two, 0.1e-6
// to 0.4e-6 with three, which take 438 us where two take 390, for 64 maps of 64 x 64).
template <typename T, int DP, int U, bool SAVE>
__global__ __launch_bounds__(512) void window_forward_kernel(const WindowParams p)
{
    using G = WinGeom<T, DP>;
    using S = Stager<T, DP, true, false, false, true>;  // keys by tokens, values by channels
    constexpr bool SUM_ROW = DP == 16;                  // the exponentials' sum is row 16 of the product
    constexpr int VT = G::F32 || SAVE ? 3 : 2;
    extern __shared__ __align__(16) char lds[];
    float *table = reinterpret_cast<float *>(lds);  // (first: its reads' addresses are then sums of two terms and a constant)
    char *const staged = lds + (size_t)p.len * 4;

    const int unit = unit_of(p);
    if (unit < 0) return;
    const int block = unit % p.blocks, head = unit / p.blocks % p.heads, wi = unit / p.blocks / p.heads;
    const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
    const int queries = p.owners / p.ksplit * (U * 32), q0 = block * queries;
    if (q0 >= w.L) return;
    const TableRange range = table_range(w, q0, min(q0 + queries, w.L), -1);

    const long hw = (long)p.H * p.W;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int share = wave % p.ksplit, wq0 = q0 + wave / p.ksplit * (U * 32);
    const int kvh = head / (p.heads / p.kv_heads);
    const T *q = static_cast<const T *>(p.q) + w.n * p.qs + head * (long)p.d * hw;
    const T *k = static_cast<const T *>(p.k) + w.n * p.ks + kvh * (long)p.d * hw;
    const T *v = static_cast<const T *>(p.v) + w.n * p.vs + kvh * (long)p.d * hw;

    S stager;
    stager.fetch(p, w, k, v, 0);
    Fragment<T, DP> own[U];
    int pixel[U], place[U];  // place: in the table, in bytes, of the offset to the key that has off = 0
    bool ok[U], there[U];
    float top[U], limit[U], shift[U], sum[U];
    bool far = false;  // (uniform) a shift is large
    wf32x16 acc[U][G::DT];
    {
        OwnValues<T, DP> values[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const OwnToken own_token(p, w, wq0 + u * 32 + (lane & 31));
            there[u] = own_token.there, pixel[u] = own_token.pixel, ok[u] = own_token.ok(p);
            place[u] = 4 * (w.centre - own_token.off - range.base);
            values[u].fetch(p, q, pixel[u]);
        }
        stage_table<false>(p, w, table, range, head);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            values[u].clean(p, ok[u]);
            own[u] = fragment_of(values[u]);
            top[u] = limit[u] = -__builtin_inff(), shift[u] = sum[u] = 0.f;
#pragma unroll
            for (int b = 0; b < G::DT; ++b) acc[u][b] = wf32x16{};
        }
    }
    S::clear(p, staged);
    if (p.buffers == 2) S::clear(p, staged + S::BYTES);
    __syncthreads();
    S::ones(staged + S::CM1_AT);
    if (p.buffers == 2) S::ones(staged + S::BYTES + S::CM1_AT);
    stager.write(p, w, k, v, 0, staged);
    __syncthreads();
    const float slack = kSlack / p.log2_scale;
    const bool busy = wave < p.owners && wq0 < w.L;

    for (int t0 = 0, turn = 0; t0 < w.L; t0 += G::TK, turn ^= 1) {
        const bool more = t0 + G::TK < w.L;
        if (more) stager.fetch(p, w, k, v, t0 + G::TK);
        const char *buf = staged + turn * S::BYTES;
        const int *off = reinterpret_cast<const int *>(buf + S::OFF_AT);
        if (busy)
#pragma unroll  // (in a loop the compiler waits for the next chunk's loads first)
            for (int tile = 0; tile < G::TK / 32; ++tile) {
                if (t0 + tile * 32 >= w.L || (tile & (p.ksplit - 1)) != share) continue;
                const wu32x4 bits = *reinterpret_cast<const wu32x4 *>(buf + S::BITS_AT + tile * 16);
                const bool whole = all_take_part(bits);
                wi32x2 key[4];
#pragma unroll
                for (int a = 0; a < 4; ++a) key[a] = *reinterpret_cast<const wi32x2 *>(off + tile * 16 + 4 * a + 2 * half);
                wf32x16 s[U];
                float m[U];
                bool over = false;
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float *from = reinterpret_cast<const float *>(reinterpret_cast<const char *>(table) + (place[u] + key[a][j]));
                            s[u][4 * a + 2 * j] = from[0], s[u][4 * a + 2 * j + 1] = from[1];
                        }
                    }
                    s[u] = score<T, DP>(buf + S::RM0_AT, tile, own[u], s[u]);
                }
                if (!whole) {
#pragma unroll
                    for (int u = 0; u < U; ++u) leave_out(bits, -__builtin_inff(), s[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    m[u] = fmaxf(s[u][0], s[u][1]);
#pragma unroll
                    for (int i = 2; i < 16; i += 2) m[u] = fmaxf(fmaxf(m[u], s[u][i]), s[u][i + 1]);
                    m[u] = max_of_halves(m[u]);
                    over = over || m[u] > limit[u];
                }
                if (__any(over)) {
                    far = false;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const float old = top[u], next = fmaxf(old, m[u]);
                        // (a row that has seen no key yet has nothing to shrink)
                        const float shrink = old == -__builtin_inff() ? 0.f : rescale(p, old, next);
                        top[u] = next, limit[u] = next + slack;
                        shift[u] = next == -__builtin_inff() ? 0.f : next * p.log2_scale;
                        far = far || __any(__builtin_fabsf(shift[u]) > kLargeShift);
                        sum[u] *= shrink;
#pragma unroll
                        for (int b = 0; b < G::DT; ++b)
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[u][b][i] *= shrink;
                    }
                }
                if (__builtin_expect(!far, 1)) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[u][i] = __builtin_fmaf(s[u][i], p.log2_scale, -shift[u]);
                } else {
                    asm volatile("; large scores");
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const float from = top[u] == -__builtin_inff() ? 0.f : top[u], rest = shift_rest(from, p.log2_scale);
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[u][i] = __builtin_fmaf(s[u][i] - from, p.log2_scale, rest);
                    }
                }
                Packed<VT> e[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[u][i] = exp2_of(s[u][i]);
                    if constexpr (!SUM_ROW) {
                        float add = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) add += s[u][i];
                        sum[u] += add;
                    }
                    e[u] = pack<VT>(s[u]);
                }
                accumulate<T, DP>(buf + S::CM1_AT, tile, e, acc);
            }
        if (more) stager.write(p, w, k, v, t0 + G::TK, staged + (turn ^ 1) * S::BYTES);
        __syncthreads();
    }

    if (p.ksplit > 1) {  // (uniform) one tile a wavefront then
        constexpr int WORDS = 64 * (2 + G::DT * 16);
        float *room = reinterpret_cast<float *>(lds);
        if (share != 0 && wave < p.owners) {
            float *to = room + wave * WORDS + lane;
            to[0] = top[0], to[64] = sum[0];
#pragma unroll
            for (int b = 0; b < G::DT; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) to[(2 + b * 16 + i) * 64] = acc[0][b][i];
        }
        __syncthreads();
        if (share != 0 || wave >= p.owners) return;
        for (int other = 1; other < p.ksplit; ++other) {
            const float *from = room + (wave + other) * WORDS + lane;
            const float mine = top[0], theirs = from[0], next = fmaxf(mine, theirs);
            const float fm = mine == -__builtin_inff() ? 0.f : rescale(p, mine, next);
            const float ft = theirs == -__builtin_inff() ? 0.f : rescale(p, theirs, next);
            top[0] = next;
            sum[0] = sum[0] * fm + from[64] * ft;
#pragma unroll
            for (int b = 0; b < G::DT; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[0][b][i] = acc[0][b][i] * fm + from[(2 + b * 16 + i) * 64] * ft;
        }
    }
    if (!busy) return;
    const long planes = ((long)w.n * p.heads + head) * p.d * hw, row = ((long)w.n * p.heads + head) * hw;
    T *out = static_cast<T *>(p.out) + planes;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float all;
        if constexpr (SUM_ROW) {  // (row 16 lies with the lower half)
            all = sum_of_halves(half == 0 ? acc[u][0][8] : 0.f);
        } else {
            all = sum_of_halves(sum[u]);
        }
        if (!there[u]) continue;
        const bool some = ok[u] && !(all == 0.f);
        const float over = some ? 1.f / all : 0.f;
        if (SAVE && half == 0) {
            p.top[row + pixel[u]] = some && top[u] != -__builtin_inff() ? top[u] : 0.f;
            p.log_sum[row + pixel[u]] = some ? __builtin_log2f(all) : __builtin_inff();
        }
#pragma unroll
        for (int b = 0; b < G::DT; ++b)
#pragma unroll
            for (int i = 0; i < (DP == 16 ? 8 : 16); ++i) {
                const int c = b * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (c < p.d) {
                    const float o = some ? acc[u][b][i] * over : 0.f;
                    const T r = narrow<T>(o);
                    out[c * hw + pixel[u]] = r;
                    if constexpr (SAVE && !G::F32) static_cast<T *>(p.rest)[planes + c * hw + pixel[u]] = taken_by_rounding(o, r);
                }
            }
    }
}

template <typename T, int DP>
size_t lds_of(const WindowParams &p)
{
    using G = WinGeom<T, DP>;
    const size_t staged = p.buffers * (size_t)Stager<T, DP, true, false, false, true>::BYTES + (size_t)p.len * 4;
    const size_t joined = p.ksplit > 1 ? (size_t)p.owners * 256 * (2 + G::DT * 16) : 0;
    return staged > joined ? staged : joined;
}

template <typename T, int DP, int U, bool SAVE>
hipError_t launch_one(const WindowParams &p, hipStream_t s)
{
    const size_t lds = lds_of<T, DP>(p);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&window_forward_kernel<T, DP, U, SAVE>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((window_forward_kernel<T, DP, U, SAVE>), dim3((unsigned)p.grid), dim3(64 * p.waves), lds, s, p);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch(const WindowParams &p, hipStream_t s)
{
    if (p.tiles == 1) return p.top != nullptr ? launch_one<T, DP, 1, true>(p, s) : launch_one<T, DP, 1, false>(p, s);
    if constexpr (std::is_same<T, float>::value && DP == 64) return hipErrorInvalidValue;  // (two tiles would not fit the registers)
    else return p.top != nullptr ? launch_one<T, DP, 2, true>(p, s) : launch_one<T, DP, 2, false>(p, s);
}

}  // namespace

size_t window_forward_lds(const WindowParams &p, bool f32, int dp)
{
    if (f32) return dp == 16 ? lds_of<float, 16>(p) : dp == 32 ? lds_of<float, 32>(p) : lds_of<float, 64>(p);
    return dp == 16 ? lds_of<uint16_t, 16>(p) : dp == 32 ? lds_of<uint16_t, 32>(p) : lds_of<uint16_t, 64>(p);
}

hipError_t launch_window_forward(const WindowParams &p, bool f32, int dp, hipStream_t s)
{
    if (f32) return dp == 16 ? launch<float, 16>(p, s) : dp == 32 ? launch<float, 32>(p, s) : launch<float, 64>(p, s);
    return dp == 16 ? launch<uint16_t, 16>(p, s) : dp == 32 ? launch<uint16_t, 32>(p, s) : launch<uint16_t, 64>(p, s);
}

}  // namespace esc
