// Window attention, backward.  With p = exp2(log2(e) (scale q.k + bias - top) - log_sum), dp = dout . v and ds = p (dp - delta), delta the
// sum over the channels of out * dout:
//   dq = scale sum_keys ds k      dk = scale sum_queries ds q      dv = sum_queries p dout      dbias[offset] = sum ds
//
// Two kernels form the scores again, each in the orientation in which its sums need no exchange between lanes:
//   window_dq_kernel: the forward's layout (a lane holds 16 keys of a query); dq^T = K^T ds^T, and the offsets' sums.
//   window_dkv_kernel: queries down, keys across (a lane holds 16 queries of a key); dv^T = dO^T p, dk^T = Q^T ds, over all
//     query heads that share the key's.
//
// The sums of equal offsets, in a fixed order.  Each wavefront adds to a ring of its own in LDS, in 64 bits: ds_add_f64 takes 8.5 clocks for 64
// lanes where ds_add_f32 takes 193 (measured).  No instruction holds two values of one offset: its lanes are 32 queries and one
// key, one half of the wavefront after the other.  What the ring spans are the offsets between the wavefront's queries and ONE tile of
// keys; offsets that the next tile no longer reaches are complete and leave for memory.  Two small kernels add the wavefronts' parts and
// the offsets of each bucket.
//
// What bounds it: window_dq_kernel the vector instructions and the LDS (half of its time the 32 additions in 64 bits a tile), window_dkv_kernel the
// vector instructions (80 % of the slots with 2.8 wavefronts a SIMD), and with fp32 storage what its few wavefronts (one block a compute unit)
// cannot hide.  Kernels by themselves under the profiler, 64 maps of 64 x 64, 4 heads of 16, windows of 32, bf16: dq 639 us, dk and dv 666 us, the offsets' sums
// 77 us, the buckets 9 us, beside the forward's 443 us; calls of both passes in a row take 1669 us.  Registers are short: all kernels with bf16
// storage spill, with fp32 storage those for heads wider than 32, dk and dv's wider than 16 (8 to 232 bytes a lane).
#include "esc_window.hpp"

namespace esc {
namespace {

// A ring's places behind its end: a pair of offsets that runs over it stays together (two: an even number keeps what follows aligned).
constexpr int kRingMore = 2;

// p and ds in the products that give q's, k's and v's gradients, with bf16 storage: two terms, which leave the gradients off by their own rounding alone
// (0.0017 of their norm).  With one term of p dv was 0.0023 off, for 95 us less of 1740 (64 maps of 64 x 64); ds sums to 0 over a query's keys, so that
// what one rounding of each term takes weighs more: dq and dk were 0.0025 off, for 50 us less of 571 (dq) and 77 of 589 (dkv).
template <typename T>
constexpr int kTerms = std::is_same<T, float>::value ? 3 : 2;

__device__ __forceinline__ void lds_add(double *p, float v) { __hip_atomic_fetch_add(p, (double)v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

// The offsets of all its window's keys from the 32 tokens from t0 on: from the smallest on.
__device__ __forceinline__ TableRange wave_range(const Win &w, int t0)
{
    return table_range(w, t0, min(t0 + 32, w.L), -1);
}

template <typename T, int DP>
__global__ __launch_bounds__(512, window_dq_resident(WinGeom<T, DP>::F32, DP)) void window_dq_kernel(const WindowParams p)
{
    using G = WinGeom<T, DP>;
    using S = Stager<T, DP, true, true, true, false>;  // keys by tokens and by channels, values by tokens
    constexpr int U = 1;
    extern __shared__ __align__(16) char lds[];
    float *table = reinterpret_cast<float *>(lds);  // (first: its reads' addresses are then sums of two terms and a constant)
    double *rings = reinterpret_cast<double *>(lds + (size_t)p.len * 4);  // one a wavefront
    char *const staged = reinterpret_cast<char *>(rings + (p.grad_bias != nullptr ? p.owners * (p.ring + kRingMore) : 0));

    const int unit = unit_of(p);
    if (unit < 0) return;
    const int block = unit % p.blocks, head = unit / p.blocks % p.heads, wi = unit / p.blocks / p.heads;
    const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
    const int queries = p.owners * 32 * U, q0 = block * queries;
    if (q0 >= w.L) return;
    const TableRange range = table_range(w, q0, min(q0 + queries, w.L), -1);
    const float above = 2 * kSlack / p.log2_scale;
    const bool bias_grad = p.grad_bias != nullptr;

    const long hw = (long)p.H * p.W;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wq0 = q0 + wave * 32 * U;
    const bool busy = wave < p.owners && wq0 < w.L;
    const int kvh = head / (p.heads / p.kv_heads);
    const long planes = ((long)w.n * p.heads + head) * p.d * hw, row = ((long)w.n * p.heads + head) * hw;
    const T *q = static_cast<const T *>(p.q) + w.n * p.qs + head * (long)p.d * hw;
    const T *k = static_cast<const T *>(p.k) + w.n * p.ks + kvh * (long)p.d * hw;
    const T *v = static_cast<const T *>(p.v) + w.n * p.vs + kvh * (long)p.d * hw;
    const T *go = static_cast<const T *>(p.go) + planes, *out = static_cast<const T *>(p.out_in) + planes;

    S stager;
    stager.fetch(p, w, k, v, 0);
    Fragment<T, DP> own_q[U], own_go[U];
    int pixel[U], place[U];
    bool there[U], ok[U];
    float top[U], shift[U], log_sum[U], delta[U];
    wf32x16 acc[U][G::DT];
    bool far = false, all = true;
    {
        OwnValues<T, DP> vq[U], vgo[U], vout[U], vrest[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const OwnToken own_token(p, w, wq0 + u * 32 + (lane & 31));
            there[u] = own_token.there, pixel[u] = own_token.pixel, ok[u] = own_token.ok(p);
            place[u] = 4 * (w.centre - own_token.off - range.base);
            vq[u].fetch(p, q, pixel[u]);
            vgo[u].fetch(p, go, pixel[u]);
            vout[u].fetch(p, out, pixel[u]);
            if constexpr (!G::F32) vrest[u].fetch(p, static_cast<const T *>(p.rest) + planes, pixel[u]);
            top[u] = p.top[row + pixel[u]], log_sum[u] = p.log_sum[row + pixel[u]];
        }
        stage_table<false>(p, w, table, range, head);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            vq[u].clean(p, ok[u]);
            vgo[u].clean(p, ok[u]);
            vout[u].clean(p, ok[u]);
            if constexpr (!G::F32) vrest[u].clean(p, ok[u]);
            own_q[u] = fragment_of(vq[u]);
            own_go[u] = fragment_of(vgo[u]);
            float sum = 0.f;
#pragma unroll
            for (int s = 0; s < G::KS; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float o;
                    if constexpr (G::F32) o = vout[u].v[s][j];
                    else o = unrounded(vout[u].v[s][j], vrest[u].v[s][j]);
                    sum = __builtin_fmaf(o, widen(vgo[u].v[s][j]), sum);
                }
            delta[u] = sum_of_halves(sum);
            if (there[u] && half == 0) p.delta[row + pixel[u]] = delta[u];
            if (!ok[u]) top[u] = 0.f, log_sum[u] = __builtin_inff();
            shift[u] = top[u] * p.log2_scale + log_sum[u];
            log_sum[u] -= shift_rest(top[u], p.log2_scale);  // (for scores that have top subtracted)
            far = far || __any(__builtin_fabsf(top[u] * p.log2_scale) > kLargeRow);
            all = all && __all(ok[u]);
#pragma unroll
            for (int b = 0; b < G::DT; ++b) acc[u][b] = wf32x16{};
        }
    }
    double *const ring = rings + wave * (p.ring + kRingMore);
    const int ring_mask = 8 * p.ring - 8;  // (in bytes)
    const TableRange mine = wave_range(w, min(wq0, w.L - 1));
    const int ring_place = 2 * place[0] + 8 * (range.base - mine.base);  // in the ring, in bytes, of the offset to the key that has off = 0
    float *const part = p.part + ((long)unit * p.owners + wave) * p.part_len;
    int left = 0;  // offsets that have left the ring
    if (bias_grad && busy)
        for (int i = lane; i < p.ring + kRingMore; i += 64) ring[i] = 0.0;
    S::clear(p, staged);
    if (p.buffers == 2) S::clear(p, staged + S::BYTES);
    __syncthreads();
    stager.write(p, w, k, v, 0, staged);
    __syncthreads();

    for (int t0 = 0, turn = 0; t0 < w.L; t0 += G::TK) {
        const bool more = t0 + G::TK < w.L;
        if (more) stager.fetch(p, w, k, v, t0 + G::TK);
        const char *buf = staged + turn * S::BYTES;
        const int *off = reinterpret_cast<const int *>(buf + S::OFF_AT);
        auto tile_of = [&](int tile, auto large) {
            const wu32x4 bits = *reinterpret_cast<const wu32x4 *>(buf + S::BITS_AT + tile * 16);
            const bool whole = all && all_take_part(bits);
            wi32x2 key[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) key[a] = *reinterpret_cast<const wi32x2 *>(off + tile * 16 + 4 * a + 2 * half);
            wf32x16 ds[U];
            Packed<kTerms<T>> e[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                wf32x16 s;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float *from = reinterpret_cast<const float *>(reinterpret_cast<const char *>(table) + (place[u] + key[a][j]));
                        s[4 * a + 2 * j] = from[0], s[4 * a + 2 * j + 1] = from[1];
                    }
                }
                s = score<T, DP>(buf + S::RM0_AT, tile, own_q[u], s);
                const wf32x16 dp = score<T, DP>(buf + S::RM1_AT, tile, own_go[u], wf32x16{});
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if constexpr (decltype(large)::value) s[i] = __builtin_fmaf(fminf(s[i] - top[u], above), p.log2_scale, -log_sum[u]);
                    else s[i] = __builtin_fmaf(s[i], p.log2_scale, -shift[u]);
                    ds[u][i] = exp2_of(s[i]) * (dp[i] - delta[u]);
                }
                if (!whole) {
                    leave_out(bits, 0.f, ds[u]);
#pragma unroll
                    for (int i = 0; i < 16; ++i) ds[u][i] = ok[u] ? ds[u][i] : 0.f;
                }
                e[u] = pack<kTerms<T>>(ds[u]);
            }
            accumulate<T, DP>(buf + S::CM0_AT, tile, e, acc);
            if (bias_grad) {
                // (both halves of a query's lanes; the second after the first: keys four tokens apart see equal offsets of queries four apart)
                double *to[8];
#pragma unroll
                for (int a = 0; a < 8; ++a) to[a] = reinterpret_cast<double *>(reinterpret_cast<char *>(ring) + ((ring_place + 2 * key[a / 2][a % 2]) & ring_mask));
                if (half == 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) lds_add(to[i / 2] + i % 2, ds[0][i]);
                }
                if (half == 1) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) lds_add(to[i / 2] + i % 2, ds[0][i]);
                }
                const int t = t0 + tile * 32 + 32;  // the next tile's first key
                const int y = w.row(t), done = t < w.L ? y * w.tw + t - y * w.wp : mine.len;
                for (int i = left + lane; i < done; i += 64) {
                    const int at = i & (p.ring - 1);
                    double sum = ring[at];
                    ring[at] = 0.0;
                    if (at == 0) sum += ring[p.ring + at], ring[p.ring + at] = 0.0;
                    part[i] = (float)sum;
                }
                left = done;
            }
        };
        if (busy) {
            if (__builtin_expect(!far, 1)) {
#pragma unroll
                for (int tile = 0; tile < G::TK / 32; ++tile)
                    if (t0 + tile * 32 < w.L) tile_of(tile, std::false_type{});
            } else {
#pragma unroll 1
                for (int tile = 0; tile < G::TK / 32 && t0 + tile * 32 < w.L; ++tile) tile_of(tile, std::true_type{});
            }
        }
        if (p.buffers == 1) __syncthreads();
        else turn ^= 1;
        if (more) stager.write(p, w, k, v, t0 + G::TK, staged + turn * S::BYTES);
        __syncthreads();
    }
    if (!busy) return;
    T *gq = static_cast<T *>(p.gq) + w.n * p.gqs + head * (long)p.d * hw;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int b = 0; b < G::DT; ++b)
#pragma unroll
            for (int i = 0; i < (DP == 16 ? 8 : 16); ++i) {
                const int c = b * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (there[u] && c < p.d) gq[c * hw + pixel[u]] = narrow<T>(acc[u][b][i] * p.scale);
            }
}

template <typename T, int DP>
__global__ __launch_bounds__(512, window_dkv_resident(WinGeom<T, DP>::F32, DP)) void window_dkv_kernel(const WindowParams p)
{
    using G = WinGeom<T, DP>;
    using S = Stager<T, DP, true, true, true, true>;  // queries and the result's gradient, by tokens and by channels
    constexpr int U = 1;
    // of the staged queries: the exponent's shift with the sum's logarithm, -delta; for large shifts the largest score and the logarithm
    // by themselves; a flag of each wavefront that has seen such a shift
    constexpr int ROWS_AT = S::BYTES, FAR_AT = ROWS_AT + 4 * G::TK * 4, BYTES = FAR_AT + 4 * kWinMaxWaves;
    extern __shared__ __align__(16) char lds[];
    float *table = reinterpret_cast<float *>(lds);
    char *const staged = lds + (size_t)p.len * 4;

    const int unit = unit_of(p);
    if (unit < 0) return;
    const int block = unit % p.blocks, kvh = unit / p.blocks % p.kv_heads, wi = unit / p.blocks / p.kv_heads;
    const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
    const int keys = p.owners * 32 * U, k0 = block * keys;
    if (k0 >= w.L) return;
    const TableRange range = table_range(w, k0, min(k0 + keys, w.L), 1);
    const float above = 2 * kSlack / p.log2_scale;

    const long hw = (long)p.H * p.W;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = p.heads / p.kv_heads;
    const int wk0 = k0 + wave * 32 * U;
    const bool busy = wave < p.owners && wk0 < w.L;
    const T *k = static_cast<const T *>(p.k) + w.n * p.ks + kvh * (long)p.d * hw;
    const T *v = static_cast<const T *>(p.v) + w.n * p.vs + kvh * (long)p.d * hw;
    const T *q = static_cast<const T *>(p.q) + w.n * p.qs, *go = static_cast<const T *>(p.go) + (long)w.n * p.heads * p.d * hw;

    // chunks of queries of one head after the other of the group
    S stager;
    float from, log_sum, delta;  // of this thread's query of the next chunk, as they come
    bool in;
    auto fetch_row = [&](int head, int t) {
        const Spot spot(p, w, t, 1);
        const long pix = ((long)w.n * p.heads + head) * hw + spot.at;
        from = p.top[pix], log_sum = p.log_sum[pix], delta = p.delta[pix];
        in = spot.bits != 0;
    };
    auto fetch = [&](int head, int t0) {
        stager.fetch(p, w, q + head * (long)p.d * hw, go + head * (long)p.d * hw, t0);
        fetch_row(head, t0 + min((int)threadIdx.x, G::TK - 1));
    };
    auto write = [&](int head, int t0, char *buf) {
        stager.write(p, w, q + head * (long)p.d * hw, go + head * (long)p.d * hw, t0, buf);
        bool large = false;
        for (int r = threadIdx.x; r < G::TK; r += blockDim.x) {
            if (r != (int)threadIdx.x) fetch_row(head, t0 + r);
            // (masked pixels have a sum of +infinity and a delta of 0; those beyond the window get them here)
            float *rows = reinterpret_cast<float *>(buf + ROWS_AT) + r;
            const float shift = in ? from * p.log2_scale : 0.f, l = in ? log_sum : __builtin_inff();
            large = large || __builtin_fabsf(shift) > kLargeRow;
            rows[0] = shift + l, rows[G::TK] = in ? -delta : 0.f, rows[2 * G::TK] = from;
            rows[3 * G::TK] = in ? l - shift_rest(from, p.log2_scale) : l;
        }
        int *flags = reinterpret_cast<int *>(buf + FAR_AT);
        const bool any = __any(large);
        if (lane == 0) flags[wave] = any;
        if ((int)threadIdx.x >= p.waves && threadIdx.x < kWinMaxWaves) flags[threadIdx.x] = 0;
    };
    int head = kvh * group;
    fetch(head, 0);
    Fragment<T, DP> own_k[U], own_v[U];
    int pixel[U], place[U];
    bool there[U], ok[U];
    wf32x16 dk[U][G::DT], dv[U][G::DT];
    {
        OwnValues<T, DP> vk[U], vv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const OwnToken own_token(p, w, wk0 + u * 32 + (lane & 31));
            there[u] = own_token.there, pixel[u] = own_token.pixel, ok[u] = own_token.ok(p);
            place[u] = 4 * (range.len - 1 - (w.centre + own_token.off - range.base));
            vk[u].fetch(p, k, pixel[u]);
            vv[u].fetch(p, v, pixel[u]);
        }
        stage_table<true>(p, w, table, range, kvh * group);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            vk[u].clean(p, ok[u]);
            vv[u].clean(p, ok[u]);
            own_k[u] = fragment_of(vk[u]);
            own_v[u] = fragment_of(vv[u]);
#pragma unroll
            for (int b = 0; b < G::DT; ++b) dk[u][b] = wf32x16{}, dv[u][b] = wf32x16{};
        }
    }
    S::clear(p, staged);
    if (p.buffers == 2) S::clear(p, staged + BYTES);
    __syncthreads();
    write(head, 0, staged);
    __syncthreads();

    for (int t0 = 0, turn = 0;;) {
        const bool last = t0 + G::TK >= w.L, more = !last || head + 1 < (kvh + 1) * group;
        const int next_t0 = last ? 0 : t0 + G::TK, next_head = last ? head + 1 : head;
        if (more) fetch(next_head, next_t0);
        const char *buf = staged + turn * BYTES;
        const int *off = reinterpret_cast<const int *>(buf + S::OFF_AT);
        const float *rows = reinterpret_cast<const float *>(buf + ROWS_AT);
        const wu32x4 flags = *reinterpret_cast<const wu32x4 *>(buf + FAR_AT) | *reinterpret_cast<const wu32x4 *>(buf + FAR_AT + 16);
        const bool far = __builtin_amdgcn_readfirstlane((int)(flags.x | flags.y | flags.z | flags.w)) != 0;
        auto tile_of = [&](int tile, auto large) {
            const wu32x4 bits = *reinterpret_cast<const wu32x4 *>(buf + S::BITS_AT + tile * 16);
            const bool whole = all_take_part(bits);
            Packed<kTerms<T>> ep[U];
            Packed<kTerms<T>> es[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                wf32x16 s, dp;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const wi32x2 query = *reinterpret_cast<const wi32x2 *>(off + tile * 16 + 4 * a + 2 * half);
                    const wf32x4 d = *reinterpret_cast<const wf32x4 *>(rows + G::TK + tile * 32 + 8 * a + 4 * half);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float *at = reinterpret_cast<const float *>(reinterpret_cast<const char *>(table) + (place[u] + query[j / 2]));
                        s[4 * a + j] = at[j % 2], dp[4 * a + j] = d[j];
                    }
                }
                s = score<T, DP, true>(buf + S::RM0_AT, tile, own_k[u], s);
                dp = score<T, DP>(buf + S::RM1_AT, tile, own_v[u], dp);
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const float *at = rows + (decltype(large)::value ? 3 * G::TK : 0) + tile * 32 + 8 * a + 4 * half;
                    const wf32x4 l = *reinterpret_cast<const wf32x4 *>(at);
                    wf32x4 m;
                    if constexpr (decltype(large)::value) m = *reinterpret_cast<const wf32x4 *>(at - G::TK);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x = s[4 * a + j];
                        if constexpr (decltype(large)::value) x = fminf(x - m[j], above);
                        s[4 * a + j] = exp2_of(__builtin_fmaf(x, p.log2_scale, -l[j]));
                    }
                }
                if (!whole) {
                    leave_out(bits, 0.f, s);
                }
                ep[u] = pack<kTerms<T>>(s);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] *= dp[i];
                es[u] = pack<kTerms<T>>(s);
            }
            accumulate<T, DP>(buf + S::CM1_AT, tile, ep, dv);
            accumulate<T, DP>(buf + S::CM0_AT, tile, es, dk);
        };
        if (busy) {
            if (__builtin_expect(!far, 1)) {
#pragma unroll
                for (int tile = 0; tile < G::TK / 32; ++tile)
                    if (t0 + tile * 32 < w.L) tile_of(tile, std::false_type{});
            } else {
#pragma unroll 1
                for (int tile = 0; tile < G::TK / 32 && t0 + tile * 32 < w.L; ++tile) tile_of(tile, std::true_type{});
            }
        }
        if (p.buffers == 1) __syncthreads();
        else turn ^= 1;
        if (!more) break;
        write(next_head, next_t0, staged + turn * BYTES);
        if (last) {  // (uniform) another head's biases: nobody may still read the last one's
            if (p.buffers != 1) __syncthreads();
            stage_table<true>(p, w, table, range, next_head);
        }
        __syncthreads();
        t0 = next_t0, head = next_head;
    }
    if (!busy) return;
    T *gk = static_cast<T *>(p.gk) + w.n * p.gks + kvh * (long)p.d * hw;
    T *gv = static_cast<T *>(p.gv) + w.n * p.gvs + kvh * (long)p.d * hw;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int b = 0; b < G::DT; ++b)
#pragma unroll
            for (int i = 0; i < (DP == 16 ? 8 : 16); ++i) {
                const int c = b * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (there[u] && c < p.d) {
                    gk[c * hw + pixel[u]] = narrow<T>(ok[u] ? dk[u][b][i] * p.scale : 0.f);
                    gv[c * hw + pixel[u]] = narrow<T>(ok[u] ? dv[u][b][i] : 0.f);
                }
            }
}

// Sums of equal offsets over the wavefronts' parts, every `splits`-th window's, in order.  A thread has four offsets (the parts' ranges are worked
// out once for them), and reads four parts at a time.
__global__ __launch_bounds__(256) void window_offsets_kernel(const WindowParams p)
{
    constexpr int EACH = 4, AHEAD = 4;
    const int at0 = blockIdx.x * (256 * EACH) + threadIdx.x, head = blockIdx.y;
    const int windows = p.N * p.gy * p.gx;
    float sum[EACH] = {};
    int oy[EACH], ox[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) oy[e] = (at0 + 256 * e) / p.tw, ox[e] = (at0 + 256 * e) % p.tw - (p.ww - 1);
    for (int wi = blockIdx.z; wi < windows; wi += p.splits) {
        const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
        const float *part = p.part + (long)(wi * p.heads + head) * p.blocks * p.owners * p.part_len;
        int at[EACH];  // the offset's number in this window
#pragma unroll
        for (int e = 0; e < EACH; ++e) at[e] = abs(ox[e]) < w.w ? oy[e] * w.tw + ox[e] + w.w - 1 : -1;
        for (int t0 = 0; t0 < w.L; t0 += 32 * AHEAD) {
            float v[AHEAD][EACH];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int t = t0 + 32 * i;
                const TableRange r = wave_range(w, t);
#pragma unroll
                for (int e = 0; e < EACH; ++e) {
                    const int in = at[e] - r.base;
                    v[i][e] = t < w.L && at[e] >= 0 && in >= 0 && in < r.len ? part[in] : 0.f;
                }
                part += p.part_len;
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                for (int e = 0; e < EACH; ++e) sum[e] += v[i][e];
        }
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if (at0 + 256 * e < p.th * p.tw) p.part2[((long)blockIdx.z * p.heads + head) * p.th * p.tw + at0 + 256 * e] = sum[e];
}

// The offsets (inclusive) along one axis that a bucket holds, cut to those that exist.
__device__ __forceinline__ void bucket_range(const WindowParams &p, int b, int full, int n, int *lo, int *hi)
{
    if (p.n_edges == 0) {
        *lo = *hi = b - (full - 1);
    } else {
        const int s = b - p.n_edges, a = s < 0 ? -s : s;
        const int near = a == 0 ? 0 : p.edges[a - 1], far = a == p.n_edges ? n : p.edges[a] - 1;
        *lo = s > 0 ? near : -far;
        *hi = s < 0 ? -near : far;
    }
    *lo = max(*lo, -(n - 1));
    *hi = min(*hi, n - 1);
}

// The sums of each bucket's offsets: a wavefront for each where every offset has its own, a block where buckets hold many.  (A table may have far more
// buckets than the map has offsets: up to kBucketBlocks blocks a head go through them.)
constexpr int kBucketBlocks = 1 << 16;
__global__ __launch_bounds__(256) void window_buckets_kernel(const WindowParams p)
{
    __shared__ float part[4];
    const int wave = threadIdx.x >> 6, head = blockIdx.y, lane = threadIdx.x & 63, buckets = p.nby * p.nbx;
    const bool whole = p.n_edges > 0;
    const int threads = whole ? 256 : 64, step = whole ? gridDim.x : gridDim.x * 4;
    for (int b = whole ? blockIdx.x : blockIdx.x * 4 + wave; b < buckets; b += step) {
        int y0, y1, x0, x1;
        bucket_range(p, b / p.nbx, p.win_h, p.wh, &y0, &y1);
        bucket_range(p, b % p.nbx, p.win_w, p.ww, &x0, &x1);
        const int cols = x1 - x0 + 1, count = y1 >= y0 && cols > 0 ? (y1 - y0 + 1) * cols * p.splits : 0;
        float sum = 0.f;
#pragma unroll 4
        for (int i = whole ? threadIdx.x : lane; i < count; i += threads) {
            const int split = i % p.splits, o = i / p.splits, y = y0 + o / cols, x = x0 + o % cols;
            sum += p.part2[((long)split * p.heads + head) * p.th * p.tw + (y + p.wh - 1) * p.tw + x + p.ww - 1];
        }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
        if (whole) {  // (b is the block's then: all of it comes here)
            if (lane == 0) part[wave] = sum;
            __syncthreads();
            sum = part[0] + part[1] + part[2] + part[3];
            __syncthreads();
        }
        if (whole ? threadIdx.x == 0 : lane == 0) {
            float *to = p.grad_bias + (long)head * buckets + b;
            *to = p.accumulate != 0 ? *to + sum : sum;
        }
    }
}

template <typename T, int DP>
size_t dq_lds(const WindowParams &p)
{
    return p.buffers * (size_t)Stager<T, DP, true, true, true, false>::BYTES + (p.grad_bias != nullptr ? (size_t)p.owners * (p.ring + kRingMore) * 8 : 0) + (size_t)p.len * 4;
}
template <typename T, int DP>
size_t dkv_lds(const WindowParams &p)
{
    return p.buffers * (size_t)(Stager<T, DP, true, true, true, true>::BYTES + 4 * WinGeom<T, DP>::TK * 4 + 4 * kWinMaxWaves) + (size_t)p.len * 4;
}

hipError_t allow(const void *kernel, size_t lds)
{
    return lds <= 64 * 1024 ? hipSuccess : hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
}

template <typename T, int DP>
hipError_t launch_dq(const WindowParams &p, hipStream_t s)
{
    const size_t lds = dq_lds<T, DP>(p);
    const hipError_t e = allow(reinterpret_cast<const void *>(&window_dq_kernel<T, DP>), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_dq_kernel<T, DP>), dim3((unsigned)p.grid), dim3(64 * p.waves), lds, s, p);
    return hipGetLastError();
}
template <typename T, int DP>
hipError_t launch_dkv(const WindowParams &p, hipStream_t s)
{
    const size_t lds = dkv_lds<T, DP>(p);
    const hipError_t e = allow(reinterpret_cast<const void *>(&window_dkv_kernel<T, DP>), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_dkv_kernel<T, DP>), dim3((unsigned)p.grid), dim3(64 * p.waves), lds, s, p);
    return hipGetLastError();
}

}  // namespace

size_t window_dq_lds(const WindowParams &p, bool f32, int dp)
{
    if (f32) return dp == 16 ? dq_lds<float, 16>(p) : dp == 32 ? dq_lds<float, 32>(p) : dq_lds<float, 64>(p);
    return dp == 16 ? dq_lds<uint16_t, 16>(p) : dp == 32 ? dq_lds<uint16_t, 32>(p) : dq_lds<uint16_t, 64>(p);
}

size_t window_dkv_lds(const WindowParams &p, bool f32, int dp)
{
    if (f32) return dp == 16 ? dkv_lds<float, 16>(p) : dp == 32 ? dkv_lds<float, 32>(p) : dkv_lds<float, 64>(p);
    return dp == 16 ? dkv_lds<uint16_t, 16>(p) : dp == 32 ? dkv_lds<uint16_t, 32>(p) : dkv_lds<uint16_t, 64>(p);
}

hipError_t launch_window_dq(const WindowParams &p, bool f32, int dp, hipStream_t s)
{
    if (f32) return dp == 16 ? launch_dq<float, 16>(p, s) : dp == 32 ? launch_dq<float, 32>(p, s) : launch_dq<float, 64>(p, s);
    return dp == 16 ? launch_dq<uint16_t, 16>(p, s) : dp == 32 ? launch_dq<uint16_t, 32>(p, s) : launch_dq<uint16_t, 64>(p, s);
}

hipError_t launch_window_dkv(const WindowParams &p, bool f32, int dp, hipStream_t s)
{
    if (f32) return dp == 16 ? launch_dkv<float, 16>(p, s) : dp == 32 ? launch_dkv<float, 32>(p, s) : launch_dkv<float, 64>(p, s);
    return dp == 16 ? launch_dkv<uint16_t, 16>(p, s) : dp == 32 ? launch_dkv<uint16_t, 32>(p, s) : launch_dkv<uint16_t, 64>(p, s);
}

hipError_t launch_window_bias_grad(const WindowParams &p, hipStream_t s)
{
    hipLaunchKernelGGL(window_offsets_kernel, dim3((unsigned)((p.th * p.tw + 1023) / 1024), (unsigned)p.heads, (unsigned)p.splits), dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int buckets = p.nby * p.nbx, blocks = p.n_edges > 0 ? buckets : (buckets + 3) / 4;
    hipLaunchKernelGGL(window_buckets_kernel, dim3((unsigned)(blocks < kBucketBlocks ? blocks : kBucketBlocks), (unsigned)p.heads), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace esc
