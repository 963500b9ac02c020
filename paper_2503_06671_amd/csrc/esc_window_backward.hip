// Window attention, backward.  With p = exp2(log2(e) (scale q.k + bias - top) - log_sum), dp = dout . v and ds = p (dp - delta), delta the
// sum over the channels of out * dout:
//   dq = scale sum_keys ds k      dk = scale sum_queries ds q      dv = sum_queries p dout      dbias[offset] = sum ds
//
// Two kernels form the scores again, each in the orientation in which its sums need no exchange between lanes:
//   window_dq_kernel: the forward's layout (a lane holds 16 keys of a query); dq^T = K^T ds^T, and the offsets' sums.
//   window_dkv_kernel: queries down, keys across (a lane holds 16 queries of a key); dv^T = dO^T p, dk^T = Q^T ds, over all
//     query heads that share the key's.
// The sums of equal offsets have a fixed order: each wavefront adds to a table of its own in LDS, and no instruction holds two
// values of one offset (its 64 lanes are 64 queries and one key: permlane32_swap brings the two tiles' halves together).  The
// wavefronts' tables are added in order, written, and two small kernels add the blocks' tables and the offsets of each bucket.
#include "esc_window.hpp"

namespace esc {
namespace {

__device__ __forceinline__ void lds_add(float *p, float v)
{
    __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void window_dq_kernel(const WindowParams p)
{
    using G = WinGeom<T, DP>;
    extern __shared__ __align__(16) char lds[];
    char *k_rm = lds, *k_cm = k_rm + G::RM_BYTES, *v_rm = k_cm + G::CM_BYTES;
    int *off = reinterpret_cast<int *>(v_rm + G::RM_BYTES);
    uint8_t *bits = reinterpret_cast<uint8_t *>(off + G::TK / 4);
    float *table = reinterpret_cast<float *>(bits + G::TK / 4);
    float *sums = table + p.len;  // one table a wavefront

    const int unit = unit_of(p.units);
    if (unit < 0) return;
    const int block = unit % p.blocks, head = unit / p.blocks % p.heads, wi = unit / p.blocks / p.heads;
    const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
    const int q0 = block * p.waves * kWinWaveTokens;
    if (q0 >= w.L) return;
    const int centre = (p.wh - 1) * p.tw + p.ww - 1;
    const TableRange range = table_range(q0, min(q0 + p.waves * kWinWaveTokens, w.L), w.h, w.wp, p.tw, centre, -1);
    stage_table(p, table, range, head);
    const bool bias_grad = p.grad_bias != nullptr;
    if (bias_grad)
        for (int i = threadIdx.x; i < p.waves * p.len; i += blockDim.x) sums[i] = 0.f;

    const long hw = (long)p.H * p.W;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int kvh = head / (p.heads / p.kv_heads);
    const long planes = ((long)w.n * p.heads + head) * p.d * hw, row = ((long)w.n * p.heads + head) * hw;
    const T *q = static_cast<const T *>(p.q) + w.n * p.qs + head * (long)p.d * hw;
    const T *k = static_cast<const T *>(p.k) + w.n * p.ks + kvh * (long)p.d * hw;
    const T *v = static_cast<const T *>(p.v) + w.n * p.vs + kvh * (long)p.d * hw;
    const T *go = static_cast<const T *>(p.go) + planes, *out = static_cast<const T *>(p.out_in) + planes;

    Fragment<T, DP> own_q[2], own_go[2];
    long pixel[2];
    bool there[2], ok[2], large[2];
    int place[2];
    float top[2], shift[2], log_sum[2], delta[2];
    wf32x16 acc[2][G::DT];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int t = q0 + wave * kWinWaveTokens + u * 32 + (lane & 31), tc = min(t, w.L - 1);
        const int y = tc / w.wp, x = tc - y * w.wp;
        there[u] = t < w.L && x < w.w;
        ok[u] = there[u] && seen(p, w, y, x);
        pixel[u] = (long)(w.y0 + y) * p.W + w.x0 + x;
        place[u] = centre - (y * p.tw + x) - range.base;
        own_q[u] = own_fragment<T, DP>(p, q + pixel[u], ok[u]);
        own_go[u] = own_fragment<T, DP>(p, go + pixel[u], ok[u]);
        top[u] = ok[u] ? p.top[row + pixel[u]] : 0.f;
        log_sum[u] = ok[u] ? p.log_sum[row + pixel[u]] : __builtin_inff();
        shift[u] = top[u] * p.log2_scale;
        large[u] = __any(__builtin_fabsf(shift[u]) > kLargeShift);
        float sum = 0.f;
        if (ok[u])
            for (int c = half; c < p.d; c += 2) {
                float o = widen(out[c * hw + pixel[u]]);
                if constexpr (!G::F32) o += widen(static_cast<const T *>(p.rest)[planes + c * hw + pixel[u]]);
                sum = __builtin_fmaf(o, widen(go[c * hw + pixel[u]]), sum);
            }
        delta[u] = sum + other_half(sum);
        if (there[u] && half == 0) p.delta[row + pixel[u]] = delta[u];
#pragma unroll
        for (int b = 0; b < G::DT; ++b) acc[u][b] = wf32x16{};
    }
    // the table place of the lane's query where the wavefront's 64 lanes are its 64 queries
    const int place64 = half == 0 ? place[0] : place[1];
    float *const mine = sums + wave * p.len + place64;
    const bool busy = q0 + wave * kWinWaveTokens < w.L;

    for (int t0 = 0; t0 < w.L; t0 += G::TK) {
        __syncthreads();
        stage<T, DP, true, true>(p, w, k, t0, k_rm, k_cm, threadIdx.x, blockDim.x);
        stage<T, DP, true, false>(p, w, v, t0, v_rm, nullptr, threadIdx.x, blockDim.x);
        stage_tokens<G::TK>(p, w, t0, off, bits);
        __syncthreads();
        if (!busy) continue;
        for (int tile = 0; tile < G::TK / 32 && t0 + tile * 32 < w.L; ++tile) {
            const wu32x2 nibbles = *reinterpret_cast<const wu32x2 *>(bits + tile * 8);
            const bool whole = __builtin_amdgcn_readfirstlane((int)((nibbles.x & nibbles.y) == 0x0f0f0f0fu));
            wf32x16 ds[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                wf32x16 s;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const float *from = table + place[u] + off[tile * 8 + 2 * a + half];
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[4 * a + j] = from[j];
                }
                s = score<T, DP>(k_rm, tile, own_q[u], s);
                const wf32x16 dp = score<T, DP>(v_rm, tile, own_go[u], wf32x16{});
                if (__builtin_expect(!large[u], 1)) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], p.log2_scale, -(shift[u] + log_sum[u]));
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(fminf(s[i] - top[u], 0.f), p.log2_scale, -log_sum[u]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[u][i] = exp2_of(s[i]) * (dp[i] - delta[u]);
                if (!whole || !ok[u]) {
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const uint32_t b = (a < 2 ? nibbles.x : nibbles.y) >> (16 * (a & 1) + 8 * half);
#pragma unroll
                        for (int j = 0; j < 4; ++j) ds[u][4 * a + j] = ok[u] && (b >> j & 1) != 0 ? ds[u][4 * a + j] : 0.f;
                    }
                }
                accumulate<T, DP>(k_cm, tile, pack<G::NT>(ds[u]), acc[u]);
            }
            if (bias_grad) {
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const int lo = off[tile * 8 + 2 * a], hi = off[tile * 8 + 2 * a + 1];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(ds[0][4 * a + j]), __float_as_uint(ds[1][4 * a + j]), false, false);
                        lds_add(mine + lo + j, __uint_as_float(x[0]));
                        lds_add(mine + hi + j, __uint_as_float(x[1]));
                    }
                }
            }
        }
    }
    if (busy) {
        T *gq = static_cast<T *>(p.gq) + w.n * p.gqs + head * (long)p.d * hw;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int b = 0; b < G::DT; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int c = b * 32 + 8 * (i / 4) + 4 * half + i % 4;
                    if (there[u] && c < p.d) gq[c * hw + pixel[u]] = narrow<T>(acc[u][b][i] * p.scale);
                }
    }
    if (bias_grad) {
        __syncthreads();
        float *to = p.part + (long)unit * p.len;
        for (int i = threadIdx.x; i < range.len; i += blockDim.x) {
            float s = sums[i];
            for (int j = 1; j < p.waves; ++j) s += sums[j * p.len + i];
            to[i] = s;
        }
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(256) void window_dkv_kernel(const WindowParams p)
{
    using G = WinGeom<T, DP>;
    extern __shared__ __align__(16) char lds[];
    char *q_rm = lds, *q_cm = q_rm + G::RM_BYTES, *g_rm = q_cm + G::CM_BYTES, *g_cm = g_rm + G::RM_BYTES;
    // of the staged queries: the exponent's shift (with the sum's logarithm; without it and the largest score, where a shift is large), -delta
    float *shift = reinterpret_cast<float *>(g_cm + G::CM_BYTES), *top = shift + G::TK, *minus_delta = top + G::TK;
    int *off = reinterpret_cast<int *>(minus_delta + G::TK);
    uint8_t *bits = reinterpret_cast<uint8_t *>(off + G::TK / 4);
    int *large = reinterpret_cast<int *>(bits + G::TK / 4);
    float *table = reinterpret_cast<float *>(large + 1);

    const int unit = unit_of(p.units);
    if (unit < 0) return;
    const int block = unit % p.blocks, kvh = unit / p.blocks % p.kv_heads, wi = unit / p.blocks / p.kv_heads;
    const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
    const int k0 = block * p.waves * kWinWaveTokens;
    if (k0 >= w.L) return;
    const int centre = (p.wh - 1) * p.tw + p.ww - 1;
    const TableRange range = table_range(k0, min(k0 + p.waves * kWinWaveTokens, w.L), w.h, w.wp, p.tw, centre, 1);

    const long hw = (long)p.H * p.W;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int group = p.heads / p.kv_heads;
    const T *k = static_cast<const T *>(p.k) + w.n * p.ks + kvh * (long)p.d * hw;
    const T *v = static_cast<const T *>(p.v) + w.n * p.vs + kvh * (long)p.d * hw;

    Fragment<T, DP> own_k[2], own_v[2];
    long pixel[2];
    bool there[2], ok[2];
    int place[2];
    wf32x16 dk[2][G::DT], dv[2][G::DT];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int t = k0 + wave * kWinWaveTokens + u * 32 + (lane & 31), tc = min(t, w.L - 1);
        const int y = tc / w.wp, x = tc - y * w.wp;
        there[u] = t < w.L && x < w.w;
        ok[u] = there[u] && seen(p, w, y, x);
        pixel[u] = (long)(w.y0 + y) * p.W + w.x0 + x;
        place[u] = centre + (y * p.tw + x) - range.base;
        own_k[u] = own_fragment<T, DP>(p, k + pixel[u], ok[u]);
        own_v[u] = own_fragment<T, DP>(p, v + pixel[u], ok[u]);
#pragma unroll
        for (int b = 0; b < G::DT; ++b) dk[u][b] = wf32x16{}, dv[u][b] = wf32x16{};
    }
    const bool busy = k0 + wave * kWinWaveTokens < w.L;

    for (int head = kvh * group; head < (kvh + 1) * group; ++head) {
        const long planes = ((long)w.n * p.heads + head) * p.d * hw, row = ((long)w.n * p.heads + head) * hw;
        const T *q = static_cast<const T *>(p.q) + w.n * p.qs + head * (long)p.d * hw;
        const T *go = static_cast<const T *>(p.go) + planes;
        __syncthreads();
        stage_table(p, table, range, head);
        for (int t0 = 0; t0 < w.L; t0 += G::TK) {
            __syncthreads();
            stage<T, DP, true, true>(p, w, q, t0, q_rm, q_cm, threadIdx.x, blockDim.x);
            stage<T, DP, true, true>(p, w, go, t0, g_rm, g_cm, threadIdx.x, blockDim.x);
            stage_tokens<G::TK>(p, w, t0, off, bits);
            bool far = false;
            if (threadIdx.x < G::TK) {
                const int t = t0 + threadIdx.x;
                float from = 0.f, log_sum = __builtin_inff(), d = 0.f;
                if (t < w.L) {
                    const int y = t / w.wp, x = t - y * w.wp;
                    if (seen(p, w, y, x)) {
                        const long pix = row + (long)(w.y0 + y) * p.W + w.x0 + x;
                        from = p.top[pix], log_sum = p.log_sum[pix], d = -p.delta[pix];
                    }
                }
                far = __any(__builtin_fabsf(from * p.log2_scale) > kLargeShift);  // (a wavefront's threads: TK is at most 64)
                shift[threadIdx.x] = far ? log_sum : from * p.log2_scale + log_sum;
                top[threadIdx.x] = from, minus_delta[threadIdx.x] = d;
                if (threadIdx.x == 0) *large = far;
            }
            __syncthreads();
            if (!busy) continue;
            far = __builtin_amdgcn_readfirstlane(*large) != 0;
            for (int tile = 0; tile < G::TK / 32 && t0 + tile * 32 < w.L; ++tile) {
                const wu32x2 nibbles = *reinterpret_cast<const wu32x2 *>(bits + tile * 8);
                const bool whole = __builtin_amdgcn_readfirstlane((int)((nibbles.x & nibbles.y) == 0x0f0f0f0fu));
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    wf32x16 s, dp;
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const float *from = table + place[u] - off[tile * 8 + 2 * a + half];
                        const wf32x4 d = *reinterpret_cast<const wf32x4 *>(minus_delta + tile * 32 + 8 * a + 4 * half);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[4 * a + j] = from[-j], dp[4 * a + j] = d[j];
                    }
                    s = score<T, DP, true>(q_rm, tile, own_k[u], s);
                    dp = score<T, DP>(g_rm, tile, own_v[u], dp);
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const wf32x4 l = *reinterpret_cast<const wf32x4 *>(shift + tile * 32 + 8 * a + 4 * half);
                        if (__builtin_expect(far, 0)) {
                            const wf32x4 m = *reinterpret_cast<const wf32x4 *>(top + tile * 32 + 8 * a + 4 * half);
#pragma unroll
                            for (int j = 0; j < 4; ++j) s[4 * a + j] = fminf(s[4 * a + j] - m[j], 0.f);
                        }
                        const uint32_t b = (a < 2 ? nibbles.x : nibbles.y) >> (16 * (a & 1) + 8 * half);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float e = exp2_of(__builtin_fmaf(s[4 * a + j], p.log2_scale, -l[j]));
                            s[4 * a + j] = whole || (b >> j & 1) != 0 ? e : 0.f;
                        }
                    }
                    accumulate<T, DP>(g_cm, tile, pack<G::NT>(s), dv[u]);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] *= dp[i];
                    accumulate<T, DP>(q_cm, tile, pack<G::NT>(s), dk[u]);
                }
            }
        }
    }
    if (!busy) return;
    T *gk = static_cast<T *>(p.gk) + w.n * p.gks + kvh * (long)p.d * hw;
    T *gv = static_cast<T *>(p.gv) + w.n * p.gvs + kvh * (long)p.d * hw;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int b = 0; b < G::DT; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = b * 32 + 8 * (i / 4) + 4 * half + i % 4;
                if (there[u] && c < p.d) {
                    gk[c * hw + pixel[u]] = narrow<T>(ok[u] ? dk[u][b][i] * p.scale : 0.f);
                    gv[c * hw + pixel[u]] = narrow<T>(ok[u] ? dv[u][b][i] : 0.f);
                }
            }
}

// Sums of equal offsets over every `splits`-th block's table, in order.
__global__ __launch_bounds__(256) void window_offsets_kernel(const WindowParams p)
{
    const int at = blockIdx.x * 256 + threadIdx.x, head = blockIdx.y;
    if (at >= p.th * p.tw) return;
    const int centre = (p.wh - 1) * p.tw + p.ww - 1;
    float sum = 0.f;
    for (int i = blockIdx.z; i < p.units / p.heads; i += p.splits) {
        const int block = i % p.blocks, wi = i / p.blocks;
        const Win w = win_of(p, wi / (p.gy * p.gx), wi / p.gx % p.gy, wi % p.gx);
        const int q0 = block * p.waves * kWinWaveTokens;
        if (q0 >= w.L) continue;
        const TableRange r = table_range(q0, min(q0 + p.waves * kWinWaveTokens, w.L), w.h, w.wp, p.tw, centre, -1);
        const int in = at - r.base;
        if (in >= 0 && in < r.len) sum += p.part[((long)(wi * p.heads + head) * p.blocks + block) * p.len + in];
    }
    p.part2[((long)blockIdx.z * p.heads + head) * p.th * p.tw + at] = sum;
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

// A wavefront for each bucket: the sums of its offsets.
__global__ __launch_bounds__(256) void window_buckets_kernel(const WindowParams p)
{
    const int b = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y, lane = threadIdx.x & 63;
    if (b >= p.nby * p.nbx) return;
    int y0, y1, x0, x1;
    bucket_range(p, b / p.nbx, p.win_h, p.wh, &y0, &y1);
    bucket_range(p, b % p.nbx, p.win_w, p.ww, &x0, &x1);
    const int cols = x1 - x0 + 1, count = y1 >= y0 && cols > 0 ? (y1 - y0 + 1) * cols * p.splits : 0;
    float sum = 0.f;
    for (int i = lane; i < count; i += 64) {
        const int split = i % p.splits, o = i / p.splits, y = y0 + o / cols, x = x0 + o % cols;
        sum += p.part2[((long)split * p.heads + head) * p.th * p.tw + (y + p.wh - 1) * p.tw + x + p.ww - 1];
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) {
        float *to = p.grad_bias + (long)head * p.nby * p.nbx + b;
        *to = p.accumulate != 0 ? *to + sum : sum;
    }
}

template <typename T, int DP>
size_t dq_lds(int len, int tables)
{
    using G = WinGeom<T, DP>;
    return 2 * G::RM_BYTES + G::CM_BYTES + (G::TK / 4) * 5 + (size_t)len * 4 * (1 + tables);
}
template <typename T, int DP>
size_t dkv_lds(int len)
{
    using G = WinGeom<T, DP>;
    return 2 * (G::RM_BYTES + G::CM_BYTES) + G::TK * 12 + (G::TK / 4) * 5 + 4 + (size_t)len * 4;
}

hipError_t allow(const void *kernel, size_t lds)
{
    return lds <= 64 * 1024 ? hipSuccess : hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
}

template <typename T, int DP>
hipError_t launch_dq(const WindowParams &p, hipStream_t s)
{
    const size_t lds = dq_lds<T, DP>(p.len, p.grad_bias != nullptr ? p.waves : 0);
    const hipError_t e = allow(reinterpret_cast<const void *>(&window_dq_kernel<T, DP>), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_dq_kernel<T, DP>), dim3((unsigned)((p.units + 7) / 8 * 8)), dim3(64 * p.waves), lds, s, p);
    return hipGetLastError();
}
template <typename T, int DP>
hipError_t launch_dkv(const WindowParams &p, hipStream_t s)
{
    const size_t lds = dkv_lds<T, DP>(p.len);
    const hipError_t e = allow(reinterpret_cast<const void *>(&window_dkv_kernel<T, DP>), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_dkv_kernel<T, DP>), dim3((unsigned)((p.units + 7) / 8 * 8)), dim3(64 * p.waves), lds, s, p);
    return hipGetLastError();
}

}  // namespace

size_t window_dq_lds(bool f32, int dp, int len, int waves, bool bias_grad)
{
    const int tables = bias_grad ? waves : 0;
    if (f32) return dp == 16 ? dq_lds<float, 16>(len, tables) : dp == 32 ? dq_lds<float, 32>(len, tables) : dq_lds<float, 64>(len, tables);
    return dp == 16 ? dq_lds<uint16_t, 16>(len, tables) : dp == 32 ? dq_lds<uint16_t, 32>(len, tables) : dq_lds<uint16_t, 64>(len, tables);
}

size_t window_dkv_lds(bool f32, int dp, int len)
{
    if (f32) return dp == 16 ? dkv_lds<float, 16>(len) : dp == 32 ? dkv_lds<float, 32>(len) : dkv_lds<float, 64>(len);
    return dp == 16 ? dkv_lds<uint16_t, 16>(len) : dp == 32 ? dkv_lds<uint16_t, 32>(len) : dkv_lds<uint16_t, 64>(len);
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
    hipLaunchKernelGGL(window_offsets_kernel, dim3((unsigned)((p.th * p.tw + 255) / 256), (unsigned)p.heads, (unsigned)p.splits), dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(window_buckets_kernel, dim3((unsigned)((p.nby * p.nbx + 3) / 4), (unsigned)p.heads), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace esc
