// Window attention with a learned relative position bias: what its forward (esc_window_forward.hip), its backward
// (esc_window_backward.hip) and the host side (esc_window.hip) share.
//
// Tokens.  A window's pixels are numbered row by row, rows padded to a multiple of four, so that four consecutive tokens always
// lie side by side in one row; a window at the map's edge is cut to the map first, so that only the padding is lost.  Pixels
// beyond the row, beyond the last token and those that the mask hides are zeros in every operand.
//
// Offsets.  With off(t) = y(t) * tw + x(t), tw = 2 ww - 1, the offset of a key from a query has the number
// off(key) - off(query) + centre, a sum of two terms: the bias of a score is one read of a table of offsets in LDS, at a
// place that is linear in both tokens.  A block's queries see only the offsets of a range; that range alone is kept.
//
// Matrix instructions: v_mfma_f32_32x32x16_bf16.  bf16 storage as it is; fp32 values as three bf16 terms by truncation (exact),
// the six products of terms whose orders add up to two at most (what is left out lies below 2^-24 of a product).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "esc_terms.hpp"

namespace esc {

// Exponentials are exp2(fma(score, log2(e) scale, -shift)), shift the rounded product for the row's largest score.  What that rounding takes or
// adds is the same for the row and falls out of the quotient - up to this size; larger ones subtract first (one operation more a score).
constexpr float kLargeShift = 0x1p20f;
constexpr int kWinMaxEdges = 32;
constexpr int kWinMaxDim = 64;
constexpr int kWinMaxOffsets = 16384;
constexpr int kWinMaxWaves = 8;

struct WindowParams {
    const void *q, *k, *v;
    long qs, ks, vs;                     // from image to image, elements
    const void *out_in, *go;             // backward: the forward's result and its gradient
    void *out;
    float *top, *log_sum;                // [N, heads, H, W]: a row's largest score (unscaled), log2 of its sum of exponentials, +inf without keys
    void *rest;                          // bf16 storage: what rounding took from out
    void *gq, *gk, *gv;
    long gqs, gks, gvs;
    float *delta;                        // [N, heads, H, W]: sum over d of out * grad_out
    float *part;                         // sums per offset of each block, `len` words
    float *part2;                        // the same of all blocks, [splits, heads, th * tw]
    float *grad_bias;
    const float *bias;                   // [heads, nby, nbx] or nullptr
    const uint8_t *mask;                 // [N, H, W] or nullptr
    int N, H, W, heads, kv_heads, d;
    int win_h, win_w;                    // as the table has them
    int wh, ww;                          // cut to the map
    int gy, gx;                          // windows down and across
    int tw, th;                          // offsets across and down: 2 ww - 1, 2 wh - 1
    int nby, nbx, n_edges;
    int edges[kWinMaxEdges];
    int blocks, units, waves, len;       // blocks a window and head, all blocks, wavefronts a block, words of a block's table
    int tiles, ksplit;                   // tiles of 32 tokens of a wavefront; forward: wavefronts that share a tile's keys
    int buffers, ring, part_len;         // backward: staging buffers; words of a wavefront's ring (a power of two) and of its part
    int vec;                             // four pixels at a time
    int splits, accumulate;
    float scale, inv_scale, log2_scale;  // scale * log2(e) last
};

size_t window_forward_lds(bool f32, int dp, int len, int joined);  // joined: wavefronts whose sums are joined, or 0
int window_query_tiles(bool f32, int dp);
size_t window_dq_lds(const WindowParams &p, bool f32, int dp);  // (buffers, waves, ring, len and grad_bias set)
size_t window_dkv_lds(const WindowParams &p, bool f32, int dp);
hipError_t launch_window_forward(const WindowParams &p, bool f32, int dp, hipStream_t s);
hipError_t launch_window_dq(const WindowParams &p, bool f32, int dp, hipStream_t s);
hipError_t launch_window_dkv(const WindowParams &p, bool f32, int dp, hipStream_t s);
hipError_t launch_window_bias_grad(const WindowParams &p, hipStream_t s);

namespace {

typedef __bf16 wbf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 wbf16x2 __attribute__((ext_vector_type(2)));
typedef float wf32x16 __attribute__((ext_vector_type(16)));
typedef float wf32x4 __attribute__((ext_vector_type(4)));
typedef float wf32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t wu32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t wu32x2 __attribute__((ext_vector_type(2)));

// The operands' shape: DP is the head's dimension rounded up to 16, 32 or 64; TK tokens are staged at a time.
template <typename T, int DP>
struct WinGeom {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int NT = F32 ? 3 : 1;
    static constexpr int TK = F32 && DP == 64 ? 32 : 64;
    static constexpr int KS = DP / 16;                 // matrix instructions a score takes (of each pair of terms)
    static constexpr int DT = DP <= 32 ? 1 : 2;        // blocks of 32 channels of an output
#ifndef DQT
#define DQT 2
#endif
    static constexpr int QUERY_TILES = F32 || DP == 64 ? 1 : DQT;  // backward: tiles of 32 own queries of a wavefront (two where the registers hold them); its keys: one
    // rows of tokens: 16-byte pieces of eight channels, [term][channels / 8][token]; four tokens of a group lie SLOT pieces
    // apart, so that 16 lanes' pieces cover all banks once, written and read
    static constexpr int SLOT = TK / 4 + 4;
    static constexpr int RM_TERM = (DP / 8) * 4 * SLOT;
    static constexpr int RM_BYTES = NT * RM_TERM * 16;
    // rows of channels: [term][channel][token], the groups of four in the order 0 2 1 3 of each sixteen (the order in which
    // a lane of the score's result holds them).  DP = 16 leaves half of the matrix's rows free: a row of ones there gives sums over
    // the tokens.
    static constexpr int CM_ROW = TK * 2 + 16;
    static constexpr int CM_ROWS = DP == 16 ? 17 : DP;
    static constexpr int CM_TERM = CM_ROWS * CM_ROW;
    static constexpr int CM_BYTES = NT * CM_TERM;
};

struct Win {
    int n, y0, x0, h, w, wp, L;
};

__device__ __forceinline__ Win win_of(const WindowParams &p, int n, int wy, int wx)
{
    Win w;
    w.n = n, w.y0 = wy * p.wh, w.x0 = wx * p.ww;
    w.h = min(p.wh, p.H - w.y0), w.w = min(p.ww, p.W - w.x0);
    w.wp = (w.w + 3) & ~3;
    w.L = w.h * w.wp;
    return w;
}

// The block's place in the work: dies take contiguous eighths, so that the blocks of one window meet in one L2.
__device__ __forceinline__ int unit_of(int units)
{
    const int per = (units + 7) / 8, i = blockIdx.x >> 3;
    const int u = (blockIdx.x & 7) * per + i;
    return i < per && u < units ? u : -1;
}

// Range of offsets that the tokens [t0, t1) of a window see of all its tokens: first number (theirs subtracted), words.
struct TableRange {
    int base, len;
};
// `sign`: -1 for queries (offset = key - query), 1 for keys.  off() grows with the token, but in windows of one and two columns, whose
// rows of four overlap: there whole rows count.
__device__ __forceinline__ TableRange table_range(int t0, int t1, int h, int wp, int tw, int centre, int sign)
{
    const int y0 = t0 / wp, y1 = (t1 - 1) / wp, all = (h - 1) * tw + wp - 1;
    const int lo = y0 * tw + (tw >= wp ? t0 - y0 * wp : 0), hi = y1 * tw + (tw >= wp ? t1 - 1 - y1 * wp : wp - 1);
    return sign < 0 ? TableRange{centre - hi, all + hi - lo + 1} : TableRange{centre + lo - all, all + hi - lo + 1};
}

__device__ __forceinline__ int bucket_of(const WindowParams &p, int o, int full)
{
    if (p.n_edges == 0) return o + full - 1;
    const int a = o < 0 ? -o : o;
    int lo = 0, hi = p.n_edges;  // how many edges are <= a
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (p.edges[mid] <= a) lo = mid + 1;
        else hi = mid;
    }
    return p.n_edges + (o < 0 ? -lo : lo);
}

// The range of the head's table, over the scale (scores are kept unscaled; the largest magnitudes are cut to 2^120, an
// infinity stays one).
__device__ __forceinline__ void stage_table(const WindowParams &p, float *table, TableRange r, int head)
{
    for (int i = threadIdx.x; i < r.len; i += blockDim.x) {
        const int at = r.base + i;
        float b = 0.f;
        if (p.bias != nullptr && at >= 0 && at < p.th * p.tw) {
            const int y = at / p.tw, x = at - y * p.tw;
            const int by = bucket_of(p, y - (p.wh - 1), p.win_h), bx = bucket_of(p, x - (p.ww - 1), p.win_w);
            b = p.bias[((long)head * p.nby + by) * p.nbx + bx];
            if (__builtin_isfinite(b)) b = fminf(fmaxf(b * p.inv_scale, -0x1p120f), 0x1p120f);
        }
        table[i] = b;
    }
}

// Does the pixel exist and take part?
__device__ __forceinline__ bool seen(const WindowParams &p, const Win &w, int y, int x)
{
    return y < w.h && x < w.w && (p.mask == nullptr || p.mask[((long)w.n * p.H + w.y0 + y) * p.W + w.x0 + x] != 0);
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Offsets (of groups of four tokens) and the bits of those that take part.
template <int TK>
__device__ __forceinline__ void stage_tokens(const WindowParams &p, const Win &w, int t0, int *off, uint8_t *bits)
{
    const int g = threadIdx.x;
    if (g >= TK / 4) return;
    const int t = t0 + 4 * g;
    int o = 0, b = 0;
    if (t < w.L) {
        const int y = t / w.wp, x = t - y * w.wp;
        o = y * p.tw + x;
        for (int j = 0; j < 4; ++j) b |= seen(p, w, y, x + j) ? 1 << j : 0;
    }
    off[g] = o;
    bits[g] = (uint8_t)b;
}

// Four tokens of eight channels of one operand on their way from memory into LDS.
template <typename T, int DP>
struct Piece {
    using G = WinGeom<T, DP>;
    using Four = typename std::conditional<G::F32, wf32x4, wu32x2>::type;
    Four v[8];

    // tokens t ... t + 3 of the channels from 8 * d8 on; `plane` is channel 0 of the head's planes of this image
    __device__ __forceinline__ void load(const WindowParams &p, const Win &w, const T *plane, int t, int d8)
    {
        const long hw = (long)p.H * p.W;
        const int y = t / w.wp, x = t - y * w.wp;
        const bool in = t < w.L;
        const T *at = plane + (in ? (long)(w.y0 + y) * p.W + w.x0 + x : 0) + (long)(d8 * 8) * hw;
        bool ok[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) ok[j] = in && x + j < w.w;
        if (p.vec) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = Four{};
                if (in && d8 * 8 + i < p.d) v[i] = *reinterpret_cast<const Four *>(at + i * hw);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                T e[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) e[j] = ok[j] && d8 * 8 + i < p.d ? at[i * hw + j] : T(0);
                __builtin_memcpy(&v[i], e, sizeof(Four));
            }
        }
        if (p.mask != nullptr) {
            const uint8_t *m = p.mask + ((long)w.n * p.H + w.y0 + y) * p.W + w.x0 + x;
#pragma unroll
            for (int j = 0; j < 4; ++j) ok[j] = ok[j] && m[j] != 0;
        }
        if (!(ok[0] && ok[1] && ok[2] && ok[3])) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (G::F32) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i][j] = ok[j] ? v[i][j] : 0.f;
                } else {
                    v[i].x &= (ok[0] ? 0xffffu : 0u) | (ok[1] ? 0xffff0000u : 0u);
                    v[i].y &= (ok[2] ? 0xffffu : 0u) | (ok[3] ? 0xffff0000u : 0u);
                }
            }
        }
    }

    // g: the group of four within the staged tokens
    template <bool RM, bool CM>
    __device__ __forceinline__ void store(char *rm, char *cm, int g, int d8) const
    {
        uint32_t word[G::NT][8][2];  // [term][channel][pair of tokens]
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (G::F32) {
                uint32_t t01[3], t23[3];
                split_bf16(v[i][0], v[i][1], t01);
                split_bf16(v[i][2], v[i][3], t23);
#pragma unroll
                for (int q = 0; q < 3; ++q) word[q][i][0] = t01[q], word[q][i][1] = t23[q];
            } else {
                word[0][i][0] = v[i].x, word[0][i][1] = v[i].y;
            }
        }
#pragma unroll
        for (int q = 0; q < G::NT; ++q) {
            if constexpr (RM) {
                wu32x4 *to = reinterpret_cast<wu32x4 *>(rm) + q * G::RM_TERM + d8 * 4 * G::SLOT + g;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    wu32x4 r;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        r[i] = j % 2 == 0 ? low_halves(word[q][2 * i][j / 2], word[q][2 * i + 1][j / 2]) : high_halves(word[q][2 * i][j / 2], word[q][2 * i + 1][j / 2]);
                    to[j * G::SLOT] = r;
                }
            }
            if constexpr (CM) {
                const int place = (g & ~3) | ((g & 1) << 1) | ((g & 2) >> 1);
                char *to = cm + q * G::CM_TERM + d8 * 8 * G::CM_ROW + place * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i) *reinterpret_cast<wu32x2 *>(to + i * G::CM_ROW) = wu32x2{word[q][i][0], word[q][i][1]};
            }
        }
    }
};

// Two operands staged a chunk of TK tokens at a time into two buffers in turn.  A block's threads fetch the next chunk into registers before
// they multiply this one (as many pieces as there are threads; where a block has fewer threads, the rest follows behind).
template <typename T, int DP, bool RM0, bool CM0, bool RM1, bool CM1>
struct Stager {
    using G = WinGeom<T, DP>;
    static constexpr int GROUPS = G::TK / 4;
    static constexpr int ITEMS = 2 * (DP / 8) * GROUPS;
    static constexpr int RM0_AT = 0, CM0_AT = RM0_AT + (RM0 ? G::RM_BYTES : 0), RM1_AT = CM0_AT + (CM0 ? G::CM_BYTES : 0),
                         CM1_AT = RM1_AT + (RM1 ? G::RM_BYTES : 0), OFF_AT = CM1_AT + (CM1 ? G::CM_BYTES : 0), BITS_AT = OFF_AT + GROUPS * 4,
                         BYTES = (BITS_AT + GROUPS + 15) / 16 * 16;
    Piece<T, DP> next;

    __device__ __forceinline__ static void place(int item, int *which, int *g, int *d8)
    {
        *which = item / (ITEMS / 2);
        const int i = item % (ITEMS / 2);
        *g = i % GROUPS, *d8 = i / GROUPS;
    }
    __device__ __forceinline__ static void put(const Piece<T, DP> &piece, int item, char *buf)
    {
        int which, g, d8;
        place(item, &which, &g, &d8);
        if (which == 0) piece.template store<RM0, CM0>(buf + RM0_AT, buf + CM0_AT, g, d8);
        else piece.template store<RM1, CM1>(buf + RM1_AT, buf + CM1_AT, g, d8);
    }
    __device__ __forceinline__ void fetch(const WindowParams &p, const Win &w, const T *op0, const T *op1, int t0)
    {
        int which, g, d8;
        const int item = threadIdx.x;
        if (item < ITEMS) {
            place(item, &which, &g, &d8);
            next.load(p, w, which == 0 ? op0 : op1, t0 + 4 * g, d8);
        }
    }
    __device__ __forceinline__ void write(const WindowParams &p, const Win &w, const T *op0, const T *op1, int t0, char *buf)
    {
        if ((int)threadIdx.x < ITEMS) put(next, threadIdx.x, buf);
        for (int item = threadIdx.x + blockDim.x; item < ITEMS; item += blockDim.x) {
            int which, g, d8;
            place(item, &which, &g, &d8);
            Piece<T, DP> piece;
            piece.load(p, w, which == 0 ? op0 : op1, t0 + 4 * g, d8);
            put(piece, item, buf);
        }
        stage_tokens<G::TK>(p, w, t0, reinterpret_cast<int *>(buf + OFF_AT), reinterpret_cast<uint8_t *>(buf + BITS_AT));
    }
    // the rows of ones (DP = 16), once for each buffer
    __device__ __forceinline__ static void ones(char *cm)
    {
        if constexpr (DP == 16)
            for (int i = threadIdx.x; i < G::NT * G::CM_ROW / 4; i += blockDim.x)
                *reinterpret_cast<uint32_t *>(cm + i / (G::CM_ROW / 4) * G::CM_TERM + 16 * G::CM_ROW + i % (G::CM_ROW / 4) * 4) = i < G::CM_ROW / 4 ? 0x3f803f80u : 0u;
    }
};

// A wavefront's own tokens as operands kept in registers: lane n = token, eight channels 16 s + 8 (lane / 32) on.
template <typename T, int DP>
struct Fragment {
    wu32x4 r[WinGeom<T, DP>::NT][WinGeom<T, DP>::KS];
};
template <typename T, int DP>
__device__ __forceinline__ Fragment<T, DP> own_fragment(const WindowParams &p, const T *pixel, bool ok)
{
    using G = WinGeom<T, DP>;
    Fragment<T, DP> f;
    const long hw = (long)p.H * p.W;
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int s = 0; s < G::KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 16 * s + 8 * half + 2 * i;
            const T a = ok && c < p.d ? pixel[c * hw] : T(0), b = ok && c + 1 < p.d ? pixel[(c + 1) * hw] : T(0);
            if constexpr (G::F32) {
                uint32_t t[3];
                split_bf16(a, b, t);
#pragma unroll
                for (int q = 0; q < 3; ++q) f.r[q][s][i] = t[q];
            } else {
                f.r[0][s][i] = (uint32_t)a | (uint32_t)b << 16;
            }
        }
    return f;
}

__device__ __forceinline__ wf32x16 mfma(wu32x4 a, wu32x4 b, wf32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(wbf16x8, a), __builtin_bit_cast(wbf16x8, b), c, 0, 0, 0);
}

// c + rows (32 tokens of a staged operand) x own tokens, over the channels.  OWN_FIRST: the pairs of terms in the order in which the call with the
// operands' roles exchanged has them, so that both orientations of a score give the same bits.
template <typename T, int DP, bool OWN_FIRST = false>
__device__ __forceinline__ wf32x16 score(const char *rm, int tile, const Fragment<T, DP> &own, wf32x16 c)
{
    using G = WinGeom<T, DP>;
    const int lane = threadIdx.x & 63, m = lane & 31, half = lane >> 5;
    const wu32x4 *from = reinterpret_cast<const wu32x4 *>(rm) + half * 4 * G::SLOT + (m & 3) * G::SLOT + tile * 8 + (m >> 2);
#pragma unroll
    for (int s = 0; s < G::KS; ++s) {
        wu32x4 a[G::NT];
#pragma unroll
        for (int q = 0; q < G::NT; ++q) a[q] = from[q * G::RM_TERM + s * 8 * G::SLOT];
#pragma unroll
        for (int q = 0; q < G::NT; ++q)
#pragma unroll
            for (int r = 0; r + q < G::NT; ++r) c = OWN_FIRST ? mfma(a[r], own.r[q][s], c) : mfma(a[q], own.r[r][s], c);
    }
    return c;
}

// The score's result as the next product's right operand: a lane holds its token's values at 16 of the tile's 32 rows,
// 16 a + 8 (j / 4) + 4 (lane / 32) + j % 4 for the j-th of the a-th eight - the order in which rows of channels are staged.
template <int NT>
struct Packed {  // one term: to the nearest; two: what rounding took as a second; three: exact
    wu32x4 r[NT][2];
};
template <int NT>
__device__ __forceinline__ Packed<NT> pack(const wf32x16 &v)
{
    Packed<NT> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (NT < 3) {
            const float a = v[2 * i], b = v[2 * i + 1];
            const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector(wf32x2{a, b}, wbf16x2));
            o.r[0][i / 4][i % 4] = h;
            if constexpr (NT == 2)
                o.r[1][i / 4][i % 4] = __builtin_bit_cast(
                    uint32_t, __builtin_convertvector(wf32x2{a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xffff0000u)}, wbf16x2));
        } else {
            uint32_t t[3];
            split_bf16(v[2 * i], v[2 * i + 1], t);
#pragma unroll
            for (int q = 0; q < 3; ++q) o.r[q][i / 4][i % 4] = t[q];
        }
    }
    return o;
}

// acc += rows of channels x the tile's values (VT terms of them), of U tiles of own tokens.  DP = 16: the matrix's rows from 16 on take the row
// of ones.
// fp32 storage: the tile's products are summed by themselves first, so that a long sum takes one rounding a tile and not one
// for each pair of terms (1024 keys: 1.0e-6 off the exact result instead of 3e-7 with the products added one by one).
template <typename T, int DP, int VT, int U>
__device__ __forceinline__ void accumulate(const char *cm, int tile, const Packed<VT> (&v)[U], wf32x16 (&acc)[U][WinGeom<T, DP>::DT])
{
    using G = WinGeom<T, DP>;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int row = DP == 16 ? min(lane & 31, 16) : lane & 31;
    const char *from = cm + row * G::CM_ROW + tile * 64 + half * 16;
#pragma unroll
    for (int b = 0; b < G::DT; ++b) {
        wf32x16 sum[U];
#pragma unroll
        for (int u = 0; u < U; ++u) sum[u] = G::F32 ? wf32x16{} : acc[u][b];
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int q = G::NT - 1; q >= 0; --q) {
                const wu32x4 x = *reinterpret_cast<const wu32x4 *>(from + q * G::CM_TERM + b * 32 * G::CM_ROW + a * 32);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int r = VT - 1; r >= 0; --r)
                        if (!G::F32 || r + q < G::NT) sum[u] = mfma(x, v[u].r[r][a], sum[u]);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (G::F32) acc[u][b] += sum[u];
            else acc[u][b] = sum[u];
        }
    }
}

// (lanes l and l + 32 hold halves of a token's values)
__device__ __forceinline__ float other_half(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((threadIdx.x & 32) != 0 ? s[0] : s[1]);
}

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ uint16_t to_bf16(float v)
{
    typedef __bf16 one;
    return __builtin_bit_cast(uint16_t, (one)v);
}
template <typename T>
__device__ __forceinline__ T narrow(float v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return to_bf16(v);
}

}  // namespace
}  // namespace esc
