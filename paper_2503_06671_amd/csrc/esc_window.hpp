// Window attention with a learned relative position bias: what its forward (esc_window_forward.hip), its backward
// (esc_window_backward.hip) and the host side (esc_window.hip) share.
//
// Tokens.  A window's pixels are numbered row by row, rows padded to whole pairs, so that the two tokens of a pair always
// lie side by side in one row; a window at the map's edge is cut to the map first, so that only the padding is lost.  Pixels
// beyond the row, beyond the last token and those that the mask hides are zeros in every operand.
//
// Offsets.  With off(t) = y(t) * tw + x(t), tw = 2 w - 1 (w the window's own width), the offset of a key from a query has the number
// off(key) - off(query) + centre, a sum of two terms: the bias of a score is one read of a table of offsets in LDS, at a
// place that is linear in both tokens.  A block's queries see only the offsets of a range; that range alone is kept.
//
// Matrix instructions: v_mfma_f32_32x32x16_bf16.  bf16 storage as it is; fp32 values as three bf16 terms by truncation (exact),
// the six products of terms whose orders add up to two at most (what is left out: below 2^-21 of a product, 2^-24 on average).
// Where a branch lies between such an instruction and the first use of its result, the compiler has been seen to leave out the wait that
// the use needs.  The kernels keep branches away from there but for tiles that are not whole; tests/test_window_waits.py looks for such a use in the built code.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "esc_terms.hpp"

namespace esc {

// Exponentials are exp2(fma(score, log2(e) scale, -shift)), shift the rounded product for the row's largest score.  What that rounding takes or
// adds is the same for the row and falls out of the quotient, where what has been summed is rescaled by the rounded shifts' difference (shift_rest) - up to
// this size; larger ones subtract first (one operation more a score).
constexpr float kLargeShift = 0x1p20f;
// The backward pass rounds shift and logarithm of the sum to one number, which scales a row's probabilities by up to 2^-24 of that number: it subtracts
// first where shifts are beyond this.  1e-5 of a probability, as much as the rounding of scores of that size; at 2^16 it would be 2.7e-3.  Subtracting first
// costs 64 x 64 x 64 in bf16 40 % (1667 us, 2373 where a row of each block is beyond), so not from smaller shifts on.
constexpr float kLargeRow = 256.f;
// The running maximum that scores are taken relative to is followed only where one exceeds it by more than kSlack / (log2(e) scale), so that much, or its
// rounding to the scores' last place (twice the slack at most), a score may lie above the largest that the backward pass gets.
constexpr float kSlack = 8.f;
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
    void *rest;                          // bf16 storage: what rounding took from out (16 bits each)
    void *gq, *gk, *gv;
    long gqs, gks, gvs;
    float *delta;                        // [N, heads, H, W]: sum over d of out * grad_out
    float *part;                         // sums per offset of each block, `len` words
    float *part2;                        // the same of all blocks, [splits, heads, th * tw]
    float *grad_bias;
    const float *bias;                   // [heads, nby, nbx] or nullptr
    const uint8_t *mask;                 // [N, H, W] or nullptr
    const uint8_t *mask_read;            // what is read in its place where there is none (and not used), so that the loads need no condition
    long mask_step;
    uint32_t mask_set;                   // no mask: all bits
    int N, H, W, heads, kv_heads, d;
    int win_h, win_w;                    // as the table has them
    int wh, ww;                          // cut to the map
    int gy, gx;                          // windows down and across
    int tw, th;                          // offsets across and down of a whole window: 2 ww - 1, 2 wh - 1
    int nby, nbx, n_edges;
    int edges[kWinMaxEdges];
    int blocks, units, waves, len;       // blocks a window and head, all blocks, wavefronts a block, words of a block's table
    int run, grid;                       // how blocks go to the dies
    int owners;                          // so many of a block's wavefronts have tokens of their own (the others help staging)
    int tiles, ksplit;                   // tiles of 32 tokens of a wavefront; forward: wavefronts that share a tile's keys
    int buffers, ring, part_len;         // staging buffers; backward: words of a wavefront's ring (a power of two) and of its part
    int pairs;                           // planes have two pixels at least
    int splits, accumulate;
    float scale, inv_scale, log2_scale;  // scale * log2(e) last
};

// Wavefronts that a SIMD holds: of the forward's kernel with one tile a wavefront, by the registers it takes, and of the backward's, by those that their
// launch bounds leave them.
constexpr int window_forward_resident(bool f32, int dp) { return f32 ? (dp == 64 ? 2 : 3) : dp == 64 ? 3 : 4; }
constexpr int window_dq_resident(bool f32, int dp) { return f32 || dp == 64 ? 2 : 4; }
constexpr int window_dkv_resident(bool f32, int dp) { return f32 || dp == 64 ? 2 : 3; }

size_t window_forward_lds(const WindowParams &p, bool f32, int dp);  // (buffers, waves, ksplit and len set)
size_t window_dq_lds(const WindowParams &p, bool f32, int dp);  // (buffers, owners, ring, len and grad_bias set)
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
typedef int wi32x2 __attribute__((ext_vector_type(2)));

// Tokens staged at a time.
constexpr int win_chunk(bool f32, int dp) { return f32 ? (dp == 64 ? 32 : 64) : (dp == 16 ? 128 : 64); }

// The operands' shape: DP is the head's dimension rounded up to 16, 32 or 64.
template <typename T, int DP>
struct WinGeom {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int NT = F32 ? 3 : 1;
    static constexpr int TK = win_chunk(F32, DP);
    static constexpr int KS = DP / 16;                 // matrix instructions a score takes (of each pair of terms)
    static constexpr int DT = DP <= 32 ? 1 : 2;        // blocks of 32 channels of an output
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

// A window's row in tokens: whole pairs, which share the address of a bias (pairs, not fours: windows of 13 x 13 are 6 tiles and not 7; when
// it was tried, 307 us and not 391 for 3 x 339 x 511 bf16, and the additions cost windows of 32 and 48 2 %).
__host__ __device__ __forceinline__ int in_pairs(int width) { return (width + 1) & ~1; }

struct Win {
    int n, y0, x0, h, w, wp, L, tw, centre;
    float inv;
    // the row of a token: a quotient that is at least 0.5 / wp away from whole numbers, which the product's error (2^-22 of it) does not reach
    // below two million tokens
    __device__ __forceinline__ int row(int t) const { return (int)(((float)t + 0.5f) * inv); }
};

__device__ __forceinline__ Win win_of(const WindowParams &p, int n, int wy, int wx)
{
    Win w;
    w.n = n, w.y0 = wy * p.wh, w.x0 = wx * p.ww;
    w.h = min(p.wh, p.H - w.y0), w.w = min(p.ww, p.W - w.x0);
    w.wp = in_pairs(w.w);
    w.L = w.h * w.wp;
    w.tw = 2 * w.w - 1, w.centre = (p.wh - 1) * w.tw + w.w - 1;
    w.inv = __builtin_amdgcn_rcpf((float)w.wp);
    return w;
}

// The block's place in the work: the dies, which blocks go to one after the other, take runs of it in turn.
__device__ __forceinline__ int unit_of(const WindowParams &p)
{
    const int i = blockIdx.x >> 3, r = i / p.run, u = (r * 8 + (blockIdx.x & 7)) * p.run + i - r * p.run;
    return u < p.units ? u : -1;
}

// Range of offsets that the tokens [t0, t1) of a window see of all its tokens: first number (theirs subtracted), words.
struct TableRange {
    int base, len;
};
// `sign`: -1 for queries (offset = key - query), 1 for keys.  off() grows with the token, but in windows of one column, whose
// rows of two overlap: there whole rows count.
__device__ __forceinline__ TableRange table_range(const Win &w, int t0, int t1, int sign)
{
    const int wp = w.wp, tw = w.tw, centre = w.centre, y0 = w.row(t0), y1 = w.row(t1 - 1), all = (w.h - 1) * tw + wp - 1;
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
// infinity stays one).  REVERSED: last first, for lanes that hold a key and go through queries.  Four loads on their way at a time.
template <bool REVERSED>
__device__ __forceinline__ void stage_table(const WindowParams &p, const Win &w, float *table, TableRange r, int head)
{
    const float *bias = p.bias + (long)head * p.nby * p.nbx, inv_tw = __builtin_amdgcn_rcpf((float)w.tw);
    for (int i0 = threadIdx.x; i0 < r.len; i0 += 4 * blockDim.x) {
        float b[4];
        bool in[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = r.base + i0 + k * blockDim.x;
            in[k] = at >= 0 && at < p.th * w.tw;
            const int c = in[k] ? at : 0, y = (int)(((float)c + 0.5f) * inv_tw), x = c - y * w.tw;  // (as Win::row)
            const int by = bucket_of(p, y - (p.wh - 1), p.win_h), bx = bucket_of(p, x - (w.w - 1), p.win_w);
            b[k] = p.bias != nullptr ? bias[(long)by * p.nbx + bx] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + k * blockDim.x;
            float v = in[k] ? b[k] : 0.f;
            if (__builtin_isfinite(v)) v = fminf(fmaxf(v * p.inv_scale, -0x1p120f), 0x1p120f);
            if (i < r.len) table[REVERSED ? r.len - 1 - i : i] = v;
        }
    }
}

// split_bf16's three terms of two values, in eleven instructions: the halves are taken from the values as they are.
__device__ __forceinline__ void three_terms(float v0, float v1, uint32_t (&t)[3])
{
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const uint32_t a = __float_as_uint(v0), b = __float_as_uint(v1);
        t[q] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        if (q < 2) v0 -= __uint_as_float(a & 0xffff0000u), v1 -= __uint_as_float(b & 0xffff0000u);
    }
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Where a group of tokens t ... lies in its image's planes: `at`, which `near` brings so far from the plane's end that `n` elements can be read
// from there, and how many of them to skip then; which of the n tokens exist (but for the mask).
struct Spot {
    int at, skip;
    uint32_t bits;
    Spot() = default;
    __device__ __forceinline__ Spot(const WindowParams &p, const Win &w, int t, int n)
    {
        const int y = w.row(t), x = t - y * w.wp;
        const bool in = t < w.L;
        const int pos = in ? (w.y0 + y) * p.W + w.x0 + x : 0;
        at = max(min(pos, p.H * p.W - n), 0), skip = pos - at;
        bits = in ? (1u << max(min(w.w - x, n), 0)) - 1 : 0u;
    }
};

// Offsets of pairs of tokens, in bytes of a table of floats.
template <int TK>
__device__ __forceinline__ void stage_offsets(const WindowParams &p, const Win &w, int t0, int *off)
{
    if (threadIdx.x >= TK / 2) return;
    const int t = t0 + 2 * threadIdx.x, y = w.row(t), x = t - y * w.wp;
    off[threadIdx.x] = t < w.L ? 4 * (y * w.tw + x) : 0;
}

// A lane's 16 tokens of a staged tile, of which those whose pair's bit is not set get `none`.  bits: a byte for each pair of tokens.
__device__ __forceinline__ bool all_take_part(wu32x4 bits)
{
    return __builtin_amdgcn_readfirstlane((int)(bits.x & bits.y & bits.z & bits.w)) == 0x03030303;
}
__device__ __forceinline__ void leave_out(wu32x4 bits, float none, wf32x16 &s)
{
    // (called where a tile is not whole: the compiler would work out the sixteen conditions for every tile)
    asm volatile("; tokens that do not take part" : "+v"(bits));
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const uint32_t b = bits[a] >> 16 * half;
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * a + j] = (b >> (8 * (j / 2) + j % 2) & 1) != 0 ? s[4 * a + j] : none;
    }
}

// Two tokens of four channels of one operand on their way from memory into LDS: as they come (fetch asks for nothing under a condition, so that
// nothing waits for an answer before `store`), and cleaned and laid out.  Reads need no alignment beyond the element's.
template <typename T, int DP>
struct Piece {
    using G = WinGeom<T, DP>;
    using Two = typename std::conditional<G::F32, wf32x2, uint32_t>::type;
    Two v[4];
    uint16_t mask;  // (two bytes)
    Spot spot;

    __device__ __forceinline__ void fetch(const WindowParams &p, const Win &w, const T *plane, int t, int c4)
    {
        const long hw = (long)p.H * p.W;
        const Spot s = spot = Spot(p, w, t, 2);
        const T *a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = plane + min(c4 * 4 + i, p.d - 1) * hw + s.at;
        const uint8_t *m = p.mask_read + w.n * p.mask_step + s.at;
        if (p.pairs) {  // (uniform: not where a plane is one pixel)
#pragma unroll
            for (int i = 0; i < 4; ++i) __builtin_memcpy(&v[i], a[i], sizeof(Two));
            __builtin_memcpy(&mask, m, 2);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const T e[2] = {a[i][0], T(0)};
                __builtin_memcpy(&v[i], e, sizeof(Two));
            }
            mask = m[0];
        }
    }

    // g2: the pair within the staged tokens
    template <bool RM, bool CM>
    __device__ __forceinline__ void store(const WindowParams &p, char *rm, char *cm, uint8_t *bits, int g2, int c4) const
    {
        const Spot s = spot;
        const uint32_t m = (mask | p.mask_set) >> 8 * s.skip;  // (used in any case: a load whose answer is not used is waited for where its register is next)
        const bool ok0 = (s.bits & 1) != 0 && (m & 0xff) != 0, ok1 = (s.bits & 2) != 0 && (m & 0xff00) != 0;
        if (bits != nullptr && c4 == 0) bits[g2] = (uint8_t)((ok0 ? 1 : 0) | (ok1 ? 2 : 0));
        uint32_t word[G::NT][4];  // [term][channel]: both tokens
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool c = c4 * 4 + i < p.d;
            if constexpr (G::F32) {
                uint32_t q[3];
                three_terms(c && ok0 ? (s.skip != 0 ? v[i].y : v[i].x) : 0.f, c && ok1 ? v[i].y : 0.f, q);
#pragma unroll
                for (int k = 0; k < 3; ++k) word[k][i] = q[k];
            } else {
                const uint32_t x = s.skip != 0 ? v[i] >> 16 : v[i];
                word[0][i] = c ? x & ((ok0 ? 0xffffu : 0u) | (ok1 ? 0xffff0000u : 0u)) : 0u;
            }
        }
        const int g = g2 / 2, odd = g2 & 1;
#pragma unroll
        for (int k = 0; k < G::NT; ++k) {
            if constexpr (RM) {
                char *to = rm + ((k * G::RM_TERM + (c4 >> 1) * 4 * G::SLOT + odd * 2 * G::SLOT + g) * 16 + (c4 & 1) * 8);
                *reinterpret_cast<wu32x2 *>(to) = wu32x2{low_halves(word[k][0], word[k][1]), low_halves(word[k][2], word[k][3])};
                *reinterpret_cast<wu32x2 *>(to + G::SLOT * 16) = wu32x2{high_halves(word[k][0], word[k][1]), high_halves(word[k][2], word[k][3])};
            }
            if constexpr (CM) {
                const int place = (g & ~3) | ((g & 1) << 1) | ((g & 2) >> 1);
                char *to = cm + k * G::CM_TERM + c4 * 4 * G::CM_ROW + place * 8 + odd * 4;
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t *>(to + i * G::CM_ROW) = word[k][i];
            }
        }
    }
};

// Two operands staged a chunk of TK tokens at a time into two buffers in turn.  A block's threads fetch the next chunk into registers before
// they multiply this one (a piece each; where a block has so few threads that there are more pieces, the rest follows behind).
template <typename T, int DP, bool RM0, bool CM0, bool RM1, bool CM1>
struct Stager {
    using G = WinGeom<T, DP>;
    static constexpr int PAIRS = G::TK / 2;
    static constexpr int RM0_AT = 0, CM0_AT = RM0_AT + (RM0 ? G::RM_BYTES : 0), RM1_AT = CM0_AT + (CM0 ? G::CM_BYTES : 0),
                         CM1_AT = RM1_AT + (RM1 ? G::RM_BYTES : 0), BITS_AT = CM1_AT + (CM1 ? G::CM_BYTES : 0), OFF_AT = BITS_AT + PAIRS,
                         BYTES = (OFF_AT + PAIRS * 4 + 15) / 16 * 16;
    Piece<T, DP> next;

    // pieces of one operand: of the channels that exist (the others' place is cleared once)
    __device__ __forceinline__ static int half(const WindowParams &p) { return (p.d + 3) / 4 * PAIRS; }
    __device__ __forceinline__ static int pair_of(int item) { return item % PAIRS; }
    __device__ __forceinline__ static int channels_of(int item, int half) { return (item < half ? item : item - half) / PAIRS; }
    __device__ __forceinline__ static void put(const Piece<T, DP> &piece, const WindowParams &p, int item, char *buf)
    {
        const int h = half(p), g2 = pair_of(item), c4 = channels_of(item, h);
        if (item < h) piece.template store<RM0, CM0>(p, buf + RM0_AT, buf + CM0_AT, reinterpret_cast<uint8_t *>(buf + BITS_AT), g2, c4);
        else piece.template store<RM1, CM1>(p, buf + RM1_AT, buf + CM1_AT, nullptr, g2, c4);
    }
    __device__ __forceinline__ void fetch(const WindowParams &p, const Win &w, const T *op0, const T *op1, int t0)
    {
        const int h = half(p), item = min((int)threadIdx.x, 2 * h - 1);
        next.fetch(p, w, item < h ? op0 : op1, t0 + 2 * pair_of(item), channels_of(item, h));
    }
    __device__ __forceinline__ void write(const WindowParams &p, const Win &w, const T *op0, const T *op1, int t0, char *buf)
    {
        const int h = half(p);
        if ((int)threadIdx.x < 2 * h) put(next, p, threadIdx.x, buf);
        for (int item = threadIdx.x + blockDim.x; item < 2 * h; item += blockDim.x) {
            Piece<T, DP> piece;
            piece.fetch(p, w, item < h ? op0 : op1, t0 + 2 * pair_of(item), channels_of(item, h));
            put(piece, p, item, buf);
            __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): all have come, but the compiler sees paths on which nobody waited
        }
        stage_offsets<G::TK>(p, w, t0, reinterpret_cast<int *>(buf + OFF_AT));
    }
    // What no piece writes, once for each buffer and in front of a barrier: zeros for the channels that do not exist, rows of ones (DP = 16).
    __device__ __forceinline__ static void clear(const WindowParams &p, char *buf)
    {
        if ((p.d + 3) / 4 * 4 < DP)
            for (int i = threadIdx.x; i < BITS_AT / 16; i += blockDim.x) reinterpret_cast<wu32x4 *>(buf)[i] = wu32x4{};
    }
    __device__ __forceinline__ static void ones(char *cm)
    {
        if constexpr (DP == 16)
            for (int i = threadIdx.x; i < G::NT * G::CM_ROW / 4; i += blockDim.x)
                *reinterpret_cast<uint32_t *>(cm + i / (G::CM_ROW / 4) * G::CM_TERM + 16 * G::CM_ROW + i % (G::CM_ROW / 4) * 4) = i < G::CM_ROW / 4 ? 0x3f803f80u : 0u;
    }
};

// A wavefront's own token: where it lies, whether it exists and takes part, its offset.  The loads need no condition (the place is one of the
// window's in any case), so that they can all be on their way before the first is waited for.
struct OwnToken {
    int pixel, off;
    bool there;
    uint8_t mask;
    __device__ __forceinline__ OwnToken(const WindowParams &p, const Win &w, int t)
    {
        const int tc = min(t, w.L - 1), y = w.row(tc), x = tc - y * w.wp;
        there = t < w.L && x < w.w;
        off = y * w.tw + x;
        pixel = (w.y0 + y) * p.W + w.x0 + min(x, w.w - 1);
        mask = p.mask_read[w.n * p.mask_step + pixel];
    }
    __device__ __forceinline__ bool ok(const WindowParams &p) const { return there && (mask | p.mask_set) != 0; }
};

// Eight channels 16 s + 8 (lane / 32) on of an own token, as they come ...
template <typename T, int DP>
struct OwnValues {
    T v[WinGeom<T, DP>::KS][8];
    __device__ __forceinline__ void fetch(const WindowParams &p, const T *plane, int pixel)
    {
        const long hw = (long)p.H * p.W;
        const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
        for (int s = 0; s < WinGeom<T, DP>::KS; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[s][j] = plane[min(16 * s + 8 * half + j, p.d - 1) * hw + pixel];
    }
    __device__ __forceinline__ void clean(const WindowParams &p, bool ok)
    {
        const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
        for (int s = 0; s < WinGeom<T, DP>::KS; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[s][j] = ok && 16 * s + 8 * half + j < p.d ? v[s][j] : T(0);
    }
};
// ... and as an operand that stays in registers.
template <typename T, int DP>
struct Fragment {
    wu32x4 r[WinGeom<T, DP>::NT][WinGeom<T, DP>::KS];
};
template <typename T, int DP>
__device__ __forceinline__ Fragment<T, DP> fragment_of(const OwnValues<T, DP> &o)
{
    using G = WinGeom<T, DP>;
    Fragment<T, DP> f;
#pragma unroll
    for (int s = 0; s < G::KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const T a = o.v[s][2 * i], b = o.v[s][2 * i + 1];
            if constexpr (G::F32) {
                uint32_t t[3];
                three_terms(a, b, t);
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
            three_terms(v[2 * i], v[2 * i + 1], t);
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

// lanes l and l + 32 hold halves of a token's values: of both halves together
__device__ __forceinline__ float max_of_halves(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_of_halves(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// What rounding took from the shift of a row whose largest score is `top` (0 where scores subtract it first).
__device__ __forceinline__ float shift_rest(float top, float log2_scale)
{
    const float shift = top * log2_scale;
    return __builtin_fabsf(shift) > kLargeShift ? 0.f : __builtin_fmaf(top, log2_scale, -shift);
}

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ uint16_t to_bf16(float v)
{
    typedef __bf16 one;
    return __builtin_bit_cast(uint16_t, (one)v);
}
// What rounding v to r took from it, so that the two give v again: v's bits less those of r, 16 of them.  (v halfway between two, rounded down: 2^15 does
// not fit, one less does, 2^-24 off.)
__device__ __forceinline__ uint16_t taken_by_rounding(float v, uint16_t r)
{
    return (uint16_t)min((int)(__float_as_uint(v) - ((uint32_t)r << 16)), 0x7fff);
}
__device__ __forceinline__ float unrounded(uint16_t r, uint16_t taken) { return __uint_as_float(((uint32_t)r << 16) + (uint32_t)(int)(int16_t)taken); }
template <typename T>
__device__ __forceinline__ T narrow(float v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return to_bf16(v);
}

}  // namespace
}  // namespace esc
