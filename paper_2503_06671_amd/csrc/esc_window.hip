// Host side of window attention (esc_window_attention_* of include/esc_convattn.h): argument checks, geometry, launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "esc_convattn.h"
#include "esc_host.hpp"
#include "esc_window.hpp"

namespace {

using namespace esc;

constexpr size_t kAlign = 256;
constexpr size_t kLdsPerCu = 160 * 1024;
constexpr long kCus = 256, kSimds = 4 * kCus;

int dim_padded(int d) { return d <= 16 ? 16 : d <= 32 ? 32 : 64; }

// How far the offsets' numbers of `tokens` consecutive tokens of a window lie apart at most.
int span(const WindowParams &p, int width, long tokens)
{
    const int wp = in_pairs(width), tw = 2 * width - 1;
    const long rows = std::min<long>(p.wh - 1, (tokens - 1 + wp - 1) / wp);
    if (tw < wp) return (int)(rows * tw) + wp - 1;
    return (int)std::min<long>(tokens - 1 + rows * (tw - wp), (long)rows * tw + wp - 1);
}

// The most over the windows' widths (the last one of a row may be narrower) of f(width).
template <typename F>
int widest(const WindowParams &p, F f)
{
    return std::max(f(p.ww), f(p.W - (p.gx - 1) * p.ww));
}

// Words of the table of a block that has `tokens` tokens: their offsets to all tokens of any window of the map.
int table_words(const WindowParams &p, long tokens)
{
    return widest(p, [&](int width) { return (p.wh - 1) * (2 * width - 1) + in_pairs(width) + span(p, width, tokens); });
}

// Blocks of so many wavefronts that fit a compute unit whose SIMDs hold `simd` each.  A block's wavefronts go to the four in turn: five to eight take two
// places of each.
int places(int waves, int simd) { return waves < 4 ? 4 * simd / waves : simd / ((waves + 3) / 4); }

// The backward's wavefronts, up to eight a block and no more than leave a block for each compute unit, and its staging buffers.  What is weighed: how many
// wavefronts a compute unit holds (by LDS, and by registers), how many of the blocks' wavefronts have tokens, what a block's beginning and staging cost (as
// much as a wavefront's work),
// and that with one buffer nothing is on its way while a block multiplies (where there is more than one chunk).  Forward and gradients, bf16, dk and dv's
// kernel with three wavefronts a SIMD in blocks of four, and, counted as four a SIMD, of eight or five: 64 x 64 x 64, windows of 32: 1667 and 1744 us;
// 8 x 96 x 96, 6 heads of 32, windows of 24: 742 and 1007 us.
template <typename F>
bool choose_waves(WindowParams &p, int heads, bool f32, int dp, int simd, F lds)
{
    const long tokens = (long)p.wh * in_pairs(p.ww), windows = (long)p.N * p.gy * p.gx * heads;
    const long all = (tokens + 31) / 32;
    const int want = (int)std::max<long>(1, std::min({(long)kWinMaxWaves, all, all * windows / kCus}));
    const int most = tokens <= win_chunk(f32, dp) ? 1 : 2;
    auto take = [&](int owners, int buffers) {
        p.owners = owners, p.buffers = buffers, p.len = (table_words(p, owners * 32) + 3) & ~3;
        p.blocks = (int)((all + owners - 1) / owners);
    };
    float best = 0.f;
    int best_owners = 0, best_buffers = 0;
    for (int buffers = most; buffers >= 1; --buffers)
        for (int owners = want; owners >= 1; --owners) {
            take(owners, buffers);
            const int resident = (int)std::min<size_t>(kLdsPerCu / lds(p), places(owners, simd)) * owners;
            const float score = (float)resident * all / ((float)p.blocks * (owners + 1)) * (buffers < most ? 0.85f : 1.f);
            if (score > best) best = score, best_owners = owners, best_buffers = buffers;
        }
    if (best == 0.f) return false;
    take(best_owners, best_buffers);
    return true;
}

// All blocks, and how they go to the eight dies: in runs, so that what lies together meets in one L2 (heads that share keys; windows beside each
// other, whose rows share cache lines), and in many runs, so that no die gets all the windows that the map's edge cuts short (2 x 29 x 579, 3 heads of 33,
// windows of 21 x 13, gradients: 320 us, with one run a die 454).  Where there are few blocks, of few wavefronts, up to four help staging (6 heads of 48
// channels that share one key, 8 sequences of 969 in windows of 600, bf16, gradients: 390 us, without 720; with many blocks they only take
// room: 3 x 339 x 511, windows of 13: 833, without 349).
bool set_units(WindowParams &p, int heads)
{
    const __int128 all = (__int128)p.N * p.gy * p.gx * heads * p.blocks;
    if (all > 1 << 26) return false;
    const long units = (long)all, windows = (long)p.N * p.gy * p.gx, share = (long)(heads / p.kv_heads) * p.blocks;
    const long run = windows >= 64 ? windows / 64 * heads * p.blocks : windows * p.kv_heads >= 64 ? share : (units + 7) / 8;
    const long runs = (units + run - 1) / run;
    p.units = (int)units, p.run = (int)run, p.grid = (int)((runs + 7) / 8 * 8 * run);
    for (p.waves = p.owners; p.waves < 4 && units * p.waves < 2 * kSimds;) p.waves *= 2;
    return (size_t)p.grid * p.waves * 64 <= 0xffff0000u;  // (a launch has fewer than 2^32 lanes)
}

esc_status shape(const esc_window_attn *a, WindowParams *p)
{
    *p = WindowParams{};
    if (a->N < 1 || a->H < 1 || a->W < 1 || a->heads < 1 || a->kv_heads < 1 || a->head_dim < 1 || a->win_h < 1 || a->win_w < 1) return ESC_ERR_SHAPE;
    if (a->heads % a->kv_heads != 0) return ESC_ERR_SHAPE;
    if (a->head_dim > kWinMaxDim || a->heads > 1024 || a->win_h > 8192 || a->win_w > 8192) return ESC_ERR_UNSUPPORTED;
    if ((size_t)a->H * (size_t)a->W >= ((size_t)1 << 31)) return ESC_ERR_UNSUPPORTED;
    if ((__int128)a->N * a->heads * a->head_dim * a->H * a->W > (__int128)1 << 46) return ESC_ERR_UNSUPPORTED;  // (sizes in bytes stay far from 64 bits)
    if (a->n_edges < 0) return ESC_ERR_SHAPE;
    if (a->n_edges > kWinMaxEdges) return ESC_ERR_UNSUPPORTED;
    p->N = a->N, p->H = a->H, p->W = a->W, p->heads = a->heads, p->kv_heads = a->kv_heads, p->d = a->head_dim;
    p->win_h = a->win_h, p->win_w = a->win_w;
    p->wh = std::min(a->win_h, a->H), p->ww = std::min(a->win_w, a->W);
    p->gy = (a->H + p->wh - 1) / p->wh, p->gx = (a->W + p->ww - 1) / p->ww;
    p->pairs = a->H > 1 || a->W > 1;
    p->th = 2 * p->wh - 1, p->tw = 2 * p->ww - 1;
    if ((long)p->th * p->tw > kWinMaxOffsets) return ESC_ERR_UNSUPPORTED;
    p->n_edges = a->n_edges;
    p->nby = a->n_edges > 0 ? 2 * a->n_edges + 1 : 2 * a->win_h - 1;
    p->nbx = a->n_edges > 0 ? 2 * a->n_edges + 1 : 2 * a->win_w - 1;
    return ESC_OK;
}

size_t table_bytes(const WindowParams &p) { return (size_t)p.heads * p.nby * p.nbx * 4; }

// The forward's wavefronts.  A wavefront with two tiles of queries reads keys and values half as often, with one it takes so few registers that
// four of a SIMD hide each other's waits.  Two: fp32 storage, whose three terms make the reads dear (180 x 320, windows of 32: 174 us, with one
// 195), and bf16 storage in windows of fewer than 16 tiles, where a block's beginning weighs (3 x 339 x 511, windows of 13: 349 us, with one 550; windows of
// 48: 345, with one 308) - where a window has more than four tiles (4 x 171 x 171, windows of 9 x 9, fp32: 96 us, with one 81; 9 x 123 x 110, 8 heads, windows
// of 13 x 7, bf16: heads of 32 217, with one 185, heads of 16 128, with one 138) and the call leaves two wavefronts a SIMD.  Where even those are fewer than
// one a SIMD, up to four wavefronts, and no more than a chunk has tiles, share a tile's keys (64 x 64, 4 heads, windows of 32: heads of 16 in bf16 18.3 us
// with four, 23.8 with two, 30 without; in fp32 30 us with two, 40 without), and others help staging as long as there are pieces for them and all blocks
// are on the chip at once (heads of 64, bf16: 33 us, without 47).  Blocks are as large as leaves one for each compute unit: they stage a window's keys
// and values once for all their queries.
bool plan_forward(WindowParams &p, bool f32)
{
    const int dp = dim_padded(p.d);
    const long tokens = (long)p.wh * in_pairs(p.ww), each = (tokens + 31) / 32, windows = (long)p.N * p.gy * p.gx * p.heads;
    const long all = each * windows;
    p.tiles = (f32 ? dp < 64 : each < 16) && each > 4 && all >= 2 * 2 * kSimds ? 2 : 1;
    const long waves = (each + p.tiles - 1) / p.tiles;
    p.ksplit = 1;
    const int sharers = std::min(4, win_chunk(f32, dp) / 32);
    while (p.tiles == 1 && p.ksplit < sharers && waves * windows * p.ksplit < 2 * kSimds && tokens >= 128 * p.ksplit) p.ksplit *= 2;
    long queries = std::min<long>(kWinMaxWaves / p.ksplit, waves);
    queries = std::max<long>(1, std::min(queries, waves * windows / kCus));
    p.buffers = tokens <= win_chunk(f32, dp) ? 1 : 2;
    const int pieces = (p.d + 3) / 4 * win_chunk(f32, dp);  // (of keys and values, two tokens and four channels each)
    const auto on_a_cu = [&](int waves) { return (long)std::min<size_t>(kLdsPerCu / window_forward_lds(p, f32, dp), places(waves, window_forward_resident(f32, dp))); };
    for (; queries >= 1; --queries) {
        p.owners = (int)queries * p.ksplit;
        p.len = (table_words(p, (int)queries * p.tiles * 32) + 3) & ~3;
        if (window_forward_lds(p, f32, dp) <= kLdsPerCu) {
            p.blocks = (int)((waves + queries - 1) / queries);
            const long even = (waves + p.blocks - 1) / p.blocks;  // (equal blocks)
            if (even < queries) {
                queries = even + 1;
                continue;
            }
            if (!set_units(p, p.heads)) return false;
            while (p.ksplit > 1 && 2 * p.waves <= kWinMaxWaves && p.waves * 64 < pieces && p.units <= kCus * on_a_cu(2 * p.waves)) p.waves *= 2;
            return true;
        }
    }
    return false;
}
bool plan_dq(WindowParams &p, bool f32)
{
    const int dp = dim_padded(p.d);
    const int reach = widest(p, [&](int width) { return 2 * span(p, width, 32) + 1; });
    for (p.ring = 64; p.ring < reach;) p.ring *= 2;
    p.part_len = table_words(p, 32);
    // (the same plan with and without the table's gradient)
    float *const grad = p.grad_bias;
    p.grad_bias = reinterpret_cast<float *>(16);
    const bool fits = choose_waves(p, p.heads, f32, dp, window_dq_resident(f32, dp), [&](const WindowParams &x) { return window_dq_lds(x, f32, dp); });
    p.grad_bias = grad;
    if (!fits || !set_units(p, p.heads)) return false;
    // the sums over the windows: blocks for the whole card, sixteen windows each at least
    const long cells = (long)p.heads * ((p.th * p.tw + 1023) / 1024), all = (long)p.N * p.gy * p.gx;
    p.splits = (int)std::min(all, std::max<long>(64, std::min(4 * kCus / cells, all / 16)));
    return true;
}
bool plan_dkv(WindowParams &p, bool f32)
{
    const int dp = dim_padded(p.d);
    return choose_waves(p, p.kv_heads, f32, dp, window_dkv_resident(f32, dp), [&](const WindowParams &x) { return window_dkv_lds(x, f32, dp); }) &&
           set_units(p, p.kv_heads);
}

struct Scratch {
    size_t delta, part, part2, total;
};
Scratch scratch(const WindowParams &p)  // (of plan_dq)
{
    Scratch s;
    s.delta = 0;
    s.part = round_up((size_t)p.N * p.heads * p.H * p.W * 4, kAlign);
    s.part2 = s.part + round_up((size_t)p.units * p.owners * p.part_len * 4, kAlign);
    s.total = s.part2 + round_up((size_t)p.splits * p.heads * p.th * p.tw * 4, kAlign);
    return s;
}

// two planes of row values, and what rounding took from out
size_t rows_bytes(const WindowParams &p) { return round_up((size_t)p.N * p.heads * p.H * p.W * 8, kAlign); }
size_t saved_size(const WindowParams &p, esc_dtype dt)
{
    return rows_bytes(p) + (dt == ESC_BF16 ? round_up((size_t)p.N * p.heads * p.d * p.H * p.W * 2, kAlign) : 0);
}

// Planes of N images, `stride` bytes from image to image.
struct Images {
    const void *at;
    size_t stride, bytes;  // bytes: one image's
    int N;
    size_t extent() const { return (size_t)(N - 1) * stride + bytes; }
};

bool meet(const Images &a, const Images &b)
{
    if (!overlaps(a.at, a.extent(), b.at, b.extent())) return false;
    if (a.stride != b.stride || a.N == 1 || b.N == 1) return true;
    // the same step from image to image: parts of one tensor may lie between each other
    const uintptr_t ua = (uintptr_t)a.at, ub = (uintptr_t)b.at;
    const size_t s = a.stride, from = ub >= ua ? (ub - ua) % s : (s - (ua - ub) % s) % s;
    return from < a.bytes || from + b.bytes > s;
}
bool meets(const Images &a, const void *b, size_t bytes) { return b != nullptr && overlaps(a.at, a.extent(), b, bytes); }

// Checks what both directions take, and fills in the parameters.
esc_status common(const void *q, const void *k, const void *v, esc_dtype dt, const esc_window_attn *a, WindowParams *p, Images (&in)[3])
{
    if (a == nullptr) return ESC_ERR_NULL;
    if (dt != ESC_F32 && dt != ESC_BF16) return ESC_ERR_DTYPE;
    const esc_status st = shape(a, p);
    if (st != ESC_OK) return st;
    if (q == nullptr || k == nullptr || v == nullptr) return ESC_ERR_NULL;
    if (a->n_edges > 0) {
        if (a->edges == nullptr) return ESC_ERR_NULL;
        for (int i = 0; i < a->n_edges; ++i) {
            if (a->edges[i] < 1 || (i > 0 && a->edges[i] <= a->edges[i - 1])) return ESC_ERR_SHAPE;
            p->edges[i] = a->edges[i];
        }
    }
    if (!isfinite(a->scale) || !(a->scale > 0.f)) return ESC_ERR_SHAPE;
    if (a->scale < 0x1p-20f || a->scale > 64.f) return ESC_ERR_UNSUPPORTED;
    const size_t es = dt == ESC_F32 ? 4 : 2, plane = (size_t)p->H * p->W;
    const void *const ptr[3] = {q, k, v};
    const long stride[3] = {a->q_stride, a->k_stride, a->v_stride};
    for (int i = 0; i < 3; ++i) {
        const size_t one = (size_t)(i == 0 ? p->heads : p->kv_heads) * p->d * plane;
        if ((uintptr_t)ptr[i] % es != 0) return ESC_ERR_SHAPE;
        if (p->N > 1 && (stride[i] < 0 || (size_t)stride[i] < one || (size_t)stride[i] > ((size_t)1 << 46))) return ESC_ERR_SHAPE;
        in[i] = Images{ptr[i], p->N > 1 ? (size_t)stride[i] * es : one * es, one * es, p->N};
    }
    if ((uintptr_t)a->bias % 4 != 0) return ESC_ERR_SHAPE;
    p->q = q, p->k = k, p->v = v;
    p->qs = (long)(in[0].stride / es), p->ks = (long)(in[1].stride / es), p->vs = (long)(in[2].stride / es);
    p->bias = a->bias, p->mask = a->mask;
    // (without a mask, the first image of k: more bytes than a plane has pixels)
    p->mask_read = a->mask != nullptr ? a->mask : static_cast<const uint8_t *>(k), p->mask_step = a->mask != nullptr ? (long)plane : 0;
    p->mask_set = a->mask != nullptr ? 0 : 0xffff;
    p->scale = a->scale, p->inv_scale = 1.f / a->scale, p->log2_scale = (float)((double)a->scale * 1.4426950408889634);
    return ESC_OK;
}

}  // namespace

extern "C" {

size_t esc_window_attention_saved_bytes(const esc_window_attn *a, esc_dtype dt)
{
    WindowParams p;
    if (a == nullptr || (dt != ESC_F32 && dt != ESC_BF16) || shape(a, &p) != ESC_OK) return 0;
    return saved_size(p, dt);
}

size_t esc_window_attention_backward_workspace_bytes(const esc_window_attn *a)
{
    WindowParams p;
    size_t most = 0;
    for (bool f32 : {false, true}) {
        if (a == nullptr || shape(a, &p) != ESC_OK || !plan_dq(p, f32)) return 0;
        most = std::max(most, scratch(p).total);
    }
    return most;
}

esc_status esc_window_attention_forward(const void *q, const void *k, const void *v, esc_dtype dt, const esc_window_attn *a, void *out, void *saved,
                                        size_t saved_bytes, void *stream)
{
    WindowParams p;
    Images in[3];
    const esc_status st = common(q, k, v, dt, a, &p, in);
    if (st != ESC_OK) return st;
    if (out == nullptr) return ESC_ERR_NULL;
    const size_t es = dt == ESC_F32 ? 4 : 2;
    if ((uintptr_t)out % es != 0) return ESC_ERR_SHAPE;
    if (saved != nullptr && ((uintptr_t)saved % kAlign != 0 || saved_bytes < saved_size(p, dt))) return ESC_ERR_WORKSPACE;
    const Images o{out, in[0].bytes, in[0].bytes, p.N};
    const size_t mask_bytes = (size_t)p.N * p.H * p.W, sv = saved_size(p, dt);
    for (const Images &x : in)
        if (meet(o, x) || meets(x, saved, sv)) return ESC_ERR_ALIAS;
    if (meets(o, p.mask, mask_bytes) || meets(o, p.bias, table_bytes(p)) || meets(o, saved, sv)) return ESC_ERR_ALIAS;
    if (saved != nullptr && ((p.mask != nullptr && overlaps(saved, sv, p.mask, mask_bytes)) || (p.bias != nullptr && overlaps(saved, sv, p.bias, table_bytes(p)))))
        return ESC_ERR_ALIAS;
    p.out = out;
    if (saved != nullptr) {
        p.top = static_cast<float *>(saved);
        p.log_sum = p.top + (size_t)p.N * p.heads * p.H * p.W;
        p.rest = dt == ESC_BF16 ? static_cast<char *>(saved) + rows_bytes(p) : nullptr;
    }
    if (!plan_forward(p, dt == ESC_F32)) return ESC_ERR_UNSUPPORTED;
    return launch_window_forward(p, dt == ESC_F32, dim_padded(p.d), static_cast<hipStream_t>(stream)) == hipSuccess ? ESC_OK : ESC_ERR_HIP;
}

esc_status esc_window_attention_backward(const void *q, const void *k, const void *v, esc_dtype dt, const esc_window_attn *a, const void *out,
                                         const void *grad_out, const void *saved, size_t saved_bytes, const esc_window_grads *g, int accumulate,
                                         void *workspace, size_t workspace_bytes, void *stream)
{
    WindowParams p;
    Images in[3];
    const esc_status st = common(q, k, v, dt, a, &p, in);
    if (st != ESC_OK) return st;
    if (out == nullptr || grad_out == nullptr || saved == nullptr || g == nullptr || g->q == nullptr || g->k == nullptr || g->v == nullptr) return ESC_ERR_NULL;
    if (g->bias != nullptr && p.bias == nullptr) return ESC_ERR_NULL;
    const bool f32 = dt == ESC_F32;
    const size_t es = f32 ? 4 : 2;
    if ((uintptr_t)out % es != 0 || (uintptr_t)grad_out % es != 0 || (uintptr_t)g->bias % 4 != 0) return ESC_ERR_SHAPE;
    const size_t sv = saved_size(p, dt), mask_bytes = (size_t)p.N * p.H * p.W;
    if ((uintptr_t)saved % kAlign != 0 || saved_bytes < sv) return ESC_ERR_WORKSPACE;
    void *const gp[3] = {g->q, g->k, g->v};
    const long gstride[3] = {g->q_stride, g->k_stride, g->v_stride};
    Images written[3];
    for (int i = 0; i < 3; ++i) {
        if ((uintptr_t)gp[i] % es != 0) return ESC_ERR_SHAPE;
        if (p.N > 1 && (gstride[i] < 0 || (size_t)gstride[i] < in[i].bytes / es || (size_t)gstride[i] > ((size_t)1 << 46))) return ESC_ERR_SHAPE;
        written[i] = Images{gp[i], p.N > 1 ? (size_t)gstride[i] * es : in[i].bytes, in[i].bytes, p.N};
    }
    WindowParams pq = p, pk = p;
    if (!plan_dq(pq, f32) || !plan_dkv(pk, f32)) return ESC_ERR_UNSUPPORTED;
    const Scratch sc = scratch(pq);
    if (workspace == nullptr || (uintptr_t)workspace % kAlign != 0 || workspace_bytes < sc.total) return ESC_ERR_WORKSPACE;
    const Images o{out, in[0].bytes, in[0].bytes, p.N}, go{grad_out, in[0].bytes, in[0].bytes, p.N};
    const size_t tb = table_bytes(p);
    for (int i = 0; i < 3; ++i) {
        for (const Images &x : in)
            if (meet(written[i], x)) return ESC_ERR_ALIAS;
        if (meet(written[i], o) || meet(written[i], go) || meets(written[i], saved, sv) || meets(written[i], workspace, sc.total) ||
            meets(written[i], p.mask, mask_bytes) || meets(written[i], p.bias, tb) || meets(written[i], g->bias, tb) ||
            meet(written[i], written[(i + 1) % 3]) || meets(in[i], workspace, sc.total) || meets(in[i], g->bias, tb))
            return ESC_ERR_ALIAS;
    }
    const auto apart = [&](const void *b, size_t n) {  // from what lies in one piece and is read
        return !(meets(o, b, n) || meets(go, b, n) || overlaps(saved, sv, b, n) || (p.mask != nullptr && overlaps(p.mask, mask_bytes, b, n)) ||
                 (p.bias != nullptr && overlaps(p.bias, tb, b, n)));
    };
    if (!apart(workspace, sc.total)) return ESC_ERR_ALIAS;
    if (g->bias != nullptr && (!apart(g->bias, tb) || overlaps(workspace, sc.total, g->bias, tb))) return ESC_ERR_ALIAS;

    char *ws = static_cast<char *>(workspace);
    for (WindowParams *x : {&pq, &pk}) {
        x->out_in = out, x->go = grad_out;
        x->top = static_cast<float *>(const_cast<void *>(saved));
        x->log_sum = x->top + (size_t)p.N * p.heads * p.H * p.W;
        x->rest = f32 ? nullptr : static_cast<char *>(const_cast<void *>(saved)) + rows_bytes(p);
        x->gq = g->q, x->gk = g->k, x->gv = g->v;
        x->gqs = (long)(written[0].stride / es), x->gks = (long)(written[1].stride / es), x->gvs = (long)(written[2].stride / es);
        x->grad_bias = g->bias;
        x->accumulate = accumulate;
        x->delta = reinterpret_cast<float *>(ws + sc.delta);
        x->part = reinterpret_cast<float *>(ws + sc.part);
        x->part2 = reinterpret_cast<float *>(ws + sc.part2);
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int dp = dim_padded(p.d);
    if (launch_window_dq(pq, f32, dp, s) != hipSuccess || launch_window_dkv(pk, f32, dp, s) != hipSuccess) return ESC_ERR_HIP;
    if (g->bias != nullptr && launch_window_bias_grad(pq, s) != hipSuccess) return ESC_ERR_HIP;
    return ESC_OK;
}

}  // extern "C"
