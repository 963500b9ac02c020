// The AdamW step over all of a network's parameter tensors in one launch, states in 32 or in 8 bits
// (esc_adamw_* of include/esc_convattn.h).
//
// Per element, in fp32, every operation rounded by itself:
//   g' = grad_scale g
//   m  = beta1 m + (1 - beta1) g'          v = beta2 v + (1 - beta2) g' g'          r = sqrt(v)
//   p  = p (1 - lr wd) - lr / (1 - beta1^t) * ( m / (r / sqrt(1 - beta2^t) + eps) )
// (the factors in front are made in 64 bits and rounded once; r is multiplied by the rounded 1 / sqrt(1 - beta2^t)).
//
// In 8 bits a state is the code e4m3(x * (448 * (1 / a))) of x = m, or of x = r (not v: half the exponent range), and a fp32
// scale a * (1 / 448) for each block of 256 consecutive elements of a tensor, a the block's largest finite magnitude; blocks
// whose magnitudes all lie below 2^-100 hold zeros.  A positive r never becomes zero (it takes the smallest code): the next
// step would divide what is left of m by eps.
//
// What bounds it: memory.  28 bytes an element with fp32 states and gradients (p, g, m, v in; p, m, v out), 16 and a sixteenth with
// 8-bit states, 14 and a sixteenth with bf16 gradients.  Measured, one MI355X, 169 million elements: 8-bit states, bf16 gradients 498 us, 4.8 TB/s (a copy of 1 GiB:
// 5.1); fp32 states, fp32 gradients 1004 us, bf16 gradients 939, 4.7 TB/s both.  A network of 0.8 million elements, fp32 states: 9.0 us with fp32 gradients,
// 10.3 with bf16.
// Layout: the plan (device memory) holds one record per tensor and the tensor's number for every chunk of kChunk elements, so
// that a block finds its work in two dependent loads whatever the number of tensors, and small tensors cost a block each, not
// a launch.  A wavefront takes 256 consecutive elements at a time, four a lane (16-byte accesses; one block of
// 8-bit states, its maximum a wavefront reduction); four such units of a block's wavefront are independent of each other.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>
#include <type_traits>
#include <vector>

#include "esc_convattn.h"
#include "esc_host.hpp"
#include "esc_terms.hpp"

namespace {

using namespace esc;

constexpr int kThreads = 256;
constexpr int kUnit = 256;       // elements a wavefront takes at a time: the elements that share a scale
constexpr int kUnits = 4;        // units of a wavefront in a chunk
constexpr int kChunk = kUnit * kUnits * (kThreads / 64);
constexpr int kMaxGrid = 2048;   // eight blocks a compute unit
constexpr int kLeaves = 64;      // counters that blocks sign off on
constexpr int kRecordsPerLaunch = 32;
constexpr float kCodeMax = 448.f;
constexpr float kTiny = 0x1p-100f;

struct Record {  // of a tensor, in device memory
    float *p;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale;
    long n;
    int first_chunk;
    float weight_decay;
};
static_assert(sizeof(Record) == 64, "one cache line each");

struct Control {  // at the front of the plan; everything else behind it at multiples of 256 bytes
    long step;
    unsigned root;
    unsigned pad[61];
    struct {
        unsigned count;
        unsigned pad[15];
    } leaf[kLeaves];
};
static_assert(sizeof(Control) == 256 + 64 * kLeaves, "");

size_t records_offset() { return sizeof(Control); }
size_t map_offset(int tensors) { return round_up(records_offset() + (size_t)tensors * sizeof(Record), 256); }
size_t plan_size(int tensors, long chunks) { return round_up(map_offset(tensors) + (size_t)chunks * sizeof(int), 256); }

struct RecordBatch {
    Record r[kRecordsPerLaunch];
};

__global__ void control_kernel(Control *c, long step)
{
    const int i = threadIdx.x;
    if (i == 0) c->step = step, c->root = 0;
    if (i < kLeaves) c->leaf[i].count = 0;
}

// Writes a batch of records and their part of the chunk map.
__global__ void records_kernel(Record *records, int *map, RecordBatch b, int first, int n)
{
    for (int i = 0; i < n; ++i) {
        if (blockIdx.x == 0 && threadIdx.x == 0) records[first + i] = b.r[i];
        const int chunks = (int)((b.r[i].n + kChunk - 1) / kChunk);
        for (int c = blockIdx.x * blockDim.x + threadIdx.x; c < chunks; c += gridDim.x * blockDim.x) map[b.r[i].first_chunk + c] = first + i;
    }
}

struct StepArgs {
    Control *control;
    const Record *records;
    const int *map;
    const float *lr_device;
    double lr, beta1, beta2, eps, grad_scale;
    int chunks;
};

__device__ double power(double b, long n)
{
    double r = 1.0;
    for (; n > 0; n >>= 1) {
        if (n & 1) r *= b;
        b *= b;
    }
    return r;
}

// Four neighbouring elements: at once where the chunk is WHOLE (and its buffers aligned), else those below n.
template <bool WHOLE, typename V, typename E>
__device__ __forceinline__ V load4(const E *a, long i, long n)
{
    static_assert(sizeof(V) == 4 * sizeof(E), "");
    if constexpr (WHOLE) return *reinterpret_cast<const V *>(a + i);
    E e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = i + j < n ? a[i + j] : E(0);
    return __builtin_bit_cast(V, e);
}
template <bool WHOLE, typename V, typename E>
__device__ __forceinline__ void store4(E *a, long i, long n, V v)
{
    if constexpr (WHOLE) {
        *reinterpret_cast<V *>(a + i) = v;
        return;
    }
    E e[4];
    __builtin_memcpy(e, &v, sizeof(V));
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) a[i + j] = e[j];
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 decode(uint32_t c)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    return f32x4{a.x, a.y, b.x, b.y};
}

// The codes of a wavefront's 256 values and their scale.
template <bool UP>
__device__ __forceinline__ uint32_t encode(f32x4 x, float *scale)
{
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned a = __float_as_uint(x[j]) & 0x7fffffffu;
        top = max(top, a < 0x7f800000u ? a : 0u);
    }
    const float a = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)wave_max(top), 63));
    const bool full = a >= kTiny;
    *scale = full ? a * (1.f / kCodeMax) : 0.f;
    const float inverse = full ? kCodeMax * (1.f / a) : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float y = x[j] * inverse;
        // what is not finite is held as NaN (the conversion alone would hold an infinity as 448)
        if ((__float_as_uint(y) & 0x7fffffffu) >= 0x7f800000u) y = __builtin_nanf("");
        if (UP && y > 0.f && y < 0x1p-9f) y = 0x1p-9f;
        x[j] = y;
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], c, true);
}

// What a step has in common.
struct Factors {
    float beta1, rest1, beta2, rest2, eps, grad_scale, size, correct;
};

// A wavefront's part of a chunk: kUnits units of 256 elements, all of whose loads are on their way before the first is waited for.
template <bool EIGHT, bool BF16, bool WHOLE>
__device__ __forceinline__ void part_of_chunk(const Record &r, const Factors &f, float keep, long base)
{
    using G = typename std::conditional<BF16, uint16_t, float>::type;
    typedef G g4 __attribute__((ext_vector_type(4)));
    typedef uint8_t u8x4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63;
    f32x4 p[kUnits], m[kUnits], v[kUnits];
    g4 g[kUnits];
    u8x4 mc[kUnits], vc[kUnits];
    float ms[kUnits], vs[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const long i = base + u * kUnit + lane * 4, unit = base / kUnit + u;
        p[u] = load4<WHOLE, f32x4>(r.p, i, r.n);
        g[u] = load4<WHOLE, g4>(static_cast<const G *>(r.g), i, r.n);
        if constexpr (EIGHT) {
            mc[u] = load4<WHOLE, u8x4>(static_cast<const uint8_t *>(r.m), i, r.n), vc[u] = load4<WHOLE, u8x4>(static_cast<const uint8_t *>(r.v), i, r.n);
            const bool any = WHOLE || unit * kUnit < r.n;
            ms[u] = any ? r.m_scale[unit] : 0.f, vs[u] = any ? r.v_scale[unit] : 0.f;
        } else {
            m[u] = load4<WHOLE, f32x4>(static_cast<const float *>(r.m), i, r.n);
            v[u] = load4<WHOLE, f32x4>(static_cast<const float *>(r.v), i, r.n);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const long i = base + u * kUnit + lane * 4, unit = base / kUnit + u;
        if (!WHOLE && unit * kUnit >= r.n) break;  // (the same for the wavefront)
        if constexpr (EIGHT) {
            m[u] = decode(__builtin_bit_cast(uint32_t, mc[u]));
            v[u] = decode(__builtin_bit_cast(uint32_t, vc[u]));
        }
        f32x4 root;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (EIGHT) {
                m[u][j] = m[u][j] * ms[u];
                const float held = v[u][j] * vs[u];
                v[u][j] = held * held;
            }
            float gs;
            if constexpr (BF16) gs = __uint_as_float((uint32_t)g[u][j] << 16);
            else gs = g[u][j];
            gs *= f.grad_scale;
            m[u][j] = f.beta1 * m[u][j] + f.rest1 * gs;
            v[u][j] = f.beta2 * v[u][j] + f.rest2 * (gs * gs);
            root[j] = sqrtf(v[u][j]);
            p[u][j] = p[u][j] * keep - f.size * (m[u][j] / (root[j] * f.correct + f.eps));
        }
        store4<WHOLE>(r.p, i, r.n, p[u]);
        if constexpr (EIGHT) {
            float ns, nr;
            // (lanes beyond the tensor's end have loaded zeros: their states stay zero and below any maximum)
            const uint32_t nm = encode<false>(m[u], &ns), nv = encode<true>(root, &nr);
            store4<WHOLE>(static_cast<uint8_t *>(r.m), i, r.n, __builtin_bit_cast(u8x4, nm));
            store4<WHOLE>(static_cast<uint8_t *>(r.v), i, r.n, __builtin_bit_cast(u8x4, nv));
            if (lane == 0) r.m_scale[unit] = ns, r.v_scale[unit] = nr;
        } else {
            store4<WHOLE>(static_cast<float *>(r.m), i, r.n, m[u]);
            store4<WHOLE>(static_cast<float *>(r.v), i, r.n, v[u]);
        }
    }
}

template <bool EIGHT, bool BF16>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const StepArgs a)
{
    constexpr uintptr_t kGradMask = BF16 ? 7 : 15, kStateMask = EIGHT ? 3 : 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long step = a.control->step + 1;
    const double lr = a.lr_device != nullptr ? (double)*a.lr_device : a.lr;
    const Factors f{(float)a.beta1, (float)(1.0 - a.beta1), (float)a.beta2, (float)(1.0 - a.beta2), (float)a.eps, (float)a.grad_scale,
                    (float)(lr / (1.0 - power(a.beta1, step))), (float)(1.0 / sqrt(1.0 - power(a.beta2, step)))};
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const Record r = a.records[a.map[c]];
        const long base = (long)(c - r.first_chunk) * kChunk + wave * (kUnit * kUnits);
        const bool aligned = (((uintptr_t)r.p & 15) | ((uintptr_t)r.g & kGradMask) | (((uintptr_t)r.m | (uintptr_t)r.v) & kStateMask)) == 0;
        const float keep = (float)(1.0 - lr * (double)r.weight_decay);
        if (aligned && base + kUnit * kUnits <= r.n) part_of_chunk<EIGHT, BF16, true>(r, f, keep, base);
        else if (base < r.n) part_of_chunk<EIGHT, BF16, false>(r, f, keep, base);
    }
    // The last block to leave counts the step, after all of its wavefronts have read the count.  Two levels, so that no word sees more than
    // kMaxGrid / kLeaves or kLeaves atomics.
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned leaf = blockIdx.x % kLeaves, leaves = min((unsigned)kLeaves, gridDim.x);
        const unsigned here = (gridDim.x - leaf + kLeaves - 1) / kLeaves;
        if (atomicAdd(&a.control->leaf[leaf].count, 1u) + 1 == here) {
            a.control->leaf[leaf].count = 0;
            if (atomicAdd(&a.control->root, 1u) + 1 == leaves) {
                a.control->root = 0;
                a.control->step = step;
            }
        }
    }
}

// chunks of all tensors, -1 where there are too many or an argument is bad (then *st says why)
long count_chunks(const esc_adamw_tensor *t, int n, esc_adamw_state state, esc_status *st)
{
    *st = ESC_ERR_SHAPE;
    if (n < 1) return -1;
    if (state != ESC_ADAMW_F32 && state != ESC_ADAMW_EIGHT) {
        *st = ESC_ERR_DTYPE;
        return -1;
    }
    if (t == nullptr) {
        *st = ESC_ERR_NULL;
        return -1;
    }
    long chunks = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].n < 0) return -1;
        if (t[i].n > ((long)1 << 48)) {
            *st = ESC_ERR_UNSUPPORTED;
            return -1;
        }
        chunks += (t[i].n + kChunk - 1) / kChunk;
        if (chunks > 0x3fffffff) {
            *st = ESC_ERR_UNSUPPORTED;
            return -1;
        }
    }
    *st = ESC_OK;
    return chunks;
}

struct Span {
    uintptr_t at, end;
    bool written;
};

}  // namespace

extern "C" {

size_t esc_adamw_plan_bytes(const esc_adamw_tensor *tensors, int n, esc_adamw_state state)
{
    esc_status st;
    const long chunks = count_chunks(tensors, n, state, &st);
    return chunks < 0 ? 0 : plan_size(n, chunks);
}

esc_status esc_adamw_plan_init(const esc_adamw_tensor *tensors, int n, esc_adamw_state state, esc_dtype grad_dt, long step, void *memory, size_t bytes,
                               esc_adamw_plan *plan, void *stream)
{
    esc_status st;
    if (grad_dt != ESC_F32 && grad_dt != ESC_BF16) return ESC_ERR_DTYPE;
    const long chunks = count_chunks(tensors, n, state, &st);
    if (chunks < 0) return st;
    if (plan == nullptr) return ESC_ERR_NULL;
    if (step < 0) return ESC_ERR_SHAPE;
    if (memory == nullptr || ((uintptr_t)memory & 255) != 0 || bytes < plan_size(n, chunks)) return ESC_ERR_WORKSPACE;
    const size_t gs = grad_dt == ESC_F32 ? 4 : 2, ss = state == ESC_ADAMW_F32 ? 4 : 1;
    try {
        std::vector<Span> ranges;
        ranges.reserve(6 * (size_t)n + 1);
        auto range = [&](const void *p, size_t nbytes, bool written) {
            if (nbytes > 0) ranges.push_back(Span{(uintptr_t)p, (uintptr_t)p + nbytes, written});
        };
        range(memory, plan_size(n, chunks), true);
        for (int i = 0; i < n; ++i) {
            const esc_adamw_tensor &t = tensors[i];
            if (!(t.weight_decay >= 0.f) || !isfinite(t.weight_decay)) return ESC_ERR_SHAPE;
            if (t.n == 0) continue;
            if (t.param == nullptr || t.grad == nullptr || t.m == nullptr || t.v == nullptr) return ESC_ERR_NULL;
            if (state == ESC_ADAMW_EIGHT && (t.m_scale == nullptr || t.v_scale == nullptr)) return ESC_ERR_NULL;
            if ((uintptr_t)t.param % 4 != 0 || (uintptr_t)t.grad % gs != 0 || (uintptr_t)t.m % ss != 0 || (uintptr_t)t.v % ss != 0) return ESC_ERR_SHAPE;
            range(t.param, (size_t)t.n * 4, true);
            range(t.grad, (size_t)t.n * gs, false);
            range(t.m, (size_t)t.n * ss, true);
            range(t.v, (size_t)t.n * ss, true);
            if (state == ESC_ADAMW_EIGHT) {
                if (((uintptr_t)t.m_scale | (uintptr_t)t.v_scale) % 4 != 0) return ESC_ERR_SHAPE;
                range(t.m_scale, (size_t)((t.n + kUnit - 1) / kUnit) * 4, true);
                range(t.v_scale, (size_t)((t.n + kUnit - 1) / kUnit) * 4, true);
            }
        }
        // what is written overlaps nothing else (a tensor that is named twice would be stepped by two blocks at a time)
        std::sort(ranges.begin(), ranges.end(), [](const Span &a, const Span &b) { return a.at < b.at; });
        uintptr_t end = 0, written_end = 0;
        for (const Span &r : ranges) {
            if (r.at < written_end || (r.written && r.at < end)) return ESC_ERR_ALIAS;
            end = std::max(end, r.end);
            if (r.written) written_end = std::max(written_end, r.end);
        }
    } catch (const std::bad_alloc &) {
        return ESC_ERR_UNSUPPORTED;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    Control *control = static_cast<Control *>(memory);
    Record *records = reinterpret_cast<Record *>(static_cast<char *>(memory) + records_offset());
    int *map = reinterpret_cast<int *>(static_cast<char *>(memory) + map_offset(n));
    hipLaunchKernelGGL(control_kernel, dim3(1), dim3(64), 0, s, control, step);
    if (hipGetLastError() != hipSuccess) return ESC_ERR_HIP;
    long first_chunk = 0;
    for (int i = 0; i < n; i += kRecordsPerLaunch) {
        RecordBatch b{};
        const int k = std::min(kRecordsPerLaunch, n - i);
        long most = 0;
        for (int j = 0; j < k; ++j) {
            const esc_adamw_tensor &t = tensors[i + j];
            b.r[j] = Record{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.n, (int)first_chunk, t.weight_decay};
            const long c = (t.n + kChunk - 1) / kChunk;
            first_chunk += c;
            most = std::max(most, c);
        }
        const unsigned blocks = (unsigned)std::min<long>(std::max<long>(1, (most + 255) / 256), 1024);
        hipLaunchKernelGGL(records_kernel, dim3(blocks), dim3(256), 0, s, records, map, b, i, k);
        if (hipGetLastError() != hipSuccess) return ESC_ERR_HIP;
    }
    *plan = esc_adamw_plan{memory, plan_size(n, chunks), n, chunks, state, grad_dt};
    return ESC_OK;
}

esc_status esc_adamw_step(const esc_adamw_plan *plan, const esc_adamw_hyper *h, void *stream)
{
    if (plan == nullptr || h == nullptr) return ESC_ERR_NULL;
    if (plan->state != ESC_ADAMW_F32 && plan->state != ESC_ADAMW_EIGHT) return ESC_ERR_DTYPE;
    if (plan->grad_dt != ESC_F32 && plan->grad_dt != ESC_BF16) return ESC_ERR_DTYPE;
    if (plan->n < 1 || plan->chunks < 0 || plan->chunks > 0x3fffffff) return ESC_ERR_SHAPE;
    if (plan->memory == nullptr || ((uintptr_t)plan->memory & 255) != 0 || plan->bytes < plan_size(plan->n, plan->chunks)) return ESC_ERR_WORKSPACE;
    const auto ok = [](double x, double most) { return x >= 0.0 && x < most; };  // (false for NaN)
    if (!ok(h->beta1, 1.0) || !ok(h->beta2, 1.0) || !ok(h->lr, 1e30) || !ok(h->eps, 1e30) || !isfinite(h->grad_scale)) return ESC_ERR_SHAPE;
    if (((uintptr_t)h->lr_device & 3) != 0) return ESC_ERR_SHAPE;
    char *mem = static_cast<char *>(plan->memory);
    const StepArgs a{reinterpret_cast<Control *>(mem), reinterpret_cast<const Record *>(mem + records_offset()),
                     reinterpret_cast<const int *>(mem + map_offset(plan->n)), h->lr_device, h->lr, h->beta1, h->beta2, h->eps, h->grad_scale, (int)plan->chunks};
    // (one block at least: it counts the step, also of tensors that are all empty)
    const dim3 grid((unsigned)std::max<long>(1, std::min<long>(plan->chunks, kMaxGrid))), block(kThreads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = plan->grad_dt == ESC_BF16;
    if (plan->state == ESC_ADAMW_EIGHT) {
        if (bf16) hipLaunchKernelGGL((adamw_kernel<true, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((adamw_kernel<true, false>), grid, block, 0, s, a);
    } else {
        if (bf16) hipLaunchKernelGGL((adamw_kernel<false, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((adamw_kernel<false, false>), grid, block, 0, s, a);
    }
    return hipGetLastError() == hipSuccess ? ESC_OK : ESC_ERR_HIP;
}

}  // extern "C"
