// Distillation loss from a teacher's top logits: forward, backward, both in one pass.
//
// Per row: lse = log sum_v exp(z_v / T) needs all of z before the first gradient value can be
// written, so the gradient is a second walk over the row.  The floor is one read of the logits and
// one write of the gradient.
//
// A CTA owns a row.  The first walk keeps a running maximum and sum per thread (the sum is rescaled only
// when the maximum moves), the second finds the row, which the same CTA read a moment ago, in L2.  One more warp
// has the teacher: it fetches and weighs the entries beside the first walk.
// What bounds it: backward and forward alone the memory (4096 x 32000 float 160 us, 6.5 TB/s; 3000 x 131072 bfloat16 loss
// 128-138 us, 5.7-6.1 TB/s); the step its two exponentials per element, 8 cycles per warp and scheduler each, and its
// instructions beside three passes of L2 (8192 x 50257 bfloat16, rows on 2-byte boundaries: 313-330 us, 5.0-5.3 TB/s of
// the read and the write).  Tried for the step: the row kept in shared memory by a cluster 392-448 us; a persistent ring of bulk
// copies, the row held in it, 407-470 us: many warps from several rows hide the exponentials better than a held row saves.
// 256 walkers and four CTAs an SM; 128 and seven 390 us, 512 and three 326 (and 137 against 133 for the loss alone).
#include "context.h"
#include "vector.cuh"

namespace omni {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
enum Mode { kForward = 0, kBackward = 1, kStep = 2 };

struct DistillParams {
    const void *logits;
    unsigned long long row_stride, grad_stride, top_stride;
    const float *top_logits;
    const void *top_index;
    const float *grad_loss;
    const float *lse_in;
    float *loss, *lse_out;
    void *grad;
    int vocab, top;
    float temperature;
};

// Eight logits as loaded, their largest, and as four pairs of floats.
template <typename T> struct Group;
template <> struct Group<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p)
    {
        float f[kGroup];
        load_group(p, f);
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ float largest() const
    {
        return fmaxf(fmaxf(fmaxf(a.x, a.y), fmaxf(a.z, a.w)), fmaxf(fmaxf(b.x, b.y), fmaxf(b.z, b.w)));
    }
    __device__ __forceinline__ float2 pair(int i) const
    {
        return i == 0 ? make_float2(a.x, a.y) : i == 1 ? make_float2(a.z, a.w) : i == 2 ? make_float2(b.x, b.y) : make_float2(b.z, b.w);
    }
};
template <> struct Group<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { u = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ static uint32_t larger(uint32_t x, uint32_t y)
    {
        uint32_t z;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
        return z;
    }
    __device__ __forceinline__ float largest() const
    {
        const uint32_t m = larger(larger(u.x, u.y), larger(u.z, u.w));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    __device__ __forceinline__ float2 pair(int i) const
    {
        const uint32_t w = i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
};

// A thread's running maximum m and sum of 2^(x - m), x = logit * unit.  Products and sums are spelled out
// where the compiler could contract them one way in one variant and another way in the next: forward
// and step give the same bits.
struct Running {
    float m = -INFINITY;
    float2 a = {0.0f, 0.0f}, b = {0.0f, 0.0f};
    template <typename T, int K> __device__ __forceinline__ void take(const Group<T> (&g)[K], float unit)
    {
        float top = g[0].largest();
#pragma unroll
        for (int k = 1; k < K; ++k) top = fmaxf(top, g[k].largest());
        raise(__fmul_rn(top, unit));
        const float ref = m == -INFINITY ? 0.0f : -m;
        const float2 u = {unit, unit}, r = {ref, ref};
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 x = fma2(g[k].pair(i), u, r);
                const float2 e = {exp2_fast(x.x), exp2_fast(x.y)};
                if (i % 2 == 0) a = add2(a, e);
                else b = add2(b, e);
            }
    }
    __device__ __forceinline__ void take_one(float z, float unit)
    {
        const float x = __fmul_rn(z, unit);
        raise(x);
        a.x += exp2_fast(x - (m == -INFINITY ? 0.0f : m));
    }
    __device__ __forceinline__ void raise(float to)
    {
        if (to > m) {                                // rare after the first few groups
            const float f = exp2_fast(m - to);
            a = mul2(a, {f, f});
            b = mul2(b, {f, f});
            m = to;
        }
    }
    __device__ __forceinline__ float sum() const { return __fadd_rn(__fadd_rn(a.x, a.y), __fadd_rn(b.x, b.y)); }
};

struct Joined { float m, s; };
__device__ __forceinline__ float warp_max(float x)
{
    for (int o = 16; o > 0; o /= 2) x = fmaxf(x, __shfl_xor_sync(~0u, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x)
{
    for (int o = 16; o > 0; o /= 2) x = __fadd_rn(x, __shfl_xor_sync(~0u, x, o));
    return x;
}
// A warp's maximum and sum into its cell.
__device__ __forceinline__ void put_warp(const Running &run, Joined *cell)
{
    const float m = warp_max(run.m);
    const float s = run.sum();
    const float t = warp_sum(m == -INFINITY || run.m == m ? s : __fmul_rn(s, exp2_fast(run.m - m)));
    if (threadIdx.x % 32 == 0) *cell = {m, t};
}

// The walkers' cells joined, by every warp for itself: the sum for the largest maximum.
template <int N> __device__ __forceinline__ Joined join_cells(const Joined (&cell)[N], int n = N)
{
    const int lane = threadIdx.x % 32;
    const Joined x = lane < n ? cell[lane] : Joined{-INFINITY, 0.0f};
    const float m = warp_max(x.m);
    return {m, warp_sum(m == -INFINITY || x.m == m ? x.s : __fmul_rn(x.s, exp2_fast(x.m - m)))};
}

// Element range of a row in three parts: up to the first 16-byte boundary, whole groups, the rest.
template <typename T> struct Parts {
    int head, groups;
    __device__ __forceinline__ Parts(const T *row, int vocab)
    {
        const int lead = int((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / int(sizeof(T));
        head = lead < vocab ? lead : vocab;
        groups = (vocab - head) / kGroup;
    }
    // the i-th of the elements outside the groups (fewer than 16)
    __device__ __forceinline__ int edge(int i) const { return i < head ? i : groups * kGroup + i; }
};

// The teacher's side of a row: where its entries stand, the student's logit there, their probability.
struct Teacher {
    float prob[OMNI_DISTILL_MAX_TOP], hit[OMNI_DISTILL_MAX_TOP];
    int place[OMNI_DISTILL_MAX_TOP];
    float term;                                     // sum of p (log p - z / T)
    int target;                                     // some entry has a probability
    int repeated;                                   // some place is named twice
};

// One warp's work, beside the walk over the row.  `seen`: a table of 2 OMNI_DISTILL_MAX_TOP places.
template <typename T, typename I>
__device__ __forceinline__ void teacher_warp(const DistillParams &p, unsigned long long r, const T *row, Teacher &te, int *seen)
{
    const int lane = threadIdx.x % 32;
    const float *logit = p.top_logits + r * p.top_stride;
    float top = -INFINITY;
    int table = 32;                                 // at least twice the entries
    while (table < 2 * p.top) table *= 2;
    for (int j = lane; j < table; j += 32) seen[j] = -1;
    __syncwarp();
    bool repeated = false;
    for (int j = lane; j < p.top; j += 32) {
        const long long i = load_index<I>(p.top_index, r * p.top_stride + j);
        const bool there = i >= 0 && i < p.vocab;
        const float t = there ? logit[j] / p.temperature : -INFINITY;
        te.place[j] = there ? int(i) : -1;
        te.hit[j] = there ? to_float(row[i]) : 0.0f;
        te.prob[j] = t;
        top = fmaxf(top, t);
        for (int h = int(unsigned(i) * 2654435769u >> 16) & (table - 1); there; h = (h + 1) & (table - 1)) {
            const int old = atomicCAS(&seen[h], -1, int(i));
            repeated |= old == int(i);
            if (old == -1 || old == int(i)) break;
        }
    }
    repeated = __any_sync(~0u, repeated);
    top = warp_max(top);
    float total = 0.0f;
    for (int j = lane; j < p.top; j += 32) {
        const float e = top == -INFINITY && !isnan(te.prob[j]) ? 0.0f : expf(te.prob[j] - top);
        te.prob[j] = e;
        total += e;
    }
    total = warp_sum(total);
    const bool target = !(total == 0.0f);           // NaN counts as a target and shows
    float term = 0.0f;
    for (int j = lane; j < p.top; j += 32) {
        const float q = target ? te.prob[j] / total : 0.0f;
        te.prob[j] = q;
        if (!(q == 0.0f)) term = __fadd_rn(term, __fmul_rn(q, logf(q) - te.hit[j] / p.temperature));
    }
    term = warp_sum(term);
    if (lane == 0) {
        te.term = term;
        te.target = target;
        te.repeated = repeated;
    }
    __syncwarp();
}

// The gradient at the teacher's entries, over what the walk wrote there; an entry that names a token again is
// left to the first.  `ref`: minus the lse in powers of two.
template <typename T>
__device__ __forceinline__ void put_entries(const DistillParams &p, const Teacher &te, T *out, float gain, float unit, float ref, int from, int step)
{
    for (int j = from; j < p.top; j += step) {
        const int at = te.place[j];
        if (at < 0) continue;
        float total = te.prob[j];
        bool first = true;
        if (te.repeated) {
            total = 0.0f;
            for (int i = 0; i < p.top; ++i)
                if (te.place[i] == at) {
                    first = first && i >= j;
                    total += te.prob[i];
                }
        }
        if (first) out[at] = from_float<T>(gain * (exp2_fast(fmaf(te.hit[j], unit, ref)) - total));
    }
}

// gain * 2^(logit * unit + ref) of a group, stored.
template <typename T>
__device__ __forceinline__ void put_group(T *dst, const Group<T> &g, float unit, float ref, float gain)
{
    float f[kGroup];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = fma2(g.pair(i), {unit, unit}, {ref, ref});
        const float2 y = mul2({exp2_fast(x.x), exp2_fast(x.y)}, {gain, gain});
        f[2 * i] = y.x;
        f[2 * i + 1] = y.y;
    }
    store_streaming(dst, f);
}
template <typename T> __device__ __forceinline__ T put_value(T z, float unit, float ref, float gain)
{
    return from_float<T>(__fmul_rn(exp2_fast(fmaf(to_float(z), unit, ref)), gain));
}
__device__ __forceinline__ bool same_phase(const void *a, const void *b)
{
    return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}

// ---- a CTA per row, from global memory ----------------------------------------------------------

constexpr int kRowWalkers = 256;

template <typename T, typename I, int MODE>
__global__ void __launch_bounds__(kRowWalkers + 32, 4) row_kernel(DistillParams p)
{
    __shared__ Joined cell[kRowWalkers / 32];
    __shared__ Teacher te;
    __shared__ int seen[2 * OMNI_DISTILL_MAX_TOP];
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;  // groups a thread has in flight
    const int walkers = blockDim.x - 32, tid = threadIdx.x, warp = tid / 32;
    const unsigned long long r = blockIdx.x;
    const T *row = static_cast<const T *>(p.logits) + r * p.row_stride;
    const float unit = kLog2e / p.temperature;
    const Parts<T> parts(row, p.vocab);
    const int rest = p.vocab - parts.groups * kGroup;
    // f(first group, groups): kAhead at a time, then one by one
    auto walk = [&](auto f) {
        int g = tid;
        for (; g + (kAhead - 1) * walkers < parts.groups; g += walkers * kAhead) {
            Group<T> x[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) x[a].load(row + parts.head + (long long)(g + a * walkers) * kGroup);
            f(g, x);
        }
        for (; g < parts.groups; g += walkers) {
            Group<T> x[1];
            x[0].load(row + parts.head + (long long)g * kGroup);
            f(g, x);
        }
    };
    const float weight = MODE == kForward ? 0.0f : p.grad_loss[r];
    float lse2 = MODE == kBackward ? __fmul_rn(p.lse_in[r], kLog2e) : 0.0f;
    if (tid >= walkers) {
        teacher_warp<T, I>(p, r, row, te, seen);
    } else if constexpr (MODE != kBackward) {
        Running run;
        walk([&](int, const auto &x) { run.take(x, unit); });
        if (tid < rest) run.take_one(to_float(row[parts.edge(tid)]), unit);
        __syncwarp();
        put_warp(run, cell + warp);
    }
    __syncthreads();
    const bool target = te.target;
    if constexpr (MODE != kBackward) {
        const Joined all = join_cells(cell, walkers / 32);
        lse2 = all.m + log2f(all.s);
        if (tid == 0) {
            const float lse = __fmul_rn(lse2, kLn2);
            p.lse_out[r] = lse;
            p.loss[r] = target ? __fmul_rn(__fmul_rn(p.temperature, p.temperature), __fadd_rn(te.term, lse)) : 0.0f;
        }
    }
    if constexpr (MODE != kForward) {
        T *out = static_cast<T *>(p.grad) + r * p.grad_stride;
        const float gain = __fmul_rn(weight, p.temperature);
        const float ref = lse2 == -INFINITY ? 0.0f : -lse2;
        if (tid < walkers) {
            if (!target) {
                for (int v = tid; v < p.vocab; v += walkers) out[v] = from_float<T>(0.0f);
            } else if (same_phase(out, row)) {
                walk([&](int g, const auto &x) {
#pragma unroll
                    for (int a = 0; a < int(sizeof x / sizeof x[0]); ++a)
                        put_group(out + parts.head + (long long)(g + a * walkers) * kGroup, x[a], unit, ref, gain);
                });
                if (tid < rest) out[parts.edge(tid)] = put_value(row[parts.edge(tid)], unit, ref, gain);
            } else {
                for (int v = tid; v < p.vocab; v += walkers) out[v] = put_value(row[v], unit, ref, gain);
            }
        }
        __syncthreads();
        if (target) put_entries(p, te, out, gain, unit, ref, tid, blockDim.x);
    }
}

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_distill(const omni_distill *d)
{
    if (!d) return OMNI_ERR_NULL;
    if ((d->dtype != OMNI_F32 && d->dtype != OMNI_BF16) || (d->index_type != OMNI_I32 && d->index_type != OMNI_I64))
        return OMNI_ERR_BAD_CONFIG;
    if (d->vocab < 1 || d->top < 1 || !(d->temperature > 0.0f) || d->temperature - d->temperature != 0.0f) return OMNI_ERR_BAD_CONFIG;
    if (d->top > OMNI_DISTILL_MAX_TOP || d->rows >= (1ull << 31)) return OMNI_ERR_TOO_LARGE;
    if (d->rows > 1 && (d->row_stride < uint64_t(d->vocab) || d->top_stride < uint64_t(d->top))) return OMNI_ERR_BAD_CONFIG;
    if (d->rows == 0) return OMNI_OK;
    if (!d->logits || !d->top_logits || !d->top_index) return OMNI_ERR_NULL;
    if (!aligned(d->logits, d->dtype == OMNI_BF16 ? 2 : 4) || !aligned(d->top_logits, 4) ||
        !aligned(d->top_index, d->index_type == OMNI_I64 ? 8 : 4))
        return OMNI_ERR_ALIGN;
    return OMNI_OK;
}

template <typename T, typename I>
int enqueue(omni_ctx *ctx, int mode, const DistillParams &p, unsigned rows, cudaStream_t s)
{
    int walkers = 64;
    while (walkers < kRowWalkers && walkers * 8 * kGroup < p.vocab) walkers *= 2;
    if (mode == kForward) row_kernel<T, I, kForward><<<rows, walkers + 32, 0, s>>>(p);
    else if (mode == kBackward) row_kernel<T, I, kBackward><<<rows, walkers + 32, 0, s>>>(p);
    else row_kernel<T, I, kStep><<<rows, walkers + 32, 0, s>>>(p);
    return context_launched(ctx, int(cudaGetLastError()));
}

int run(omni_ctx *ctx, int mode, const omni_distill *d, const float *lse_in, const float *grad_loss, float *loss,
        float *lse_out, void *grad, uint64_t grad_stride, void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_distill(d);
    if (rc != OMNI_OK) return rc;
    if (d->rows > 0) {
        if (mode != kBackward && (!loss || !lse_out)) return OMNI_ERR_NULL;
        if (mode != kForward && (!grad || !grad_loss || (mode == kBackward && !lse_in))) return OMNI_ERR_NULL;
        if (mode != kForward && d->rows > 1 && grad_stride < uint64_t(d->vocab)) return OMNI_ERR_BAD_CONFIG;
        if (!aligned(loss, 4) || !aligned(lse_out, 4) || !aligned(lse_in, 4) || !aligned(grad_loss, 4) ||
            !aligned(grad, d->dtype == OMNI_BF16 ? 2 : 4))
            return OMNI_ERR_ALIGN;
    }
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK || d->rows == 0) return rc;
    DistillParams p;
    p.logits = d->logits;
    p.row_stride = d->row_stride;
    p.grad_stride = grad_stride;
    p.top_stride = d->top_stride;
    p.top_logits = d->top_logits;
    p.top_index = d->top_index;
    p.grad_loss = grad_loss;
    p.lse_in = lse_in;
    p.loss = loss;
    p.lse_out = lse_out;
    p.grad = grad;
    p.vocab = d->vocab;
    p.top = d->top;
    p.temperature = d->temperature;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const unsigned rows = unsigned(d->rows);
    const bool wide_index = d->index_type == OMNI_I64;
    if (d->dtype == OMNI_BF16)
        return wide_index ? enqueue<__nv_bfloat16, long long>(ctx, mode, p, rows, s) : enqueue<__nv_bfloat16, int>(ctx, mode, p, rows, s);
    return wide_index ? enqueue<float, long long>(ctx, mode, p, rows, s) : enqueue<float, int>(ctx, mode, p, rows, s);
}

}  // namespace
}  // namespace omni

using namespace omni;

extern "C" {

int omni_distill_forward(omni_ctx *ctx, const omni_distill *d, float *loss, float *lse, void *stream)
{
    return run(ctx, kForward, d, nullptr, nullptr, loss, lse, nullptr, 0, stream);
}

int omni_distill_backward(omni_ctx *ctx, const omni_distill *d, const float *lse, const float *grad_loss, void *grad,
                          uint64_t grad_stride, void *stream)
{
    return run(ctx, kBackward, d, lse, grad_loss, nullptr, nullptr, grad, grad_stride, stream);
}

int omni_distill_step(omni_ctx *ctx, const omni_distill *d, const float *grad_loss, float *loss, float *lse, void *grad,
                      uint64_t grad_stride, void *stream)
{
    return run(ctx, kStep, d, nullptr, grad_loss, loss, lse, grad, grad_stride, stream);
}

}  // extern "C"
