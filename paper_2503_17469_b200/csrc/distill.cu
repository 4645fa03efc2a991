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
// 128-140 us, 5.6-6.1 TB/s); the step its two exponentials per element, 8 cycles per warp and scheduler each, and its
// instructions beside three passes of L2 (8192 x 50257 bfloat16, rows on 2-byte boundaries: 319-335 us, 4.9-5.2 TB/s of
// the read and the write).  Few rows leave SMs idle: 1 to 148 rows of 131072 bfloat16 12-14 us a loss.  A gradient whose rows lie to
// 16-byte boundaries in another way than the logits' is written element by element: 8192 x 50257 of 50304 into dense rows 873
// instead of 319 us a step.  Tried for the step: the row kept in shared memory by a cluster 392-448 us; a persistent ring of bulk
// copies, the row held in it, 407-470 us: many warps from several rows hide the exponentials better than a held row saves.
// 256 walkers and four CTAs an SM; 128 and seven 390 us, 512 and three 326 (and 137 against 133 for the loss alone).
#include <type_traits>

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

// A thread's running maximum m and sum of exponentials over it, unit = log2(e) / T.  Near zero m = z unit, and an exponential
// 2^(z unit - m) is one fused multiply-add: whatever the rounding of m was, the sum carries it too.  Far from zero (a row masked by
// the type's lowest value or -1e30, say) that rounding, or an overflow, would leave nothing of the row, so such rows are
// walked again with m = z and 2^((z - m) unit).  Differences first for every row would cost 8192 x 50257 bfloat16 338.9 instead of
// 334.8 us a step and 3000 x 131072 142.5 instead of 139.5 us a loss.
// Products and sums are spelled out where the compiler could contract them one way in one variant and another way in the next:
// forward and step give the same bits.
constexpr float kFar = 16777216.0f;                  // of a row's m: from here on its rounding is a factor of two and more

template <bool FAR> struct Running {
    float m = -INFINITY;
    float2 a = {0.0f, 0.0f}, b = {0.0f, 0.0f};
    template <typename T, int K> __device__ __forceinline__ void take(const Group<T> (&g)[K], float unit)
    {
        float top = g[0].largest();
#pragma unroll
        for (int k = 1; k < K; ++k) top = fmaxf(top, g[k].largest());
        raise(FAR ? top : __fmul_rn(top, unit), unit);
        const float ref = reference(m);
        const float2 u = {unit, unit}, r = {ref, ref};
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 z = g[k].pair(i), x = FAR ? mul2(add2(z, r), u) : fma2(z, u, r);
                const float2 e = {exp2_fast(x.x), exp2_fast(x.y)};
                if (i % 2 == 0) a = add2(a, e);
                else b = add2(b, e);
            }
    }
    __device__ __forceinline__ void take_one(float z, float unit)
    {
        raise(FAR ? z : __fmul_rn(z, unit), unit);
        a.x += exp2_fast(FAR ? __fmul_rn(__fadd_rn(z, reference(m)), unit) : __fmaf_rn(z, unit, reference(m)));
    }
    __device__ __forceinline__ void raise(float to, float unit)
    {
        if (to > m) {                                // rare after the first few groups
            const float f = ratio(m, to, unit);
            a = mul2(a, {f, f});
            b = mul2(b, {f, f});
            m = to;
        }
    }
    __device__ __forceinline__ float sum() const { return __fadd_rn(__fadd_rn(a.x, a.y), __fadd_rn(b.x, b.y)); }
    // what is added to an exponent; -inf - -inf would be no number
    __device__ __forceinline__ static float reference(float m) { return m == -INFINITY ? 0.0f : -m; }
    // of a sum over `from` to one over `to`
    __device__ __forceinline__ static float ratio(float from, float to, float unit) { return exp2_fast(FAR ? __fmul_rn(from - to, unit) : from - to); }
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
// The warp's pairs of maximum and sum as one: the sum for the largest maximum.
template <bool FAR> __device__ __forceinline__ Joined join_warp(float own, float s, float unit)
{
    const float m = warp_max(own);
    return {m, warp_sum(m == -INFINITY || own == m ? s : __fmul_rn(s, Running<FAR>::ratio(own, m, unit)))};
}
// A warp's maximum and sum into its cell.
template <bool FAR> __device__ __forceinline__ void put_warp(const Running<FAR> &run, float unit, Joined *cell)
{
    const Joined w = join_warp<FAR>(run.m, run.sum(), unit);
    if (threadIdx.x % 32 == 0) *cell = w;
}
// The walkers' cells joined, by every warp for itself.
template <bool FAR> __device__ __forceinline__ Joined join_cells(const Joined *cell, int n, float unit)
{
    const int lane = threadIdx.x % 32;
    const Joined x = lane < n ? cell[lane] : Joined{-INFINITY, 0.0f};
    return join_warp<FAR>(x.m, x.s, unit);
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
    float best;                                     // the largest of the student's logits there, if it is finite, else 0
    float term;                                     // sum of p (log p - (z - best) / T)
    int target;                                     // some entry has a probability
    int repeated;                                   // some place is named twice
};

// One warp's work, beside the walk over the row.  `seen`: a table of 2 OMNI_DISTILL_MAX_TOP places.
template <typename T, typename I>
__device__ __forceinline__ void teacher_warp(const DistillParams &p, unsigned long long r, const T *row, Teacher &te, int *seen)
{
    const int lane = threadIdx.x % 32;
    const float *logit = p.top_logits + r * p.top_stride;
    float top = -INFINITY, best = -INFINITY;
    int table = 32;                                 // at least twice the entries
    while (table < 2 * p.top) table *= 2;
    for (int j = lane; j < table; j += 32) seen[j] = -1;
    __syncwarp();
    bool repeated = false;
    for (int j = lane; j < p.top; j += 32) {
        const long long i = load_index<I>(p.top_index, r * p.top_stride + j);
        const bool there = i >= 0 && i < p.vocab;
        const float t = there ? logit[j] : -INFINITY;
        te.place[j] = there ? int(i) : -1;
        te.hit[j] = there ? to_float(row[i]) : 0.0f;
        te.prob[j] = t;
        top = fmaxf(top, t);
        if (there) best = fmaxf(best, te.hit[j]);
        for (int h = int(unsigned(i) * 2654435769u >> 16) & (table - 1); there; h = (h + 1) & (table - 1)) {
            const int old = atomicCAS(&seen[h], -1, int(i));
            repeated |= old == int(i);
            if (old == -1 || old == int(i)) break;
        }
    }
    repeated = __any_sync(~0u, repeated);
    top = warp_max(top);
    best = warp_max(best);
    if (!isfinite(best)) best = 0.0f;
    float total = 0.0f;
    for (int j = lane; j < p.top; j += 32) {
        // the difference first: entries at the type's lowest value throughout would overflow at T < 1 and not be there
        const float e = top == -INFINITY && !isnan(te.prob[j]) ? 0.0f : expf(__fsub_rn(te.prob[j], top) / p.temperature);
        te.prob[j] = e;
        total += e;
    }
    total = warp_sum(total);
    const bool target = !(total == 0.0f);           // NaN counts as a target and shows
    float term = 0.0f;
    for (int j = lane; j < p.top; j += 32) {
        const float q = target ? te.prob[j] / total : 0.0f;
        te.prob[j] = q;
        if (!(q == 0.0f)) term = __fadd_rn(term, __fmul_rn(q, logf(q) - __fsub_rn(te.hit[j], best) / p.temperature));
    }
    term = warp_sum(term);
    if (lane == 0) {
        te.best = best;
        te.term = term;
        te.target = target;
        te.repeated = repeated;
    }
    __syncwarp();
}

// share * 2^((z times + add) unit) of a logit z: gain (the row's weight times T) times the student's probability of the token.  From
// the row's own maximum and sum near zero (u, -m, 1, gain / s) and far from it (1, -m, u, gain / s), with u = log2(e) / T; from a kept
// lse (1 / T, -lse, log2(e), gain), where the difference comes first too, and a product with 1 / T that is rounded once
// with it is exact if T is a power of two.  NEAR: unit is 1.
template <bool NEAR> struct Softmax {
    float times, add, unit, share;
    __device__ __forceinline__ float operator()(float z) const
    {
        const float x = __fmaf_rn(z, times, add);
        return __fmul_rn(exp2_fast(NEAR ? x : __fmul_rn(x, unit)), share);
    }
    __device__ __forceinline__ float2 operator()(float2 z) const
    {
        float2 x = fma2(z, {times, times}, {add, add});
        if (!NEAR) x = mul2(x, {unit, unit});
        return mul2({exp2_fast(x.x), exp2_fast(x.y)}, {share, share});
    }
};

// The gradient at the teacher's entries, over what the walk wrote there; an entry that names a token again is
// left to the first.
template <typename T, bool NEAR>
__device__ __forceinline__ void put_entries(const DistillParams &p, const Teacher &te, T *out, float gain, const Softmax<NEAR> &q, int from, int step)
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
        if (first) out[at] = from_float<T>(__fmaf_rn(-gain, total, q(te.hit[j])));
    }
}

template <typename T, bool NEAR>
__device__ __forceinline__ void put_group(T *dst, const Group<T> &g, const Softmax<NEAR> &q)
{
    float f[kGroup];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = q(g.pair(i));
        f[2 * i] = y.x;
        f[2 * i + 1] = y.y;
    }
    store_streaming(dst, f);
}
__device__ __forceinline__ bool same_phase(const void *a, const void *b)
{
    return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}

// ---- a CTA per row, from global memory ----------------------------------------------------------

constexpr int kRowWalkers = 256;

// What every thread of a row's CTA knows.
template <typename T> struct Row {
    const T *row;
    Parts<T> parts;
    int walkers, vocab;
    __device__ __forceinline__ Row(const DistillParams &p)
        : row(static_cast<const T *>(p.logits) + blockIdx.x * p.row_stride), parts(row, p.vocab), walkers(blockDim.x - 32), vocab(p.vocab) {}
    // the thread's element outside the groups, or -1
    __device__ __forceinline__ int edge() const { return int(threadIdx.x) < vocab - parts.groups * kGroup ? parts.edge(threadIdx.x) : -1; }
};

// f(first group, groups) over the groups of a thread: AHEAD at a time, then one by one.
template <int AHEAD, typename T, typename F> __device__ __forceinline__ void walk(const Row<T> &w, F f)
{
    int g = threadIdx.x;
    if constexpr (AHEAD > 1) {
        for (; g + (AHEAD - 1) * w.walkers < w.parts.groups; g += w.walkers * AHEAD) {
            Group<T> x[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) x[a].load(w.row + w.parts.head + (long long)(g + a * w.walkers) * kGroup);
            f(g, x);
        }
    }
    for (; g < w.parts.groups; g += w.walkers) {
        Group<T> x[1];
        x[0].load(w.row + w.parts.head + (long long)g * kGroup);
        f(g, x);
    }
}

// The walkers' maxima and sums into their warps' cells.
template <bool FAR, int AHEAD, typename T>
__device__ __forceinline__ void reduce_row(const Row<T> &w, float unit, Joined *cell)
{
    Running<FAR> run;
    walk<AHEAD>(w, [&](int, const auto &x) { run.take(x, unit); });
    if (w.edge() >= 0) run.take_one(to_float(w.row[w.edge()]), unit);
    __syncwarp();
    put_warp(run, unit, cell + threadIdx.x / 32);
}

// The gradient of the row, by the whole CTA.
template <int AHEAD, typename T, bool NEAR>
__device__ __forceinline__ void put_row(const DistillParams &p, const Row<T> &w, const Teacher &te, const Softmax<NEAR> &q, float gain)
{
    T *out = static_cast<T *>(p.grad) + blockIdx.x * p.grad_stride;
    const int tid = threadIdx.x, walkers = w.walkers;
    const bool target = te.target;
    if (tid < walkers) {
        if (!target) {
            for (int v = tid; v < p.vocab; v += walkers) out[v] = from_float<T>(0.0f);
        } else if (same_phase(out, w.row)) {
            walk<AHEAD>(w, [&](int g, const auto &x) {
#pragma unroll
                for (int a = 0; a < int(sizeof x / sizeof x[0]); ++a)
                    put_group(out + w.parts.head + (long long)(g + a * walkers) * kGroup, x[a], q);
            });
            if (w.edge() >= 0) out[w.edge()] = from_float<T>(q(to_float(w.row[w.edge()])));
        } else {
            for (int v = tid; v < p.vocab; v += walkers) out[v] = from_float<T>(q(to_float(w.row[v])));
        }
    }
    __syncthreads();
    if (target) put_entries(p, te, out, gain, q, tid, blockDim.x);
}

// A row far from zero from its start, by the whole CTA.
template <typename T, int MODE> __device__ __forceinline__ void far_row(const DistillParams &p, const Teacher &te, Joined *cell)
{
    const Row<T> w(p);
    const float unit = kLog2e / p.temperature;
    __syncthreads();                                // the cells have been read
    if (int(threadIdx.x) < w.walkers) reduce_row<true, 1>(w, unit, cell);
    __syncthreads();
    const Joined all = join_cells<true>(cell, w.walkers / 32, unit);
    const bool nothing = all.m == -INFINITY && all.s == 0.0f;         // a row of -inf: no token has a probability
    if (threadIdx.x == 0) {
        const float log_sum = __fmul_rn(log2f(all.s), kLn2), t = p.temperature;
        p.lse_out[blockIdx.x] = __fadd_rn(all.m / t, log_sum);
        const float ahead = nothing ? 0.0f : __fadd_rn(__fsub_rn(all.m, te.best) / t, log_sum);
        p.loss[blockIdx.x] = te.target ? __fmul_rn(__fmul_rn(t, t), __fadd_rn(te.term, ahead)) : 0.0f;
    }
    if constexpr (MODE == kStep) {
        const float gain = __fmul_rn(p.grad_loss[blockIdx.x], p.temperature);
        put_row<1>(p, w, te, Softmax<false>{1.0f, Running<true>::reference(all.m), unit, nothing ? 0.0f : gain / all.s}, gain);
    }
}

template <typename T, typename I, int MODE>
__global__ void __launch_bounds__(kRowWalkers + 32, 4) row_kernel(const __grid_constant__ DistillParams p)
{
    __shared__ Joined cell[kRowWalkers / 32];
    __shared__ Teacher te;
    __shared__ int seen[2 * OMNI_DISTILL_MAX_TOP];
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;  // groups a thread has in flight
    const Row<T> w(p);
    const unsigned long long r = blockIdx.x;
    const float unit = kLog2e / p.temperature;
    const float weight = MODE == kForward ? 0.0f : p.grad_loss[r];
    const float lse = MODE == kBackward ? p.lse_in[r] : 0.0f;
    if (int(threadIdx.x) >= w.walkers) teacher_warp<T, I>(p, r, w.row, te, seen);
    else if constexpr (MODE != kBackward) reduce_row<false, kAhead>(w, unit, cell);
    __syncthreads();
    const float gain = __fmul_rn(weight, p.temperature);
    if constexpr (MODE == kBackward) {
        put_row<kAhead>(p, w, te, Softmax<false>{1.0f / p.temperature, lse == -INFINITY ? 0.0f : -lse, kLog2e, gain}, gain);
    } else {
        const Joined all = join_cells<false>(cell, w.walkers / 32, unit);     // every warp finds the same
        if (!(fabsf(all.m) < kFar)) {
            far_row<T, MODE>(p, te, cell);
            return;
        }
        if (threadIdx.x == 0) {
            const float log_sum = log2f(all.s);
            p.lse_out[r] = __fmul_rn(__fadd_rn(all.m, log_sum), kLn2);
            // the lse less the logit that the teacher's term is measured from: what is added up is all distances
            const float ahead = __fmul_rn(__fadd_rn(__fmaf_rn(-te.best, unit, all.m), log_sum), kLn2);
            p.loss[r] = te.target ? __fmul_rn(__fmul_rn(p.temperature, p.temperature), __fadd_rn(te.term, ahead)) : 0.0f;
        }
        if constexpr (MODE == kStep) put_row<kAhead>(p, w, te, Softmax<true>{unit, -all.m, 1.0f, gain / all.s}, gain);
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
