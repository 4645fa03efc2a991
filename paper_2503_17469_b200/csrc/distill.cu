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
#include "context.h"
#include "row_softmax.cuh"

namespace omni {
namespace {

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

// ---- a CTA per row, from global memory ----------------------------------------------------------

constexpr int kRowWalkers = 256;

// The CTA's row, walked by all warps but the teacher's.
template <typename T> __device__ __forceinline__ Row<T> row_of(const DistillParams &p)
{
    return Row<T>(static_cast<const T *>(p.logits) + blockIdx.x * p.row_stride, p.vocab, blockDim.x - 32);
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
            for (unsigned v = tid; v < unsigned(p.vocab); v += walkers) out[v] = from_float<T>(0.0f);
        } else if (same_phase(out, w.row)) {
            walk<AHEAD>(w, [&](int g, const auto &x) {
#pragma unroll
                for (int a = 0; a < int(sizeof x / sizeof x[0]); ++a)
                    put_group(out + w.parts.head + (long long)(g + a * walkers) * kGroup, x[a], q);
            });
            if (w.edge() >= 0) out[w.edge()] = from_float<T>(q(to_float(w.row[w.edge()])));
        } else {
            for (unsigned v = tid; v < unsigned(p.vocab); v += walkers) out[v] = from_float<T>(q(to_float(w.row[v])));
        }
    }
    __syncthreads();
    if (target) put_entries(p, te, out, gain, q, tid, blockDim.x);
}

// A row far from zero from its start, by the whole CTA.
template <typename T, int MODE> __device__ __forceinline__ void far_row(const DistillParams &p, const Teacher &te, Joined *cell)
{
    const Row<T> w = row_of<T>(p);
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
    const Row<T> w = row_of<T>(p);
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
