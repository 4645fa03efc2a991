// Clipped policy loss on sampled tokens with a divergence from a reference policy: log-probabilities, forward, backward, both in one pass.
//
// Per row: lse = log sum_v exp(z_v / T), logp = z_t / T - lse of the token t, and from scalars of the row the loss and its slope c by
// logp; the gradient is w ([v = t] - exp(z_v / T - lse)) with w = grad_loss c / T.  The floor is one read of the logits and one
// write of the gradient.
//
// A CTA owns a row.  The first walk keeps a running maximum and sum per thread, the second finds the row, which the same CTA
// read a moment ago, in L2.  A row whose weight is zero (its ratio is clipped) is not walked again: zeros are written.
#include "context.h"
#include "row_softmax.cuh"

namespace omni {
namespace {

constexpr int kWalkers = 256, kMostWalkers = 512;     // threads of a row: backward; forward and step
constexpr int kMostHeld = 112 * 1024;                 // bytes of a row that is held: two rows an SM
enum Mode { kForward = 0, kBackward = 1, kStep = 2 };

struct PolicyParams {
    const void *logits;
    unsigned long long row_stride, grad_stride;
    const void *tokens;
    const float *old, *advantage, *reference;
    const float *grad_loss, *lse_in;
    float *loss, *logp, *lse_out;                     // loss: NULL for the log-probabilities alone
    void *grad;
    int vocab;
    float low, high, kl, temperature;                 // low, high: borders of the ratio
};

// A row's scalars, the same in every thread.
struct Sample {
    int token;                                        // -1: none
    float z;                                          // its logit
    __device__ __forceinline__ bool there() const { return token >= 0; }
};
template <typename T, typename I> __device__ __forceinline__ Sample sample_of(const PolicyParams &p, const T *row)
{
    const long long t = load_index<I>(p.tokens, blockIdx.x);
    const bool there = t >= 0 && t < p.vocab;
    return {there ? int(t) : -1, there ? to_float(row[t]) : 0.0f};
}

struct Value { float loss, slope; };
// The loss of a row with a token and its derivative by logp.  On a border of the ratio the surrogate counts as not clipped; an advantage
// of zero takes no part, whatever the ratio.
__device__ __forceinline__ Value value_of(const PolicyParams &p, float logp)
{
    const float a = p.advantage[blockIdx.x];
    const float ratio = expf(__fsub_rn(logp, p.old[blockIdx.x]));
    Value v = {0.0f, 0.0f};
    if (a != 0.0f) {
        const float gain = __fmul_rn(ratio, a), clipped = __fmul_rn(fminf(fmaxf(ratio, p.low), p.high), a);
        const bool taken = gain <= clipped, other = gain > clipped;     // neither: a NaN, which shows
        v.loss = taken ? -gain : other ? -clipped : gain + clipped;
        v.slope = taken ? -gain : other ? 0.0f : gain + clipped;
    }
    if (p.kl != 0.0f) {
        const float gap = __fsub_rn(p.reference[blockIdx.x], logp), away = expm1f(gap);
        v.loss = __fmaf_rn(p.kl, __fsub_rn(away, fminf(gap, 3.4e38f)), v.loss);     // infinite for an infinite gap, not inf - inf
        v.slope = __fmaf_rn(-p.kl, away, v.slope);
    }
    return v;
}

// A row's groups as its threads fetch them ahead, each thread those that it walks: two groups to a step, 64 to 128 bytes in flight.
// With HELD every group has a place of its own, and the second walk finds the row in shared memory; otherwise a few places go round.
template <typename T, bool HELD> struct Fetched {
    static constexpr int kStep = 2, kAhead = sizeof(T) == 2 ? 4 : 2;
    const Row<T> &w;
    char *const at;
    int own, fetched = 0;                             // groups of this thread, groups asked for
    __device__ __forceinline__ Fetched(const Row<T> &row, char *shared)
        : w(row), at(shared), own((row.parts.groups - int(threadIdx.x) + row.walkers - 1) / row.walkers) {}
    static __host__ __device__ size_t bytes(int vocab, int walkers)
    {
        return HELD ? size_t(vocab / kGroup) * kGroup * sizeof(T) : size_t(kStep * kAhead) * walkers * kGroup * sizeof(T);
    }
    __device__ __forceinline__ char *place(int i) const
    {
        return at + size_t(((HELD ? i : i % (kStep * kAhead)) * w.walkers + threadIdx.x)) * (kGroup * sizeof(T));
    }
    __device__ __forceinline__ void ask()
    {
#pragma unroll
        for (int i = 0; i < kStep; ++i, ++fetched) {
            if (fetched >= own) continue;
            const char *from = reinterpret_cast<const char *>(w.row + w.parts.head + (long long)(threadIdx.x + fetched * w.walkers) * kGroup);
            const uint32_t to = uint32_t(__cvta_generic_to_shared(place(fetched)));
#pragma unroll
            for (int piece = 0; piece < int(kGroup * sizeof(T)) / 16; ++piece)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + piece * 16), "l"(from + piece * 16) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ Group<T> group(int i) const { return *reinterpret_cast<const Group<T> *>(place(i)); }
};

// The walkers' maxima and sums into their warps' cells, over groups that are fetched ahead.
template <typename T, bool HELD> __device__ __forceinline__ void reduce_fetched(Fetched<T, HELD> &f, float unit, Joined *cell)
{
    constexpr int kStep = f.kStep, kAhead = f.kAhead;
    Running<false> run;
    if (f.w.edge() >= 0) run.take_one(to_float(f.w.row[f.w.edge()]), unit);
    for (int i = 0; i < f.own; i += kStep) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
        if (i + kStep <= f.own) {
            Group<T> x[kStep];
#pragma unroll
            for (int k = 0; k < kStep; ++k) x[k] = f.group(i + k);
            run.take(x, unit);
        } else {
            for (int k = i; k < f.own; ++k) {
                Group<T> x[1] = {f.group(k)};
                run.take(x, unit);
            }
        }
        f.ask();
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    put_warp(run, unit, cell + threadIdx.x / 32);
}

// f(first group, groups) over the groups of a thread that are held, as walk() over those in memory.
template <int AHEAD, typename T, bool HELD, typename F> __device__ __forceinline__ void walk(const Fetched<T, HELD> &held, F f)
{
    int i = 0;
    for (; i + AHEAD <= held.own; i += AHEAD) {
        Group<T> x[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) x[a] = held.group(i + a);
        f(int(threadIdx.x) + i * held.w.walkers, x);
    }
    for (; i < held.own; ++i) {
        Group<T> x[1] = {held.group(i)};
        f(int(threadIdx.x) + i * held.w.walkers, x);
    }
}

// The gradient of the row, by the whole CTA, from the groups of `walked` (the row itself, or what is held of it).  q(z) is -weight times
// the probability of a token with logit z.
template <int AHEAD, typename W, typename T, bool NEAR>
__device__ __forceinline__ void put_row(const PolicyParams &p, const W &walked, const Row<T> &w, const Sample &t, const Softmax<NEAR> &q, float weight)
{
    T *out = static_cast<T *>(p.grad) + blockIdx.x * p.grad_stride;
    const int tid = threadIdx.x, walkers = w.walkers;
    if (!t.there() || weight == 0.0f) {
        const Parts<T> parts(out, p.vocab);
        const float zeros[kGroup] = {};
        for (int g = tid; g < parts.groups; g += walkers) store_streaming(out + parts.head + (long long)g * kGroup, zeros);
        if (tid < p.vocab - parts.groups * kGroup) out[parts.edge(tid)] = from_float<T>(0.0f);
        return;
    }
    if (same_phase(out, w.row)) {
        walk<AHEAD>(walked, [&](int g, const auto &x) {
#pragma unroll
            for (int a = 0; a < int(sizeof x / sizeof x[0]); ++a)
                put_group(out + w.parts.head + (long long)(g + a * walkers) * kGroup, x[a], q);
        });
        if (w.edge() >= 0) out[w.edge()] = from_float<T>(q(to_float(w.row[w.edge()])));
    } else {
        for (int v = tid; v < p.vocab; v += walkers) out[v] = from_float<T>(q(to_float(w.row[v])));
    }
    __syncthreads();
    if (tid == 0) out[t.token] = from_float<T>(__fadd_rn(weight, q(t.z)));
}

// What follows from a row's log-sum-exp and its token's log-probability.
__device__ __forceinline__ float finish(const PolicyParams &p, const Sample &t, float lse, float logp, bool step)
{
    const Value v = t.there() && (step || p.loss) ? value_of(p, logp) : Value{0.0f, 0.0f};
    if (threadIdx.x == 0) {
        p.lse_out[blockIdx.x] = lse;
        p.logp[blockIdx.x] = t.there() ? logp : 0.0f;
        if (p.loss) p.loss[blockIdx.x] = v.loss;
    }
    return step ? __fdiv_rn(__fmul_rn(p.grad_loss[blockIdx.x], v.slope), p.temperature) : 0.0f;
}

// A row far from zero from its start, by the whole CTA.
template <typename T, int MODE> __device__ __forceinline__ void far_row(const PolicyParams &p, const Row<T> &w, const Sample &t, Joined *cell)
{
    const float unit = kLog2e / p.temperature;
    __syncthreads();                                  // the cells have been read
    reduce_row<true, 1>(w, unit, cell);
    __syncthreads();
    const Joined all = join_cells<true>(cell, w.walkers / 32, unit);
    const bool nothing = all.m == -INFINITY && all.s == 0.0f;           // a row of -inf: no token has a probability
    const float log_sum = __fmul_rn(log2f(all.s), kLn2);
    const float logp = nothing ? -INFINITY : __fsub_rn(__fsub_rn(t.z, all.m) / p.temperature, log_sum);
    const float weight = finish(p, t, __fadd_rn(all.m / p.temperature, log_sum), logp, MODE == kStep);
    if constexpr (MODE == kStep)
        put_row<1>(p, w, w, t, Softmax<false>{1.0f, Running<true>::reference(all.m), unit, nothing ? 0.0f : -weight / all.s}, weight);
}

// From a kept lse: one walk.
template <typename T, typename I> __global__ void __launch_bounds__(kWalkers, 4) policy_backward_kernel(const __grid_constant__ PolicyParams p)
{
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;    // groups a thread has in flight
    const Row<T> w(static_cast<const T *>(p.logits) + blockIdx.x * p.row_stride, p.vocab, blockDim.x);
    const Sample t = sample_of<T, I>(p, w.row);
    const float lse = p.lse_in[blockIdx.x];
    const float logp = __fsub_rn(t.z / p.temperature, lse);
    const float slope = t.there() ? value_of(p, t.z == -INFINITY ? -INFINITY : logp).slope : 0.0f;
    const float weight = __fdiv_rn(__fmul_rn(p.grad_loss[blockIdx.x], slope), p.temperature);
    __syncthreads();                                  // every thread has the token's logit: the gradient may be written over it
    put_row<kAhead>(p, w, w, t, Softmax<false>{1.0f / p.temperature, lse == -INFINITY ? 0.0f : -lse, kLog2e, -weight}, weight);
}

template <typename T, typename I, bool STEP, bool HELD>
__global__ void __launch_bounds__(kMostWalkers, 2) policy_kernel(const __grid_constant__ PolicyParams p)
{
    extern __shared__ __align__(16) char shared[];
    __shared__ Joined cell[kMostWalkers / 32];
    const Row<T> w(static_cast<const T *>(p.logits) + blockIdx.x * p.row_stride, p.vocab, blockDim.x);
    Fetched<T, HELD> fetched(w, shared);
#pragma unroll
    for (int i = 0; i < fetched.kAhead; ++i) fetched.ask();
    const Sample t = sample_of<T, I>(p, w.row);
    const float unit = kLog2e / p.temperature;
    reduce_fetched(fetched, unit, cell);
    __syncthreads();
    const Joined all = join_cells<false>(cell, w.walkers / 32, unit);         // every warp finds the same
    if (!(fabsf(all.m) < kFar)) {
        far_row<T, STEP ? kStep : kForward>(p, w, t, cell);
        return;
    }
    const float log_sum = log2f(all.s);
    // the token's exponent less the maximum first: what is added up is all distances
    const float logp = __fmul_rn(__fsub_rn(__fmaf_rn(t.z, unit, -all.m), log_sum), kLn2);
    const float weight = finish(p, t, __fmul_rn(__fadd_rn(all.m, log_sum), kLn2), logp, STEP);
    if constexpr (STEP) {
        const Softmax<true> q{unit, -all.m, 1.0f, -weight / all.s};
        if constexpr (HELD) put_row<2>(p, fetched, w, t, q, weight);
        else put_row<sizeof(T) == 2 ? 4 : 2>(p, w, w, t, q, weight);
    }
}

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool finite(float x) { return x - x == 0.0f; }

// valued: the loss or its gradient is asked for, not the log-probabilities alone.
int check_policy(const omni_policy *d, bool valued)
{
    if (!d) return OMNI_ERR_NULL;
    if ((d->dtype != OMNI_F32 && d->dtype != OMNI_BF16) || (d->index_type != OMNI_I32 && d->index_type != OMNI_I64)) return OMNI_ERR_BAD_CONFIG;
    if (d->vocab < 1 || !(d->temperature > 0.0f) || !finite(d->temperature)) return OMNI_ERR_BAD_CONFIG;
    if (valued && (!(d->clip_low >= 0.0f) || !(d->clip_high >= 0.0f) || !(d->kl >= 0.0f) || !finite(d->clip_low) || !finite(d->clip_high) || !finite(d->kl)))
        return OMNI_ERR_BAD_CONFIG;
    if (d->rows >= (1ull << 31)) return OMNI_ERR_TOO_LARGE;
    if (d->rows > 1 && d->row_stride < uint64_t(d->vocab)) return OMNI_ERR_BAD_CONFIG;
    if (d->rows == 0) return OMNI_OK;
    if (!d->logits || !d->tokens) return OMNI_ERR_NULL;
    if (!aligned(d->logits, d->dtype == OMNI_BF16 ? 2 : 4) || !aligned(d->tokens, d->index_type == OMNI_I64 ? 8 : 4)) return OMNI_ERR_ALIGN;
    if (valued) {
        if (!d->old || !d->advantage || (d->kl != 0.0f && !d->reference)) return OMNI_ERR_NULL;
        if (!aligned(d->old, 4) || !aligned(d->advantage, 4) || !aligned(d->reference, 4)) return OMNI_ERR_ALIGN;
    }
    return OMNI_OK;
}

template <typename T, typename I> int enqueue(omni_ctx *ctx, int mode, const PolicyParams &p, unsigned rows, cudaStream_t s)
{
    const int most = mode == kBackward ? kWalkers : kMostWalkers;
    int walkers = 64;
    while (walkers < most && walkers * 8 * kGroup < p.vocab) walkers *= 2;
    if (mode == kBackward) {
        policy_backward_kernel<T, I><<<rows, walkers, 0, s>>>(p);
        return context_launched(ctx, int(cudaGetLastError()));
    }
    const bool held = mode == kStep && Fetched<T, true>::bytes(p.vocab, walkers) <= size_t(kMostHeld);
    const size_t bytes = held ? Fetched<T, true>::bytes(p.vocab, walkers) : Fetched<T, false>::bytes(p.vocab, walkers);
    void (*const kernel)(PolicyParams) = mode == kForward ? policy_kernel<T, I, false, false> : held ? policy_kernel<T, I, true, true> : policy_kernel<T, I, true, false>;
    const int rc = bytes > 40 * 1024 ? context_shared(ctx, reinterpret_cast<const void *>(kernel), kMostHeld) : OMNI_OK;
    if (rc != OMNI_OK) return rc;
    kernel<<<rows, walkers, bytes, s>>>(p);
    return context_launched(ctx, int(cudaGetLastError()));
}

struct Results {
    float *loss, *logp, *lse;
    void *grad;
    uint64_t grad_stride;
};

int run(omni_ctx *ctx, int mode, bool valued, const omni_policy *d, const float *lse_in, const float *grad_loss, const Results &r, void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_policy(d, valued);
    if (rc != OMNI_OK) return rc;
    if (d->rows > 0) {
        if (mode != kBackward && ((valued && !r.loss) || !r.logp || !r.lse)) return OMNI_ERR_NULL;
        if (mode != kForward && (!r.grad || !grad_loss || (mode == kBackward && !lse_in))) return OMNI_ERR_NULL;
        if (mode != kForward && d->rows > 1 && r.grad_stride < uint64_t(d->vocab)) return OMNI_ERR_BAD_CONFIG;
        if (!aligned(r.loss, 4) || !aligned(r.logp, 4) || !aligned(r.lse, 4) || !aligned(lse_in, 4) || !aligned(grad_loss, 4) ||
            !aligned(r.grad, d->dtype == OMNI_BF16 ? 2 : 4))
            return OMNI_ERR_ALIGN;
    }
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK || d->rows == 0) return rc;
    PolicyParams p;
    p.logits = d->logits;
    p.row_stride = d->row_stride;
    p.grad_stride = r.grad_stride;
    p.tokens = d->tokens;
    p.old = d->old;
    p.advantage = d->advantage;
    p.reference = d->reference;
    p.grad_loss = grad_loss;
    p.lse_in = lse_in;
    p.loss = r.loss;
    p.logp = r.logp;
    p.lse_out = r.lse;
    p.grad = r.grad;
    p.vocab = d->vocab;
    p.low = 1.0f - d->clip_low;
    p.high = 1.0f + d->clip_high;
    p.kl = d->kl;
    p.temperature = d->temperature;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const unsigned rows = unsigned(d->rows);
    const bool wide = d->index_type == OMNI_I64;
    if (d->dtype == OMNI_BF16)
        return wide ? enqueue<__nv_bfloat16, long long>(ctx, mode, p, rows, s) : enqueue<__nv_bfloat16, int>(ctx, mode, p, rows, s);
    return wide ? enqueue<float, long long>(ctx, mode, p, rows, s) : enqueue<float, int>(ctx, mode, p, rows, s);
}

}  // namespace
}  // namespace omni

using namespace omni;

extern "C" {

int omni_policy_logprob(omni_ctx *ctx, const omni_policy *d, float *logp, float *lse, void *stream)
{
    return run(ctx, kForward, false, d, nullptr, nullptr, {nullptr, logp, lse, nullptr, 0}, stream);
}

int omni_policy_forward(omni_ctx *ctx, const omni_policy *d, float *loss, float *logp, float *lse, void *stream)
{
    return run(ctx, kForward, true, d, nullptr, nullptr, {loss, logp, lse, nullptr, 0}, stream);
}

int omni_policy_backward(omni_ctx *ctx, const omni_policy *d, const float *lse, const float *grad_loss, void *grad, uint64_t grad_stride,
                         void *stream)
{
    return run(ctx, kBackward, true, d, lse, grad_loss, {nullptr, nullptr, nullptr, grad, grad_stride}, stream);
}

int omni_policy_step(omni_ctx *ctx, const omni_policy *d, const float *grad_loss, float *loss, float *logp, float *lse, void *grad,
                     uint64_t grad_stride, void *stream)
{
    return run(ctx, kStep, true, d, nullptr, grad_loss, {loss, logp, lse, grad, grad_stride}, stream);
}

}  // extern "C"
