// Clipped policy loss on sampled tokens with a divergence from a reference policy: log-probabilities, forward, backward, both in one pass.
//
// Per row: lse = log sum_v exp(z_v / T), logp = z_t / T - lse of the token t, and from scalars of the row the loss and its slope c by
// logp; the gradient is w ([v = t] - exp(z_v / T - lse)) with w = grad_loss c / T.  The floor is one read of the logits and one
// write of the gradient.
//
// A CTA owns a row.  The first walk keeps a running maximum and sum per thread; its groups come by asynchronous copies, 128 bytes a
// thread in flight, into places of the thread's own.  The second finds the row, which the same CTA read a moment ago, in L2, and marks its
// lines as the first to leave.  A row whose weight is zero (its ratio is clipped) is not walked again: zeros are written.
// What bounds it: the gradient alone the memory (4096 x 32000 float 154 us, 6.8 TB/s; rows that are walked for their sum first 181, 8192 x 50257
// bfloat16 349 for 263); log-probabilities the memory beside one exponential an
// element, 74 % of the special-function units (3000 x 131072 bfloat16 122-135 us, floor 120); the step two exponentials and two reads of L2 (8192 x
// 50257 bfloat16, rows on 2-byte boundaries, 287 us, 323 when the 1000 W cap has brought the clock down to 1.6 GHz; floor 252).
// Rows in flight have to stay in L2 between their walks: four CTAs of 256 an SM (59 MB) 287 us, five 336, six 372, three 309.  So the
// threads of a row follow its bytes: 32 for 8 KB (16384 x 1000 bfloat16 30 us, with 128 threads 53), 512 for 128 KB and more (3000 x 131072
// 301 us, with 256 threads 338).
// Tried for the step: the row held in shared memory, two CTAs of 512 an SM 329 us, the same with the next row's loads behind the gradient 339; a batch
// of loads in registers instead of the asynchronous ones 327.  A cluster of CTAs for each row above 128 KB, whatever their number: 68 x 168451 float
// 30 instead of 44 us, but 3000 x 131072 bfloat16 331 instead of 298 and its log-probabilities 180 instead of 129.
#include "context.h"
#include "row_softmax.cuh"

namespace omni {
namespace {

constexpr int kFewestWalkers = 32, kMostWalkers = 512; // threads of a row
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

// A row's scalars, the same in every thread; asked for before the walk.
struct Sample {
    int token;                                        // -1: none
    float z;                                          // its logit
    float old, advantage, reference, grad_loss;       // what is given of them
    __device__ __forceinline__ bool there() const { return token >= 0; }
};
template <typename T, typename I> __device__ __forceinline__ Sample sample_of(const PolicyParams &p, const T *row, unsigned r, bool weighed)
{
    const long long t = load_index<I>(p.tokens, r);
    const bool there = t >= 0 && t < p.vocab;
    return {there ? int(t) : -1, there ? to_float(row[t]) : 0.0f, p.old ? p.old[r] : 0.0f, p.old ? p.advantage[r] : 0.0f,
            p.kl != 0.0f ? p.reference[r] : 0.0f, weighed ? p.grad_loss[r] : 0.0f};
}

struct Value { float loss, slope; };
// The loss of a row with a token and its derivative by logp.  On a border of the ratio the surrogate counts as not clipped; an advantage
// of zero takes no part, whatever the ratio.
__device__ __forceinline__ Value value_of(const PolicyParams &p, const Sample &t, float logp)
{
    const float a = t.advantage, ratio = expf(__fsub_rn(logp, t.old));
    Value v = {0.0f, 0.0f};
    if (a != 0.0f) {
        const float gain = __fmul_rn(ratio, a), clipped = __fmul_rn(fminf(fmaxf(ratio, p.low), p.high), a);
        const bool taken = gain <= clipped, other = gain > clipped;     // neither: a NaN, which shows
        v.loss = taken ? -gain : other ? -clipped : gain + clipped;
        v.slope = taken ? -gain : other ? 0.0f : gain + clipped;
    }
    if (p.kl != 0.0f) {
        const float gap = __fsub_rn(t.reference, logp), away = expm1f(gap);
        v.loss = __fmaf_rn(p.kl, __fsub_rn(away, fminf(gap, 3.4e38f)), v.loss);     // infinite for an infinite gap, not inf - inf
        v.slope = __fmaf_rn(-p.kl, away, v.slope);
    }
    return v;
}

// What a thread walks of a row: groups threadIdx.x, + walkers, ... and at most one element outside them.
template <typename T> __device__ __forceinline__ int own_groups(const Row<T> &w)
{
    return (w.parts.groups - int(threadIdx.x) + w.walkers - 1) / w.walkers;
}

// Groups as the threads fetch them ahead, each thread its own, kStep of them to a step, into places of 16 or 32 bytes side by side.
template <typename T> struct Places {
    static constexpr int kSize = kGroup * int(sizeof(T)), kStep = 2;
    char *at;
    __device__ __forceinline__ char *place(int i, int walkers) const { return at + (i * walkers + int(threadIdx.x)) * kSize; }
    // groups i .. i + kStep - 1 of the thread into the places from `to` on
    __device__ __forceinline__ void ask(const Row<T> &w, int own, int i, int to) const
    {
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
            if (i + k >= own) break;
            const char *from = reinterpret_cast<const char *>(w.row + w.parts.head + (long long)(threadIdx.x + (i + k) * w.walkers) * kGroup);
            const uint32_t into = uint32_t(__cvta_generic_to_shared(place(to + k, w.walkers)));
#pragma unroll
            for (int piece = 0; piece < kSize / 16; ++piece)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(into + piece * 16), "l"(from + piece * 16) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ Group<T> group(int i, int walkers) const { return *reinterpret_cast<const Group<T> *>(place(i, walkers)); }
};
template <int LEFT> __device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Takes groups i .. of the thread's `own`, group(k) being i + k: the order of a row's sum, in every call.
template <typename T, typename F> __device__ __forceinline__ void take_step(Running<false> &run, int i, int own, float unit, F group)
{
    constexpr int kStep = Places<T>::kStep;
    if (i + kStep <= own) {
        Group<T> x[kStep];
#pragma unroll
        for (int k = 0; k < kStep; ++k) x[k] = group(k);
        run.take(x, unit);
    } else if (i < own) {
        Group<T> x[1] = {group(0)};
        run.take(x, unit);
    }
}

// The thread that writes a token's element of a gradient that is written in groups, and what it writes there.
template <typename T> __device__ __forceinline__ int owner_of(const Row<T> &w, int token)
{
    const int in = token - w.parts.head, grouped = w.parts.groups * kGroup;
    return in >= 0 && in < grouped ? in / kGroup % w.walkers : in < 0 ? token : token - grouped;
}
__device__ __forceinline__ float at_token(float weight, float q) { return __fadd_rn(weight, q); }

// A walk over a row that nothing reads again: its lines are the first to leave L2, so that rows that others are in the middle of stay.
__device__ __forceinline__ void load_last(uint4 &x, const void *p)
{
    unsigned long long policy;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p), "l"(policy) : "memory");
}
template <typename T> __device__ __forceinline__ Group<T> last_group(const T *p)
{
    union { uint4 u[sizeof(Group<T>) / 16]; Group<T> g; } x;
#pragma unroll
    for (int i = 0; i < int(sizeof(Group<T>) / 16); ++i) load_last(x.u[i], reinterpret_cast<const char *>(p) + 16 * i);
    return x.g;
}
template <int AHEAD, typename T, typename F> __device__ __forceinline__ void walk_last(const Row<T> &w, F f)
{
    const T *const first = w.row + w.parts.head;
    int g = threadIdx.x;
    for (; g + (AHEAD - 1) * w.walkers < w.parts.groups; g += w.walkers * AHEAD) {
        Group<T> x[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) x[a] = last_group(first + (long long)(g + a * w.walkers) * kGroup);
        f(g, x);
    }
    for (; g < w.parts.groups; g += w.walkers) {
        Group<T> x[1] = {last_group(first + (long long)g * kGroup)};
        f(g, x);
    }
}

// A row of zeros.
template <typename T> __device__ __forceinline__ void put_zeros(T *out, int vocab, int walkers)
{
    const Parts<T> parts(out, vocab);
    const float zeros[kGroup] = {};
    for (int g = threadIdx.x; g < parts.groups; g += walkers) store_streaming(out + parts.head + (long long)g * kGroup, zeros);
    if (int(threadIdx.x) < vocab - parts.groups * kGroup) out[parts.edge(threadIdx.x)] = from_float<T>(0.0f);
}

// The gradient of a row from memory, by the whole CTA.  q(z) is -weight times the probability of a token with logit z.
template <int AHEAD, typename T, bool NEAR>
__device__ __forceinline__ void put_row(const PolicyParams &p, T *out, const Row<T> &w, const Sample &t, const Softmax<NEAR> &q, float weight)
{
    const int tid = threadIdx.x, walkers = w.walkers;
    if (!t.there() || weight == 0.0f) {
        put_zeros(out, p.vocab, walkers);
        return;
    }
    int owner = t.token % walkers;
    if (same_phase(out, w.row)) {
        walk_last<AHEAD>(w, [&](int g, const auto &x) {
#pragma unroll
            for (int a = 0; a < int(sizeof x / sizeof x[0]); ++a)
                put_group(out + w.parts.head + (long long)(g + a * walkers) * kGroup, x[a], q);
        });
        if (w.edge() >= 0) out[w.edge()] = from_float<T>(q(to_float(w.row[w.edge()])));
        owner = owner_of(w, t.token);
    } else {
        for (unsigned v = tid; v < unsigned(p.vocab); v += walkers) out[v] = from_float<T>(q(to_float(w.row[v])));
    }
    if (tid == owner) out[t.token] = from_float<T>(at_token(weight, q(t.z)));     // over what the same thread wrote
}

// What follows from a row's log-sum-exp and its token's log-probability: the results (backward has none), and the weight of the gradient.
template <int MODE> __device__ __forceinline__ float finish(const PolicyParams &p, unsigned r, const Sample &t, float lse, float logp)
{
    const Value v = t.there() && (MODE != kForward || p.loss) ? value_of(p, t, logp) : Value{0.0f, 0.0f};
    if (MODE != kBackward && threadIdx.x == 0) {
        p.lse_out[r] = lse;
        p.logp[r] = t.there() ? logp : 0.0f;
        if (p.loss) p.loss[r] = v.loss;
    }
    return MODE != kForward ? __fdiv_rn(__fmul_rn(t.grad_loss, v.slope), p.temperature) : 0.0f;
}

template <typename T> __device__ __forceinline__ T *gradient_of(const PolicyParams &p, unsigned r) { return static_cast<T *>(p.grad) + r * p.grad_stride; }

// A row far from zero from its start, by the whole CTA.
template <typename T, int MODE> __device__ __forceinline__ void far_row(const PolicyParams &p, unsigned r, const Row<T> &w, const Sample &t, Joined *cell)
{
    const float unit = kLog2e / p.temperature;
    __syncthreads();                                  // the cells have been read
    reduce_row<true, 1>(w, unit, cell);
    __syncthreads();
    const Joined all = join_cells<true>(cell, w.walkers / 32, unit);
    const bool nothing = all.m == -INFINITY && all.s == 0.0f;           // a row of -inf: no token has a probability
    const float log_sum = __fmul_rn(log2f(all.s), kLn2);
    const float logp = nothing ? -INFINITY : __fsub_rn(__fsub_rn(t.z, all.m) / p.temperature, log_sum);
    const float weight = finish<MODE>(p, r, t, __fadd_rn(all.m / p.temperature, log_sum), logp);
    if constexpr (MODE != kForward)
        put_row<1>(p, gradient_of<T>(p, r), w, t, Softmax<false>{1.0f, Running<true>::reference(all.m), unit, nothing ? 0.0f : -weight / all.s}, weight);
}

// A row near zero: its results; the gradient's softmax and weight.
struct Ending { Softmax<true> q; float weight; };
template <int MODE> __device__ __forceinline__ Ending near_row(const PolicyParams &p, unsigned r, const Sample &t, const Joined &all, float unit)
{
    const float log_sum = log2f(all.s);
    // the token's exponent less the maximum first: what is added up is all distances
    const float logp = __fmul_rn(__fsub_rn(__fmaf_rn(t.z, unit, -all.m), log_sum), kLn2);
    const float weight = finish<MODE>(p, r, t, __fmul_rn(__fadd_rn(all.m, log_sum), kLn2), logp);
    return {{unit, -all.m, 1.0f, -weight / all.s}, weight};
}

// From the threads' maxima and sums of a row to its results and its gradient.
template <typename T> constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;       // groups a thread has in flight in the second walk
template <typename T, int MODE>
__device__ __forceinline__ void end_row(const PolicyParams &p, unsigned r, const Row<T> &w, const Sample &t, const Running<false> &run, float unit, Joined *cell)
{
    __syncwarp();
    put_warp(run, unit, cell + threadIdx.x / 32);
    __syncthreads();
    const Joined all = join_cells<false>(cell, w.walkers / 32, unit);         // every warp finds the same
    if (!(fabsf(all.m) < kFar)) {
        far_row<T, MODE>(p, r, w, t, cell);
        return;
    }
    const Ending end = near_row<MODE>(p, r, t, all, unit);
    if constexpr (MODE != kForward) put_row<kAhead<T>>(p, gradient_of<T>(p, r), w, t, end.q, end.weight);
}

// A CTA a row; a few places go round.  The gradient of a step finds the row in L2.
template <typename T> constexpr int kRound = sizeof(T) == 2 ? 8 : 4;       // places of a thread
template <typename T, typename I, int MODE> __global__ void __launch_bounds__(kMostWalkers, 2) policy_kernel(const __grid_constant__ PolicyParams p)
{
    extern __shared__ __align__(16) char shared[];
    __shared__ Joined cell[kMostWalkers / 32];
    constexpr int kStep = Places<T>::kStep, kSteps = kRound<T> / kStep;
    const unsigned r = blockIdx.x;
    const Row<T> w(static_cast<const T *>(p.logits) + r * p.row_stride, p.vocab, blockDim.x);
    const Places<T> at{shared};
    const int own = own_groups(w);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) at.ask(w, own, i * kStep, i * kStep);
    const Sample t = sample_of<T, I>(p, w.row, r, MODE == kStep);
    const float unit = kLog2e / p.temperature;
    Running<false> run;
    if (w.edge() >= 0) run.take_one(to_float(w.row[w.edge()]), unit);
    for (int i = 0; i < own; i += kStep) {
        arrived<kSteps - 1>();
        take_step<T>(run, i, own, unit, [&](int k) { return at.group(i % kRound<T> + k, w.walkers); });
        at.ask(w, own, i + kRound<T>, i % kRound<T>);
    }
    end_row<T, MODE>(p, r, w, t, run, unit, cell);
}

// From a kept lse: one walk.  Its rounding is a factor of 1 + 2^-24 |lse| of every probability, and far from zero the row's sum is lost
// in it altogether, as a token's log-probability is in its difference from a logit that is far off.  So from kKept on (the logits of a model
// in use are well below) the row is walked once more for its sum, in the order of the other calls.
constexpr float kKept = 128.0f;
// Nor does the kept lse say on which side of a border a ratio stands that is within its rounding: 1 itself with a clip of 0, where forward's ratio is exact
// and half of such rows would lose their gradient.  The two log-probabilities are within 10 x 2^-24 (|z / T| + |lse|) of each other, which
// kKept keeps below 2^-12, and either's ratio is off by 4 x 2^-24 and half a rounding of the exponent.
__device__ __forceinline__ bool says_too_little(const PolicyParams &p, const Sample &t, float lse, float z, float logp)
{
    if (!(fabsf(lse) < kKept && fabsf(z) < kKept)) return true;
    const float x = __fsub_rn(logp, t.old), ratio = expf(x), room = ratio * 0x1p-20f * (fabsf(z) + fabsf(lse) + fabsf(x) + 1.0f);
    return t.advantage != 0.0f && (fabsf(ratio - p.low) <= room || fabsf(ratio - p.high) <= room);
}
template <typename T, typename I> __global__ void __launch_bounds__(kMostWalkers, 2) policy_backward_kernel(const __grid_constant__ PolicyParams p)
{
    __shared__ Joined cell[kMostWalkers / 32];
    const unsigned r = blockIdx.x;
    const Row<T> w(static_cast<const T *>(p.logits) + r * p.row_stride, p.vocab, blockDim.x);
    const Sample t = sample_of<T, I>(p, w.row, r, true);
    const float lse = p.lse_in[r];
    const float z = t.z / p.temperature, logp = __fsub_rn(z, lse);
    if (t.there() && says_too_little(p, t, lse, z, logp)) {
        const float unit = kLog2e / p.temperature;
        Running<false> run;
        if (w.edge() >= 0) run.take_one(to_float(w.row[w.edge()]), unit);
        const int own = own_groups(w);
        for (int i = 0; i < own; i += Places<T>::kStep)
            take_step<T>(run, i, own, unit, [&](int k) {
                Group<T> x;
                x.load(w.row + w.parts.head + (long long)(threadIdx.x + (i + k) * w.walkers) * kGroup);
                return x;
            });
        end_row<T, kBackward>(p, r, w, t, run, unit, cell);
        return;
    }
    const float slope = t.there() ? value_of(p, t, logp).slope : 0.0f;
    const float weight = __fdiv_rn(__fmul_rn(t.grad_loss, slope), p.temperature);
    __syncthreads();                                  // every thread has the token's logit: the gradient may be written over it
    put_row<kAhead<T>>(p, gradient_of<T>(p, r), w, t, Softmax<false>{1.0f / p.temperature, -lse, kLog2e, -weight}, weight);
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
    // About fifteen pieces of 16 bytes for each thread of a row, whatever the direction and the number of rows: sums have the same order, and
    // the log-probabilities of a step are those of an earlier call bit for bit.
    int walkers = kFewestWalkers;
    while (walkers < kMostWalkers && size_t(walkers) * 480 <= size_t(p.vocab) * sizeof(T)) walkers *= 2;
    if (mode == kBackward) {
        policy_backward_kernel<T, I><<<rows, walkers, 0, s>>>(p);
        return context_launched(ctx, int(cudaGetLastError()));
    }
    const size_t bytes = size_t(kRound<T>) * walkers * Places<T>::kSize;
    void (*const kernel)(PolicyParams) = mode == kStep ? policy_kernel<T, I, kStep> : policy_kernel<T, I, kForward>;
    constexpr int kMost = kRound<T> * kMostWalkers * Places<T>::kSize;
    const int rc = bytes > 40 * 1024 ? context_shared(ctx, reinterpret_cast<const void *>(kernel), kMost) : OMNI_OK;
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
    p.old = valued ? d->old : nullptr;                // the log-probabilities alone look at none of these
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
    p.kl = valued ? d->kl : 0.0f;
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
