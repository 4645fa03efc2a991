// Distillation loss from a teacher's top logits: forward, backward, both in one pass.
//
// Per row: lse = log sum_v exp(z_v / T) needs all of z before the first gradient value can be
// written, so the gradient is a second walk over the row.  One CTA owns a row; the first walk keeps a
// running maximum and sum per thread (a sum is rescaled only when its maximum moves), the
// second finds the row, which the same CTA read a moment ago, in L2.  HBM sees one read and one write.
#include "context.h"
#include "vector.cuh"

namespace omni {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxThreads = 1024;
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

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Maximum and sum of 2^(x - maximum), joined.  Products and sums are spelled out where the compiler could
// contract them one way in one variant and another way in the next: forward and step give the same bits.
struct Running {
    float m, s;
    __device__ __forceinline__ void join(float om, float os)
    {
        const float nm = fmaxf(m, om);
        if (nm == -INFINITY) { s += os; return; }    // both empty (a NaN sum stays one)
        s = fmaf(s, exp2_fast(m - nm), __fmul_rn(os, exp2_fast(om - nm)));
        m = nm;
    }
};

// Element range of a row in three parts: up to the first 16-byte boundary, whole groups, the rest.
template <typename T> struct Parts {
    int head, groups;
    __device__ __forceinline__ Parts(const T *row, int vocab)
    {
        const int lead = int((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / int(sizeof(T));
        head = lead < vocab ? lead : vocab;
        groups = (vocab - head) / kGroup;
    }
};

template <typename F> __device__ __forceinline__ float block_reduce(float x, float *cell, F f, float neutral)
{
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
    for (int o = 16; o > 0; o /= 2) x = f(x, __shfl_xor_sync(~0u, x, o));
    __syncthreads();
    if (lane == 0) cell[warp] = x;
    __syncthreads();
    x = lane < warps ? cell[lane] : neutral;
    for (int o = 16; o > 0; o /= 2) x = f(x, __shfl_xor_sync(~0u, x, o));
    return x;
}

template <typename T, typename I, int MODE>
__global__ void __launch_bounds__(kMaxThreads) distill_kernel(DistillParams p)
{
    __shared__ float cell[32], cell2[32];
    __shared__ float prob[OMNI_DISTILL_MAX_TOP], hit[OMNI_DISTILL_MAX_TOP];
    __shared__ int place[OMNI_DISTILL_MAX_TOP];
    const unsigned long long r = blockIdx.x;
    const T *row = static_cast<const T *>(p.logits) + r * p.row_stride;
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid % 32, warp = tid / 32;
    const float unit = kLog2e / p.temperature;      // logits to powers of two
    const Parts<T> parts(row, p.vocab);

    // the teacher's entries: place, student's logit there, probability
    float t = -INFINITY;
    if (tid < p.top) {
        const long long i = load_index<I>(p.top_index, r * p.top_stride + tid);
        const bool there = i >= 0 && i < p.vocab;
        place[tid] = there ? int(i) : -1;
        hit[tid] = there ? to_float(row[i]) : 0.0f;
        if (there) t = p.top_logits[r * p.top_stride + tid] / p.temperature;
    }
    auto larger = [](float a, float b) { return fmaxf(a, b); };
    auto plus = [](float a, float b) { return a + b; };
    const float tm = block_reduce(t, cell, larger, -INFINITY);
    const float te = tid < p.top && tm != -INFINITY ? expf(t - tm) : 0.0f;
    const float ts = block_reduce(te, cell, plus, 0.0f);
    const bool target = !(ts == 0.0f);              // NaN counts as a target and shows
    const float my_p = target ? te / ts : 0.0f;
    if (tid < p.top) prob[tid] = my_p;

    float lse2;                                     // lse in powers of two
    if constexpr (MODE != kBackward) {
        Running run{-INFINITY, 0.0f};
        for (int g = tid; g < parts.groups; g += threads) {
            float f[kGroup];
            load_group(row + parts.head + (long long)g * kGroup, f);
            float m = f[0];
#pragma unroll
            for (int e = 1; e < kGroup; ++e) m = fmaxf(m, f[e]);
            m = __fmul_rn(m, unit);
            if (m > run.m) { run.s = __fmul_rn(run.s, exp2_fast(run.m - m)); run.m = m; }
            const float ref = run.m == -INFINITY ? 0.0f : run.m;
#pragma unroll
            for (int e = 0; e < kGroup; ++e) run.s += exp2_fast(fmaf(f[e], unit, -ref));
        }
        const int rest = p.vocab - parts.groups * kGroup;   // head and tail together, < 16 elements
        if (tid < rest) {
            const int v = tid < parts.head ? tid : parts.groups * kGroup + tid;
            const float x = __fmul_rn(to_float(row[v]), unit);
            run.join(x, x == -INFINITY ? 0.0f : exp2_fast(x - x));
        }
        for (int o = 16; o > 0; o /= 2) run.join(__shfl_xor_sync(~0u, run.m, o), __shfl_xor_sync(~0u, run.s, o));
        __syncthreads();
        if (lane == 0) { cell[warp] = run.m; cell2[warp] = run.s; }
        __syncthreads();
        run.m = lane < threads / 32 ? cell[lane] : -INFINITY;
        run.s = lane < threads / 32 ? cell2[lane] : 0.0f;
        for (int o = 16; o > 0; o /= 2) run.join(__shfl_xor_sync(~0u, run.m, o), __shfl_xor_sync(~0u, run.s, o));
        lse2 = run.m + log2f(run.s);
        const float lse = __fmul_rn(lse2, kLn2);
        float term = 0.0f;
        if (tid < p.top && !(my_p == 0.0f)) term = __fmul_rn(my_p, logf(my_p) - hit[tid] / p.temperature + lse);
        const float sum = block_reduce(term, cell, plus, 0.0f);
        if (tid == 0) {
            p.loss[r] = p.temperature * p.temperature * sum;
            p.lse_out[r] = lse;
        }
    } else {
        lse2 = __fmul_rn(p.lse_in[r], kLog2e);
    }

    if constexpr (MODE != kForward) {
        T *out = static_cast<T *>(p.grad) + r * p.grad_stride;
        const float gain = target ? p.grad_loss[r] * p.temperature : 0.0f;
        const float ref = lse2 == -INFINITY ? 0.0f : lse2;
        const bool together = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15) == 0;
        auto value = [&](float z) { return target ? gain * exp2_fast(fmaf(z, unit, -ref)) : 0.0f; };
        if (together) {
            for (int g = tid; g < parts.groups; g += threads) {
                float f[kGroup];
                const long long v = parts.head + (long long)g * kGroup;
                load_group(row + v, f);
#pragma unroll
                for (int e = 0; e < kGroup; ++e) f[e] = value(f[e]);
                store_group(out + v, f);
            }
            const int rest = p.vocab - parts.groups * kGroup;
            if (tid < rest) {
                const int v = tid < parts.head ? tid : parts.groups * kGroup + tid;
                out[v] = from_float<T>(value(to_float(row[v])));
            }
        } else {
            for (int v = tid; v < p.vocab; v += threads) out[v] = from_float<T>(value(to_float(row[v])));
        }
        __syncthreads();
        // the teacher's entries over it; one that names a token again is left to the first
        if (tid < p.top && place[tid] >= 0 && target) {
            float total = 0.0f;
            bool first = true;
            for (int j = 0; j < p.top; ++j)
                if (place[j] == place[tid]) {
                    first = first && j >= tid;
                    total += prob[j];
                }
            if (first) out[place[tid]] = from_float<T>(gain * (exp2_fast(fmaf(hit[tid], unit, -ref)) - total));
        }
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

template <typename T, typename I> int enqueue(omni_ctx *ctx, int mode, const DistillParams &p, unsigned rows, cudaStream_t s)
{
    // a thread per two groups of eight, a warp per 32 entries of the teacher at least
    int threads = 128;
    while (threads < kMaxThreads && threads * 2 * kGroup < p.vocab) threads *= 2;
    while (threads < p.top) threads *= 2;
    if (mode == kForward) distill_kernel<T, I, kForward><<<rows, threads, 0, s>>>(p);
    else if (mode == kBackward) distill_kernel<T, I, kBackward><<<rows, threads, 0, s>>>(p);
    else distill_kernel<T, I, kStep><<<rows, threads, 0, s>>>(p);
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
