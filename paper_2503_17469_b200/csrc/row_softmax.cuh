// A row of logits walked by the threads of a CTA: running maximum and sum, softmax values, gradients in groups of eight.
// For the losses over a vocabulary (distill.cu, policy.cu).
#pragma once
#include <type_traits>

#include "vector.cuh"

namespace omni {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

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
    // Near zero it begins where far begins: a thread that sees nothing but a mask of -1e30 would have the power of two of that product's rounding,
    // an overflow, and infinity times the ratio of 0 to the row's maximum is no number.
    float m = FAR ? -INFINITY : -kFar;
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
    __device__ __forceinline__ static float reference(float m) { return FAR && m == -INFINITY ? 0.0f : -m; }
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
    return {m, warp_sum((FAR && m == -INFINITY) || own == m ? s : __fmul_rn(s, Running<FAR>::ratio(own, m, unit)))};
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

// What every thread of a row's CTA knows.
template <typename T> struct Row {
    const T *row;
    Parts<T> parts;
    int walkers, vocab;
    __device__ __forceinline__ Row(const T *first, int n, int threads) : row(first), parts(first, n), walkers(threads), vocab(n) {}
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

}  // namespace omni
