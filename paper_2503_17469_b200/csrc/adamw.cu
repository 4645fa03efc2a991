// AdamW over many tensors in one launch, on the weighted gradients of K workers, with moments of 32 bits or of 8.
//
// Per element, every operation in float, rounded once, FMA where written so (the states' bits are part of the contract):
//   g = fma(lambda_{K-1}, g_{K-1}, ... fma(lambda_0, g_0, 0));  m = fma(b1, m, c1 g);  v = fma(c2 g, g, b2 v)
//   theta = fma(-rate, m / fma(sqrt(v), spread, eps), keep theta)
// with c = 1 - b, rate = lr / (1 - b1^t), spread = (1 - b2^t)^(-1/2), keep = 1 - lr decay.
//
// Moments of 8 bits: a float's top twelve bits (sign, exponent, three of the fraction), counted down from the largest of the
// 256 elements of its block, which is kept beside the codes: seven bits below a sign for m (16 octaves), eight for v (32 octaves; what is not zero
// stays at least the lowest code, so that no m is divided by a root that was lost).  Decoding is a shift and an addition,
// no scale is multiplied.  The bits below are rounded by random ones: a decay of v by a thousandth a step is far below
// half of a code's step of an eighth, and would never happen with the nearest code.
//
// A table of the tensors in device memory names the owner of each 1024 elements: one launch, whatever their number; a warp has a block, a lane
// eight elements.  Every load of a lane stands before whatever waits for one (a widening between them cost a quarter of the time).
// What bounds it: with float moments the memory (140 million elements, bfloat16 gradients and copy, 570 us, 6.8 TB/s; floor 597 at the copy
// rate); with 8 bits the whole-number units, at 70 % (73 million elements 213 us, floor 180; four workers' gradients 270, floor 248), which is
// why codes are packed four at a time and shifts are written as products.  Their values as floats take 113 us more (floor 112).
// Tried for 8 bits: CTAs that stay with a ring of asynchronous copies 274-480 us; two units a CTA 272; eight or ten CTAs an SM 223 and 220
// where nine take 213.
#include "context.h"
#include "vector.cuh"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

namespace omni {
namespace {

constexpr int kThreads = 128;
constexpr int kBlock = OMNI_ADAMW_BLOCK;              // elements with one offset: a warp's, eight a lane
constexpr int kUnit = kThreads * kGroup;              // elements a CTA has at a time
static_assert(kBlock == 32 * kGroup, "a warp holds a block");

// A tensor in the record, followed by those of all tensors, the K gradient pointers of each, and the owner of each unit.
struct Entry {
    float *param;
    __nv_bfloat16 *copy;
    void *m, *v;
    uint32_t *tops;                                   // of a block: that of m in the low half, that of v in the high half
    unsigned long long n;
    double decay;
    unsigned first_unit;
    int wide;                                         // every pointer allows accesses of eight elements
};
struct Header {
    unsigned long long magic, bytes;
    int tensors, K, grad_dtype, bits;
    unsigned units;
    int pad[7];
};
static_assert(sizeof(Entry) == 64 && sizeof(Header) == 64, "the record's layout");
constexpr unsigned long long kMagic = 0x6f6d6e695f616477ull;

struct Layout {
    unsigned long long entries, grads, owners, bytes;
    __host__ __device__ Layout(int tensors, int K, unsigned units)
    {
        entries = sizeof(Header);
        grads = entries + (unsigned long long)tensors * sizeof(Entry);
        owners = grads + (unsigned long long)tensors * K * sizeof(void *);
        bytes = (owners + (unsigned long long)units * 4 + 15) / 16 * 16;
    }
};

struct AdamParams {
    const Entry *entries;
    const void *const *grads;
    const unsigned *owners;
    const long long *clock;                           // the step's number on the device, or NULL
    double lr, beta1, beta2;
    float b1, b2, c1, c2, eps, rate, spread;
    unsigned step;
    int K;
    float lambda[OMNI_MAX_K];
};

// Eight elements, those before the end, one by one.
template <typename T> __device__ __forceinline__ void load8(const T *p, int count, float *f)
{
#pragma unroll
    for (int i = 0; i < kGroup; ++i) f[i] = i < count ? to_float(p[i]) : 0.0f;
}
// Eight elements, or those of them before the end one by one.
template <typename T> __device__ __forceinline__ void store8(T *p, bool wide, int count, const float *f)
{
    if (wide && count == kGroup) {
        store_group(p, f);
        return;
    }
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
        if (i < count) p[i] = from_float<T>(f[i]);
}
__device__ __forceinline__ uint2 load_codes(const unsigned char *p, bool wide, int count)
{
    if (wide && count == kGroup) return *reinterpret_cast<const uint2 *>(p);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
        if (i < count) w[i / 4] |= uint32_t(p[i]) << (8 * (i % 4));
    return {w[0], w[1]};
}
__device__ __forceinline__ void store_codes(unsigned char *p, bool wide, int count, uint2 c)
{
    if (wide && count == kGroup) {
        *reinterpret_cast<uint2 *>(p) = c;
        return;
    }
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
        if (i < count) p[i] = (unsigned char)((i < 4 ? c.x : c.y) >> (8 * (i % 4)));
}

// What four codes in a word stand for; MOST: 127 for the signed codes of m, 255 for those of v.  A byte is put to bits 16 to 23, and one
// multiply-add shifts it and adds the block's offset: the units of whole numbers are the busiest part of this kernel.
template <int MOST> __device__ __forceinline__ void decode4(uint32_t word, uint32_t below, float *f)
{
    const uint32_t sizes = MOST == 127 ? word & 0x7f7f7f7fu : word;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = __byte_perm(sizes, 0u, 0x4044 | i << 8), bits = c ? c * 16u + below : 0u;
        f[i] = __uint_as_float(MOST == 127 ? bits | (__byte_perm(word, 0u, 0x0444 | i << 12) & 0x80000000u) : bits);
    }
}
template <int MOST> __device__ __forceinline__ void decode8(uint2 c, int top, float *f)
{
    const uint32_t below = uint32_t(top - MOST) << 20;
    decode4<MOST>(c.x, below, f);
    decode4<MOST>(c.y, below, f + 4);
}
// The float's bits less the sign, with 16 random ones added at bit 4: from bit 20 on its rounded top.  A NaN may come out one too high.
__device__ __forceinline__ uint32_t rounded(uint32_t bits, uint32_t random) { return random * 16u + bits; }
// The top bytes of four words as one.
__device__ __forceinline__ uint32_t join4(const uint32_t *c)
{
    return __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
}
// Codes of four elements from their rounded bits r, the largest top of the block, and the elements themselves (for the signs).
template <int MOST> __device__ __forceinline__ uint32_t encode4(const uint32_t *r, int top, const float *x)
{
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c[i] = uint32_t(__viaddmax_s32(int(r[i]), (MOST - top) * (1 << 20), MOST == 255 ? 1 << 20 : 0));
        if (top < MOST) c[i] = r[i] >> 20 ? c[i] : 0u;          // zero stays zero
        else if (MOST == 255) c[i] = min(c[i], r[i]);           // here as well: r is below one step then
        c[i] *= 16u;                                            // the code is the top byte
    }
    const uint32_t word = join4(c);
    const uint32_t signs = __byte_perm(__byte_perm(__float_as_uint(x[0]), __float_as_uint(x[1]), 0x0073),
                                       __byte_perm(__float_as_uint(x[2]), __float_as_uint(x[3]), 0x0073), 0x5410);
    return MOST == 255 ? word : word | (word + 0x7f7f7f7fu & 0x80808080u & signs);           // a code of 0 has no sign
}
// Root and quotient of m / fma(sqrt(v), spread, eps): short forms, within 2^-22 each, which a step of the usual size loses in theta's own rounding.
// Rounded correctly they take a small model's step from 6.0 to 6.5 us, 140 million with float moments from 570 to 574 and 73 million with 8
// bits from 205 to 228.  The short forms count numbers below float's normal range as 0, which changes the divisor by less than
// 2^-63 spread; with an eps between 2^-41 spread and 2^100 that is below 2^-22 of it, and no inverse leaves float's range.  Spread is largest in the
// first step, so an eps of 1e-8 has the short forms up to a beta2 of 1 - 2^-28.  Any other eps has the correct ones.
bool short_forms(double eps, double beta2) { return eps >= 0x1p-41 / std::sqrt(1.0 - beta2) && eps <= 0x1p100; }
template <bool SHORT> __device__ __forceinline__ float root(float x)
{
    if (!SHORT) return __fsqrt_rn(x);
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float inverse(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool SHORT> __device__ __forceinline__ float2 quotient(float2 x, float2 y)
{
    if (!SHORT) return make_float2(__fdiv_rn(x.x, y.x), __fdiv_rn(x.y, y.y));
    return mul2(x, {inverse(y.x), inverse(y.y)});
}

// 32 bits of an element's own, by multiplications and shifts of its number, its tensor's and the step's.  The multipliers are published constants of
// integer hashing: the prime next to 2^32 over the golden ratio and two others for the start, and the first of the two rounds (16, 0x7FEB352D, 15) of C. Wellons'
// search for mixers with little bias; one round is enough for bits that round.
constexpr uint32_t kStride = 0x9E3779B1u;
__device__ __forceinline__ uint32_t scramble(uint32_t x)
{
    x = (x ^ x >> 16) * 0x7FEB352Du;
    return x ^ x >> 15;
}

// The step's number and what follows from it; with a clock on the device, by one thread of the CTA.
struct Scales {
    float rate, spread;
    uint32_t step;
};
__device__ __forceinline__ Scales scales_of(const AdamParams &p)
{
    if (!p.clock) return {p.rate, p.spread, p.step};
    __shared__ Scales now;
    if (threadIdx.x == 0) {
        const long long t = *p.clock;
        now = {float(p.lr / (1.0 - pow(p.beta1, double(t)))), float(1.0 / sqrt(1.0 - pow(p.beta2, double(t)))), uint32_t(t)};
    }
    __syncthreads();
    return now;
}

// Eight gradients as loaded: what waits for a load stands behind all of them.
template <typename G> struct Raw;
template <> struct Raw<float> {
    float f[kGroup];
    __device__ __forceinline__ void load(const float *p) { load_group(p, f); }
    __device__ __forceinline__ void get(float *x) const
    {
#pragma unroll
        for (int i = 0; i < kGroup; ++i) x[i] = f[i];
    }
};
template <> struct Raw<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { u = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float *x) const { widen(u, x); }
};

// A lane's place in a tensor.
struct Place {
    unsigned tensor;
    unsigned long long at;
    int count;                                        // of its eight elements before the tensor's end
    bool block, whole;                                // the warp's block begins before the end; accesses of eight are allowed
    __device__ __forceinline__ Place(const AdamParams &p, unsigned unit, const Entry *&e) : tensor(p.owners[unit])
    {
        e = p.entries + tensor;
        at = (unsigned long long)(unit - e->first_unit) * kUnit + threadIdx.x * kGroup;
        count = at >= e->n ? 0 : e->n - at < kGroup ? int(e->n - at) : kGroup;
        block = at - threadIdx.x % 32 * kGroup < e->n;
        whole = e->wide && count == kGroup;
    }
};

// The weighted gradient, ascending k, loads of four or two workers at a time.
template <typename G> constexpr int kWorkers = sizeof(G) == 2 ? 4 : 2;
template <typename G> __device__ __forceinline__ void aggregate(const AdamParams &p, const Place &x, const Raw<G> &first, float *g)
{
    const void *const *const grads = p.grads + (unsigned long long)x.tensor * p.K;
    float f[kGroup];
    first.get(f);
#pragma unroll
    for (int i = 0; i < kGroup; ++i) g[i] = __fmaf_rn(p.lambda[0], f[i], 0.0f);
    for (int k = 1; k < p.K; k += kWorkers<G>) {
        Raw<G> raw[kWorkers<G>];
#pragma unroll
        for (int j = 0; j < kWorkers<G>; ++j)
            if (k + j < p.K) raw[j].load(static_cast<const G *>(grads[k + j]) + x.at);
#pragma unroll
        for (int j = 0; j < kWorkers<G>; ++j) {
            if (k + j >= p.K) break;
            raw[j].get(f);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) g[i] = __fmaf_rn(p.lambda[k + j], f[i], g[i]);
        }
    }
}
// The same element by element.
template <typename G> __device__ __forceinline__ void aggregate_some(const AdamParams &p, const Place &x, float *g)
{
    for (int k = 0; k < p.K; ++k) {
        float f[kGroup];
        load8(static_cast<const G *>(p.grads[(unsigned long long)x.tensor * p.K + k]) + x.at, x.count, f);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) g[i] = __fmaf_rn(p.lambda[k], f[i], k ? g[i] : 0.0f);
    }
}

template <typename G, int BITS, bool SHORT> __global__ void __launch_bounds__(kThreads, BITS == 8 ? 9 : 7) adamw_kernel(const __grid_constant__ AdamParams p)
{
    const Entry *entry;
    const Place x(p, blockIdx.x, entry);
    const Entry &e = *entry;
    float theta[kGroup], m[kGroup], v[kGroup], g[kGroup];
    float *const fm = static_cast<float *>(e.m) + x.at, *const fv = static_cast<float *>(e.v) + x.at;
    unsigned char *const cm = static_cast<unsigned char *>(e.m) + x.at, *const cv = static_cast<unsigned char *>(e.v) + x.at;
    uint2 codes_m = {0, 0}, codes_v = {0, 0};
    uint32_t tops = 0;
    Raw<G> first;
    if (x.whole) {
        first.load(static_cast<const G *>(p.grads[(unsigned long long)x.tensor * p.K]) + x.at);
        load_group(e.param + x.at, theta);
        if constexpr (BITS == 32) {
            load_group(fm, m);
            load_group(fv, v);
        } else {
            codes_m = *reinterpret_cast<const uint2 *>(cm);
            codes_v = *reinterpret_cast<const uint2 *>(cv);
            tops = e.tops[x.at / kBlock];
        }
    }
    const Scales now = scales_of(p);
    if (!x.block) return;
    if (x.whole) {
        aggregate(p, x, first, g);
    } else {
        load8(e.param + x.at, x.count, theta);
        if constexpr (BITS == 32) {
            load8(fm, x.count, m);
            load8(fv, x.count, v);
        } else {
            codes_m = load_codes(cm, false, x.count);
            codes_v = load_codes(cv, false, x.count);
            tops = e.tops[x.at / kBlock];
        }
        aggregate_some<G>(p, x, g);
    }
    if constexpr (BITS == 8) {
        decode8<127>(codes_m, int(tops & 0xffffu), m);
        decode8<255>(codes_v, int(tops >> 16), v);
    }
    const float keep = float(1.0 - p.lr * e.decay);
#pragma unroll
    for (int i = 0; i < kGroup; i += 2) {
        const float2 d = {g[i], g[i + 1]}, t = {theta[i], theta[i + 1]};
        const float2 m1 = fma2({p.b1, p.b1}, {m[i], m[i + 1]}, mul2({p.c1, p.c1}, d));
        const float2 v1 = fma2(mul2({p.c2, p.c2}, d), d, mul2({p.b2, p.b2}, {v[i], v[i + 1]}));
        const float2 below = fma2({root<SHORT>(v1.x), root<SHORT>(v1.y)}, {now.spread, now.spread}, {p.eps, p.eps});
        const float2 t1 = fma2({-now.rate, -now.rate}, quotient<SHORT>(m1, below), mul2({keep, keep}, t));
        m[i] = m1.x; m[i + 1] = m1.y;
        v[i] = v1.x; v[i + 1] = v1.y;
        theta[i] = t1.x; theta[i + 1] = t1.y;
    }
    store8(e.param + x.at, x.whole, x.count, theta);
    if (e.copy) store8(e.copy + x.at, x.whole, x.count, theta);
    if constexpr (BITS == 32) {
        store8(fm, x.whole, x.count, m);
        store8(fv, x.whole, x.count, v);
    } else {
        const uint32_t start = now.step * 0x85EBCA77u + x.tensor * 0xC2B2AE3Du + uint32_t(x.at) * kStride;
        // What stands behind the end was loaded as zeros: it is zero still, and its codes are not stored.
        uint32_t rm[kGroup], rv[kGroup], most_m = 0, most_v = 0;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            const uint32_t random = scramble(start + i * kStride);
            rm[i] = rounded(__float_as_uint(m[i]) & 0x7fffffffu, random & 0xffffu);
            rv[i] = rounded(__float_as_uint(v[i]), random >> 16);        // not negative
            most_m = max(most_m, rm[i]);
            most_v = max(most_v, rv[i]);
        }
        most_m = __reduce_max_sync(~0u, most_m);
        most_v = __reduce_max_sync(~0u, most_v);
        if (max(most_m, most_v) >> 31) {
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                rm[i] = min(rm[i], 0x7fffffffu);
                rv[i] = min(rv[i], 0x7fffffffu);
            }
            most_m = min(most_m, 0x7fffffffu);
            most_v = min(most_v, 0x7fffffffu);
        }
        most_m >>= 20;
        most_v >>= 20;
        store_codes(cm, x.whole, x.count, {encode4<127>(rm, int(most_m), m), encode4<127>(rm + 4, int(most_m), m + 4)});
        store_codes(cv, x.whole, x.count, {encode4<255>(rv, int(most_v), v), encode4<255>(rv + 4, int(most_v), v + 4)});
        if (threadIdx.x % 32 == 0) e.tops[x.at / kBlock] = most_m | most_v << 16;
    }
}

// What the codes of some tensors stand for.
constexpr int kPerLaunch = 192;
struct MomentParams {
    const Entry *entries;
    const unsigned *owners;
    unsigned first_unit;
    int first;
    float *m[kPerLaunch], *v[kPerLaunch];
};
__global__ void __launch_bounds__(kThreads) adamw_moments_kernel(const __grid_constant__ MomentParams p)
{
    const unsigned unit = p.first_unit + blockIdx.x, tensor = p.owners[unit];
    const Entry &e = p.entries[tensor];
    const unsigned long long at = (unsigned long long)(unit - e.first_unit) * kUnit + threadIdx.x * kGroup;
    if (at >= e.n) return;
    const int count = e.n - at < kGroup ? int(e.n - at) : kGroup;
    float *const m = p.m[tensor - p.first] + at, *const v = p.v[tensor - p.first] + at;
    const uint32_t tops = e.tops[at / kBlock];
    float f[kGroup];
    decode8<127>(load_codes(static_cast<const unsigned char *>(e.m) + at, e.wide, count), int(tops & 0xffffu), f);
    store8(m, (reinterpret_cast<uintptr_t>(m) & 15) == 0, count, f);
    decode8<255>(load_codes(static_cast<const unsigned char *>(e.v) + at, e.wide, count), int(tops >> 16), f);
    store8(v, (reinterpret_cast<uintptr_t>(v) & 15) == 0, count, f);
}

// ---- host ---------------------------------------------------------------------------------------

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_tensors(const omni_adamw_tensor *t, int32_t count, int32_t K, int32_t grad_dtype, int32_t bits, unsigned *units)
{
    if (K < 1 || K > OMNI_MAX_K) return OMNI_ERR_BAD_K;
    if (count < 0 || (grad_dtype != OMNI_F32 && grad_dtype != OMNI_BF16) || (bits != 32 && bits != 8)) return OMNI_ERR_BAD_CONFIG;
    if (count > 0 && !t) return OMNI_ERR_NULL;
    const size_t grad = grad_dtype == OMNI_BF16 ? 2 : 4;
    uint64_t all = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (!(t[i].weight_decay - t[i].weight_decay == 0.0)) return OMNI_ERR_BAD_CONFIG;
        if (t[i].n == 0) continue;
        if (t[i].n >= (1ull << 42)) return OMNI_ERR_TOO_LARGE;
        if (!t[i].param || !t[i].grads || !t[i].m || !t[i].v || (bits == 8 && !t[i].tops)) return OMNI_ERR_NULL;
        if (!aligned(t[i].param, 4) || !aligned(t[i].param_lp, 2) || (bits == 32 && (!aligned(t[i].m, 4) || !aligned(t[i].v, 4))) ||
            (bits == 8 && !aligned(t[i].tops, 4)))
            return OMNI_ERR_ALIGN;
        for (int k = 0; k < K; ++k) {
            if (!t[i].grads[k]) return OMNI_ERR_NULL;
            if (!aligned(t[i].grads[k], grad)) return OMNI_ERR_ALIGN;
        }
        all += (t[i].n + kUnit - 1) / kUnit;
        if (all >= (1ull << 31)) return OMNI_ERR_TOO_LARGE;
    }
    *units = unsigned(all);
    return OMNI_OK;
}

bool all_wide(const omni_adamw_tensor &t, int K, int bits)
{
    const size_t state = bits == 8 ? 8 : 16;
    bool wide = aligned(t.param, 16) && aligned(t.param_lp, 16) && aligned(t.m, state) && aligned(t.v, state);
    for (int k = 0; k < K; ++k) wide = wide && aligned(t.grads[k], 16);
    return wide;
}

// Whether what a step writes lies apart from all else that it writes or reads: a tensor that stands in the list twice would be updated
// twice at once, a gradient that is another tensor's parameter read before or after its update.
int check_apart(const omni_adamw_tensor *t, int32_t count, int32_t K, int32_t grad_dtype, int32_t bits)
{
    struct Range {
        uintptr_t from, to;
        bool written;
        bool operator<(const Range &other) const { return from < other.from; }
    };
    try {
        std::vector<Range> ranges;
        ranges.reserve(size_t(count) * (5 + size_t(K)));
        const auto add = [&](const void *p, uint64_t bytes, bool written) {
            if (p) ranges.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
        };
        for (int32_t i = 0; i < count; ++i) {
            if (t[i].n == 0) continue;
            const uint64_t n = t[i].n, state = bits == 8 ? n : 4 * n;
            add(t[i].param, 4 * n, true);
            add(t[i].param_lp, 2 * n, true);
            add(t[i].m, state, true);
            add(t[i].v, state, true);
            if (bits == 8) add(t[i].tops, (n + kBlock - 1) / kBlock * 4, true);
            for (int k = 0; k < K; ++k) add(t[i].grads[k], (grad_dtype == OMNI_BF16 ? 2 : 4) * n, false);
        }
        std::sort(ranges.begin(), ranges.end());
        uintptr_t written = 0, read = 0;              // where those before end
        for (const Range &r : ranges) {
            if (r.from < written || (r.written && r.from < read)) return OMNI_ERR_BAD_CONFIG;
            uintptr_t &last = r.written ? written : read;
            if (r.to > last) last = r.to;
        }
        return OMNI_OK;
    } catch (const std::bad_alloc &) {
        return OMNI_ERR_NO_MEMORY;
    }
}

// The header of a record that omni_adamw_plan wrote, or NULL.
const Header *header_of(const void *record)
{
    const Header *h = static_cast<const Header *>(record);
    return h->magic == kMagic && h->bytes == Layout(h->tensors, h->K, h->units).bytes ? h : nullptr;
}

template <typename G, int BITS> void launch(const AdamParams &p, unsigned units, cudaStream_t s)
{
    if (short_forms(p.eps, p.beta2)) adamw_kernel<G, BITS, true><<<units, kThreads, 0, s>>>(p);
    else adamw_kernel<G, BITS, false><<<units, kThreads, 0, s>>>(p);
}
template <typename G> void launch(const AdamParams &p, int bits, unsigned units, cudaStream_t s)
{
    if (bits == 8) launch<G, 8>(p, units, s);
    else launch<G, 32>(p, units, s);
}

}  // namespace
}  // namespace omni

using namespace omni;

extern "C" {

int omni_adamw_plan_bytes(const omni_adamw_tensor *tensors, int32_t count, int32_t K, int32_t grad_dtype, int32_t bits, uint64_t *bytes)
{
    if (!bytes) return OMNI_ERR_NULL;
    unsigned units = 0;
    const int rc = check_tensors(tensors, count, K, grad_dtype, bits, &units);
    if (rc == OMNI_OK) *bytes = Layout(count, K, units).bytes;
    return rc;
}

int omni_adamw_plan(const omni_adamw_tensor *tensors, int32_t count, int32_t K, int32_t grad_dtype, int32_t bits, void *record, uint64_t bytes)
{
    if (!record) return OMNI_ERR_NULL;
    if (!aligned(record, 8)) return OMNI_ERR_ALIGN;
    unsigned units = 0;
    int rc = check_tensors(tensors, count, K, grad_dtype, bits, &units);
    if (rc == OMNI_OK) rc = check_apart(tensors, count, K, grad_dtype, bits);
    if (rc != OMNI_OK) return rc;
    const Layout at(count, K, units);
    if (bytes < at.bytes) return OMNI_ERR_TOO_LARGE;
    char *const base = static_cast<char *>(record);
    std::memset(base, 0, at.bytes);
    Header *const h = reinterpret_cast<Header *>(base);
    *h = {kMagic, at.bytes, count, K, grad_dtype, bits, units, {}};
    Entry *const entries = reinterpret_cast<Entry *>(base + at.entries);
    const void **const grads = reinterpret_cast<const void **>(base + at.grads);
    unsigned *const owners = reinterpret_cast<unsigned *>(base + at.owners);
    unsigned unit = 0;
    for (int32_t i = 0; i < count; ++i) {
        const omni_adamw_tensor &t = tensors[i];
        entries[i] = {t.param, static_cast<__nv_bfloat16 *>(t.param_lp), t.m, t.v, static_cast<uint32_t *>(t.tops), t.n, t.weight_decay, unit,
                      t.n > 0 && all_wide(t, K, bits)};
        for (int k = 0; k < K && t.n > 0; ++k) grads[uint64_t(i) * K + k] = t.grads[k];
        for (uint64_t j = 0; j < t.n; j += kUnit) owners[unit++] = unsigned(i);
    }
    return OMNI_OK;
}

int omni_adamw_step(omni_ctx *ctx, const void *record, const void *record_dev, const int32_t *b, double lr, double beta1, double beta2, float eps,
                    int64_t step, const int64_t *clock_dev, void *stream)
{
    if (!ctx || !record || !record_dev || !b) return OMNI_ERR_NULL;
    if (!aligned(record, 8) || !aligned(record_dev, 16) || !aligned(clock_dev, 8)) return OMNI_ERR_ALIGN;
    const Header *const h = header_of(record);
    if (!h || !(lr - lr == 0.0) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0f) || eps - eps != 0.0f ||
        (!clock_dev && step < 1))
        return OMNI_ERR_BAD_CONFIG;
    double sum = 0.0;
    for (int k = 0; k < h->K; ++k) {
        if (b[k] < 1) return OMNI_ERR_BAD_BATCH;
        sum += b[k];
    }
    ContextDevice dev;
    const int rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK || h->units == 0) return rc;
    const Layout at(h->tensors, h->K, h->units);
    const char *const base = static_cast<const char *>(record_dev);
    AdamParams p;
    p.entries = reinterpret_cast<const Entry *>(base + at.entries);
    p.grads = reinterpret_cast<const void *const *>(base + at.grads);
    p.owners = reinterpret_cast<const unsigned *>(base + at.owners);
    p.clock = reinterpret_cast<const long long *>(clock_dev);
    p.lr = lr;
    p.beta1 = beta1;
    p.beta2 = beta2;
    p.b1 = float(beta1);
    p.b2 = float(beta2);
    p.c1 = float(1.0 - beta1);
    p.c2 = float(1.0 - beta2);
    p.eps = eps;
    p.rate = clock_dev ? 0.0f : float(lr / (1.0 - std::pow(beta1, double(step))));
    p.spread = clock_dev ? 0.0f : float(1.0 / std::sqrt(1.0 - std::pow(beta2, double(step))));
    p.step = unsigned(uint64_t(step));
    p.K = h->K;
    for (int k = 0; k < h->K; ++k) p.lambda[k] = float(b[k] / sum);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (h->grad_dtype == OMNI_BF16) launch<__nv_bfloat16>(p, h->bits, h->units, s);
    else launch<float>(p, h->bits, h->units, s);
    return context_launched(ctx, int(cudaGetLastError()));
}

int omni_adamw_moments(omni_ctx *ctx, const void *record, const void *record_dev, float *const *m, float *const *v, void *stream)
{
    if (!ctx || !record || !record_dev) return OMNI_ERR_NULL;
    if (!aligned(record, 8) || !aligned(record_dev, 16)) return OMNI_ERR_ALIGN;
    const Header *const h = header_of(record);
    if (!h || h->bits != 8) return OMNI_ERR_BAD_CONFIG;
    if (h->tensors > 0 && (!m || !v)) return OMNI_ERR_NULL;
    const Layout at(h->tensors, h->K, h->units);
    const Entry *const entries = reinterpret_cast<const Entry *>(static_cast<const char *>(record) + at.entries);
    for (int i = 0; i < h->tensors; ++i) {
        if (entries[i].n == 0) continue;
        if (!m[i] || !v[i]) return OMNI_ERR_NULL;
        if (!aligned(m[i], 4) || !aligned(v[i], 4)) return OMNI_ERR_ALIGN;
    }
    ContextDevice dev;
    int rc = context_bind(ctx, &dev);
    const char *const base = static_cast<const char *>(record_dev);
    MomentParams p;
    p.entries = reinterpret_cast<const Entry *>(base + at.entries);
    p.owners = reinterpret_cast<const unsigned *>(base + at.owners);
    for (int i = 0; rc == OMNI_OK && i < h->tensors; i += kPerLaunch) {
        const int last = i + kPerLaunch < h->tensors ? i + kPerLaunch : h->tensors;
        p.first = i;
        p.first_unit = entries[i].first_unit;
        const unsigned units = (last < h->tensors ? entries[last].first_unit : h->units) - p.first_unit;
        if (units == 0) continue;
        for (int j = i; j < last; ++j) {
            p.m[j - i] = m[j];
            p.v[j - i] = v[j];
        }
        adamw_moments_kernel<<<units, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
        rc = context_launched(ctx, int(cudaGetLastError()));
    }
    return rc;
}

}  // extern "C"
