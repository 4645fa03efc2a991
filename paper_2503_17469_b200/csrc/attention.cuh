// What the attention kernels share: shapes, lengths, loading of operand tiles.
#pragma once
#include <climits>

#include "tensor_core.cuh"
#include "vector.cuh"

namespace omni {

constexpr int kRows = 128;                    // rows of an MMA tile
constexpr float kAttnLog2e = 1.4426950408889634f;
constexpr float kAttnLn2 = 0.6931471805599453f;

struct AttnShape {
    int batch, heads, kv_heads, dim, q_len, kv_len, causal;
    float scale;
    const int *q_lengths, *kv_lengths;        // device, per sequence, or null
};

struct Lengths { int q, kv, shift; };         // query i sees keys j <= i + shift (causal)

__device__ __forceinline__ Lengths lengths_of(const AttnShape &s, int b)
{
    Lengths l;
    l.q = s.q_lengths ? min(max(s.q_lengths[b], 0), s.q_len) : s.q_len;
    l.kv = s.kv_lengths ? min(max(s.kv_lengths[b], 0), s.kv_len) : s.kv_len;
    l.shift = l.kv - l.q;
    return l;
}

// Which tile of rows of which head and sequence a block has.  Tiles are the slowest index, so that the
// longest ones of a causal mask (tile 0 here) of all heads come first and the short ones fill the end.
struct Place { int tile, head, batch; };
__device__ __forceinline__ Place place_of(int block, int heads, int batch)
{
    const int per = heads * batch, rest = block % per;
    return {block / per, rest % heads, rest / heads};
}

struct OutView { __nv_bfloat16 *data; long long batch, row, head; };

// 128 x DP tile as blocks of 64 columns, each 128 rows of 128 bytes.
template <int DP>
__device__ __forceinline__ void load_tile(unsigned char *dst, const CUtensorMap *map, int head, int row, int batch,
                                          unsigned long long *bar)
{
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) tensor_load(dst + c * kRows * 128, map, c * 64, head, row, batch, bar);
}

// Zeroes rows [from, to) of a tile, by one warp; the MMA that reads it next sees the zeros.
template <int DP> __device__ __forceinline__ void zero_rows(unsigned char *tile, int from, int to)
{
    const int lane = threadIdx.x % 32;
    for (int c = 0; c < DP / 64; ++c)
        for (int i = from * 8 + lane; i < to * 8; i += 32)
            *reinterpret_cast<uint4 *>(tile + c * kRows * 128 + i * 16) = make_uint4(0, 0, 0, 0);
    fence_async_proxy();
    __syncwarp();
}

// What the loading warp of a block keeps: where waits are recorded, and a barrier of its own.
struct Loader {
    unsigned long long *own;
    unsigned parity;
    volatile int *give_up;
    unsigned *status;

    __device__ __forceinline__ bool wait(unsigned long long *bar, unsigned p) { return warp_wait(bar, p, give_up, status); }

    // A 128 x DP tile into `dst`; `bar` gets this phase's one arrival and the bytes, `more` further bytes are on their way to
    // it.  Rows from `valid` on lie behind the sequence's length and rows before `from` are queries that see no key; the caller
    // may have left anything in both, and 0 x NaN would reach the sums: such a tile is waited for here, its rows outside
    // [from, valid) are zeroed, and it is handed over then.
    template <int DP>
    __device__ __forceinline__ bool tile(unsigned char *dst, const CUtensorMap *map, int head, int row, int batch,
                                         unsigned long long *bar, int valid, unsigned more = 0, int from = 0)
    {
        const bool first = threadIdx.x % 32 == 0;
        constexpr unsigned bytes = kRows * DP * 2;
        if (valid >= kRows && from <= 0) {
            if (first) {
                mbar_expect_tx(bar, bytes + more);
                load_tile<DP>(dst, map, head, row, batch, bar);
            }
            return true;
        }
        if (first) {
            mbar_expect_tx(own, bytes);
            load_tile<DP>(dst, map, head, row, batch, own);
        }
        __syncwarp();
        if (!wait(own, parity)) {
            mbar_wait(own, parity);          // the block may not end with the copy in flight
            return false;
        }
        parity ^= 1;
        zero_rows<DP>(dst, 0, from);
        zero_rows<DP>(dst, valid, kRows);
        if (first) {
            if (more) mbar_expect_tx(bar, more);
            else mbar_arrive(bar);
        }
        __syncwarp();
        return true;
    }
};

// d[128 x 128] = A B^T, both tiles with the contraction along their rows' DP columns.
template <int DP>
__device__ __forceinline__ void mma_along(unsigned d, unsigned a, unsigned b)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const unsigned at = (k / 4) * kRows * 128 + (k % 4) * 32;
        mma_ss(d, tile_desc(a + at, 1024, 16), tile_desc(b + at, 1024, 16), mma_kind(kRows, false), k > 0);
    }
}
// d[128 x DP] (+)= P B, P [128 x K] bfloat16 in tensor memory, B a tile of whose rows K are contracted over.
// P stands in stretches of RUN values, each at the start of the RUN columns whose scores it came from.
template <int DP, int K, int RUN>
__device__ __forceinline__ void mma_tmem_across(unsigned d, unsigned p, unsigned b, bool add)
{
#pragma unroll
    for (int k = 0; k < K / 16; ++k)
        mma_ts(d, p + k * 16 / RUN * RUN + k * 16 % RUN / 2, tile_desc(b + k * 2048, 1024, kRows * 128), mma_kind(DP, true), add || k > 0);
}

// Two floats to bfloat16, the first in the low half, in one instruction.
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// One row of `cols` float accumulators in tensor memory, times `gain`, to bfloat16 in global memory.
template <int DP>
__device__ __forceinline__ void store_row(unsigned tmem, float gain, __nv_bfloat16 *dst, int dim, bool write)
{
    constexpr int kAt = DP < 32 ? DP : 32;     // columns at a time
#pragma unroll
    for (int c = 0; c < DP / kAt; ++c) {
        uint32_t r[kAt];
        tmem_load(r, tmem + c * kAt);
#pragma unroll
        for (int g = 0; g < kAt / 8; ++g) {
            const int col = c * kAt + g * 8;
            if (!write || col >= dim) continue;
            uint4 o;
            o.x = pack2(gain * __uint_as_float(r[g * 8 + 0]), gain * __uint_as_float(r[g * 8 + 1]));
            o.y = pack2(gain * __uint_as_float(r[g * 8 + 2]), gain * __uint_as_float(r[g * 8 + 3]));
            o.z = pack2(gain * __uint_as_float(r[g * 8 + 4]), gain * __uint_as_float(r[g * 8 + 5]));
            o.w = pack2(gain * __uint_as_float(r[g * 8 + 6]), gain * __uint_as_float(r[g * 8 + 7]));
            *reinterpret_cast<uint4 *>(dst + col) = o;
        }
    }
}
// The same as floats, for a part of a sum.
template <int DP> __device__ __forceinline__ void store_row(unsigned tmem, float gain, float *dst, int dim, bool write)
{
    constexpr int kAt = DP < 32 ? DP : 32;
#pragma unroll
    for (int c = 0; c < DP / kAt; ++c) {
        uint32_t r[kAt];
        tmem_load(r, tmem + c * kAt);
#pragma unroll
        for (int g = 0; g < kAt / 8; ++g) {
            if (!write || c * kAt + g * 8 >= dim) continue;
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = gain * __uint_as_float(r[g * 8 + e]);
            store_group(dst + c * kAt + g * 8, f);
        }
    }
}
__device__ __forceinline__ void store_zeros(__nv_bfloat16 *dst, int dim)
{
    for (int c = 0; c < dim; c += 8) *reinterpret_cast<uint4 *>(dst + c) = make_uint4(0, 0, 0, 0);
}

// `rows` rows from `row` on set to zero by the whole block.
__device__ __forceinline__ void zero_tile(const OutView &o, int batch, int head, int row, int rows, int dim)
{
    const int groups = dim / 8;
    for (int i = threadIdx.x; i < rows * groups; i += blockDim.x)
        *reinterpret_cast<uint4 *>(o.data + batch * o.batch + (long long)(row + i / groups) * o.row + head * o.head + i % groups * 8) =
            make_uint4(0, 0, 0, 0);
}

// Few blocks with long walks leave most SMs without work, so the walk is dealt out to `splits` blocks; each leaves its float
// sums as part k of [splits][batch][len][heads][dim], and the call's last kernel joins them in order.
struct Parts {
    int splits;
    float *data;
    long long rows;     // batch * len * heads
    int len, heads;
    __device__ __forceinline__ float *at(int part, int batch, int row, int head, int dim) const
    {
        return data + (((long long)part * rows + ((long long)batch * len + row) * heads + head) * dim);
    }
};
// The stretch [from, to) of n steps that part k of `splits` takes.
__device__ __forceinline__ void stretch_of(int n, int k, int splits, int *from, int *to)
{
    *from = int((long long)n * k / splits);
    *to = int((long long)n * (k + 1) / splits);
}
__device__ __forceinline__ void zero_parts(const Parts &o, int part, int batch, int head, int row, int rows, int dim)
{
    for (int i = threadIdx.x; i < rows * dim; i += blockDim.x) o.at(part, batch, row + i / dim, head, dim)[i % dim] = 0.0f;
}
// Sum of the parts at 8 columns of a row, weighted by w(part).
template <typename W> __device__ __forceinline__ void join_parts(const Parts &o, int batch, int row, int head, int dim, int c, float *sum, W w)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    for (int k = 0; k < o.splits; ++k) {
        float f[8];
        load_group(o.at(k, batch, row, head, dim) + c, f);
        const float g = w(k);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = fmaf(g, f[e], sum[e]);
    }
}

}  // namespace omni
