// Norms of the query and key heads with the rotation by positions, forward and backward, in one pass.
//
// Per head vector x, with weights w: n_c = w_c x_c r, r = (mean_c x_c^2 + eps)^(-1/2); without weights n = x.  A pair (a, b) of n is
// turned by the angle position * frequency:
//   y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin.
// Backward, from x and dy: dn is dy turned back, dw_c = sum of dn_c x_c r over all rows and heads of the side, and with g = w dn
//   dx = r (g - x r^2 mean_c(g_c x_c)).
// Without weights the gradient is the rotation by the opposite angle.
#include "context.h"
#include "vector.cuh"

namespace omni {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxPairs = OMNI_ROTARY_MAX_DIM / 2;
constexpr int kMaxTile = 32;                          // rows whose angles a block holds
constexpr int kResident = 2;                          // backward blocks an SM
constexpr double kInvTwoPi = 0.15915494309189533577;

struct View {
    void *data;
    unsigned long long batch, row, head;
};
struct Side {
    View x, dy, out;                                  // dy: backward only
    const void *weight;
    float *partial;                                   // backward: blocks x dim sums of the weight's gradient
    int heads;
    unsigned blocks;
};
struct RotaryParams {
    Side side[2];                                     // queries, keys
    const void *positions;
    unsigned long long position_axis, position_batch, position_row;
    const int *lengths;
    unsigned rows, length;                            // batch * length, length
    int dim, pairs, lanes, tile;                      // lanes of a head vector (a power of two), rows of a tile (a power of two)
    int wide_positions, bf16_weight, interleaved, overlap;
    float eps, turn;                                  // turn: 1, or -1 for the opposite angle
    double frequency[kMaxPairs];
    unsigned char axis[kMaxPairs];
};

// V consecutive elements, kept as loaded.
template <typename T, int V> struct Chunk;
template <> struct Chunk<__nv_bfloat16, 8> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { u = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float *f) const { widen(u, f); }
};
template <> struct Chunk<float, 8> {
    float v[8];
    __device__ __forceinline__ void load(const float *p) { load_group(p, v); }
    __device__ __forceinline__ void get(float *f) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[i];
    }
};
template <typename T> struct Chunk<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void get(float *f) const { *f = to_float(v); }
};
template <typename T, int V> __device__ __forceinline__ void put(T *p, const float *f)
{
    if constexpr (V == 8) store_group(p, f);
    else *p = from_float<T>(*f);
}

// What a lane has of a head vector: UNITS units of V pairs, that is two chunks of V elements each.  With V = 8 one unit is enough
// (16 lanes hold 256 elements); element by element it takes up to four.
template <int V> constexpr int kUnits = V == 8 ? 1 : kMaxPairs / 32;

// Where a unit's two chunks stand.  The elements that are not rotated are pairs of angle zero behind the others.
struct Place { int a, b; };
template <int V> __device__ __forceinline__ Place place(const RotaryParams &p, int unit)
{
    const int first = unit * V;
    if (p.interleaved) return {2 * first, 2 * first + V};
    const int rest = p.dim / 2 - p.pairs;
    return first < p.pairs ? Place{first, first + p.pairs} : Place{first + p.pairs, first + p.pairs + rest};
}

__device__ __forceinline__ float group_sum(float x, int lanes)
{
    for (int o = lanes / 2; o > 0; o /= 2) x += __shfl_xor_sync(~0u, x, o);
    return x;
}

// The first and second elements of pair i of a unit's 2 V elements.
template <int V, bool ADJACENT> __device__ __forceinline__ constexpr int first_of(int i) { return ADJACENT ? 2 * i : i; }
template <int V, bool ADJACENT> __device__ __forceinline__ constexpr int second_of(int i) { return ADJACENT ? 2 * i + 1 : i + V; }

// A table row of cosines, then sines: a unit's eight as two pieces of four in two planes, so that neighbouring lanes
// read neighbouring 16 bytes.
template <int V> __device__ __forceinline__ int cell(int pair, int half)
{
    return V == 8 ? (pair & 4 ? half / 2 : 0) + pair / 8 * 4 + pair % 4 : pair;
}

template <int V> __device__ __forceinline__ void fill_angles(const RotaryParams &p, unsigned first, float *table)
{
    const int half = p.dim / 2;
    for (int i = threadIdx.x; i < p.tile * half; i += kThreads) {
        const int k = i / half, pair = i % half;
        const unsigned row = first + k;
        float c = 1.0f, s = 0.0f;
        if (pair < p.pairs && row < p.rows) {
            const unsigned long long at = p.axis[pair] * p.position_axis + row / p.length * p.position_batch + row % p.length * p.position_row;
            const long long position = p.wide_positions ? load_index<long long>(p.positions, at) : load_index<int>(p.positions, at);
            // in turns and in 64 bits: what is left of the angle after its whole turns keeps 2^-51 of the angle
            const double turns = double(position) * (p.frequency[pair] * kInvTwoPi);
            sincospif(2.0f * float(turns - rint(turns)), &s, &c);
            s *= p.turn;
        }
        table[k * p.dim + cell<V>(pair, half)] = c;
        table[k * p.dim + half + cell<V>(pair, half)] = s;
    }
}
template <int V> __device__ __forceinline__ void read_angles(const float *row, int half, int unit, float *c, float *s)
{
    if constexpr (V == 8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 x = *reinterpret_cast<const float4 *>(row + h * (half / 2) + unit * 4);
            const float4 y = *reinterpret_cast<const float4 *>(row + half + h * (half / 2) + unit * 4);
            c[4 * h] = x.x; c[4 * h + 1] = x.y; c[4 * h + 2] = x.z; c[4 * h + 3] = x.w;
            s[4 * h] = y.x; s[4 * h + 1] = y.y; s[4 * h + 2] = y.z; s[4 * h + 3] = y.w;
        }
    } else {
        *c = row[unit];
        *s = row[half + unit];
    }
}

template <typename T> __device__ __forceinline__ T *vector_at(const View &v, unsigned row, unsigned length, int head)
{
    return static_cast<T *>(v.data) + row / length * v.batch + row % length * v.row + head * v.head;
}

// What a lane keeps for its row: angles and places, and for the block's side its part of the weights.
template <int V> struct Lane {
    static constexpr int kN = kUnits<V>;
    int group, lane, first_head, stride;              // heads of this group: first_head, first_head + stride, ...
    float w[kN][2 * V];
    Place at[kN];
    bool has[kN];
    __device__ __forceinline__ Lane(const RotaryParams &p, const Side &side, bool norm)
    {
        group = threadIdx.x / p.lanes;
        lane = threadIdx.x % p.lanes;
        stride = kThreads / p.lanes / p.tile;         // groups of a row
        first_head = group % stride;
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            const int unit = lane + n * p.lanes;
            has[n] = unit * V < p.dim / 2;
            at[n] = place<V>(p, has[n] ? unit : 0);
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) {
                const int c = e < V ? at[n].a + e : at[n].b + e - V;
                w[n][e] = !norm ? 1.0f : p.bf16_weight ? to_float(static_cast<const __nv_bfloat16 *>(side.weight)[c])
                                                       : static_cast<const float *>(side.weight)[c];
            }
        }
    }
    __device__ __forceinline__ int row_in_tile() const { return group / stride; }
};

__device__ __forceinline__ bool row_there(const RotaryParams &p, unsigned row)
{
    return !p.lengths || int(row % p.length) < p.lengths[row / p.length];
}

// Forward: a block has a tile of rows of one side; a group of lanes goes through heads of one row, AHEAD of them in flight.
template <typename T, int V, bool ADJACENT, bool NORM>
__global__ void __launch_bounds__(kThreads) rotary_forward_kernel(const __grid_constant__ RotaryParams p)
{
    extern __shared__ __align__(16) float table[];
    constexpr int kN = kUnits<V>, kAhead = sizeof(T) == 2 ? 4 : 2;
    const bool keys = blockIdx.x >= p.side[0].blocks;
    const Side &side = p.side[keys];
    const unsigned first = (blockIdx.x - (keys ? p.side[0].blocks : 0u)) * unsigned(p.tile);
    const Lane<V> me(p, side, NORM);
    const unsigned row = first + me.row_in_tile();
    const bool mine = row < p.rows, there = mine && row_there(p, row);
    const float inverse_dim = 1.0f / float(p.dim);
    const int half = p.dim / 2;
    float c[kN][V], s[kN][V];
    // every group of a warp takes as many turns, for the shuffles
    for (int h0 = 0; h0 < side.heads; h0 += me.stride * kAhead) {
        Chunk<T, V> x[kAhead][kN][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int head = h0 + i * me.stride + me.first_head;
            if (there && head < side.heads) {
                const T *src = vector_at<T>(side.x, row, p.length, head);
#pragma unroll
                for (int n = 0; n < kN; ++n)
                    if (me.has[n]) {
                        x[i][n][0].load(src + me.at[n].a);
                        x[i][n][1].load(src + me.at[n].b);
                    }
            }
        }
        if (h0 == 0) {                                // the first loads are under way
            fill_angles<V>(p, first, table);
            __syncthreads();
#pragma unroll
            for (int n = 0; n < kN; ++n)
                if (me.has[n]) read_angles<V>(table + me.row_in_tile() * p.dim, half, me.lane + n * p.lanes, c[n], s[n]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int head = h0 + i * me.stride + me.first_head;
            const bool work = mine && head < side.heads;
            float f[kN][2 * V], r = 1.0f;
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                if (work && there && me.has[n]) {
                    x[i][n][0].get(f[n]);
                    x[i][n][1].get(f[n] + V);
                } else {
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) f[n][e] = 0.0f;
                }
            }
            if constexpr (NORM) {
                float sum = 0.0f;
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) sum = fmaf(f[n][e], f[n][e], sum);
                r = 1.0f / sqrtf(fmaf(group_sum(sum, p.lanes), inverse_dim, p.eps));
            }
            if (!work) continue;
            T *dst = vector_at<T>(side.out, row, p.length, head);
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                if (!me.has[n]) continue;
                if (there) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const int a = first_of<V, ADJACENT>(j), b = second_of<V, ADJACENT>(j);
                        const float na = NORM ? f[n][a] * r * me.w[n][a] : f[n][a], nb = NORM ? f[n][b] * r * me.w[n][b] : f[n][b];
                        f[n][a] = fmaf(na, c[n][j], -nb * s[n][j]);
                        f[n][b] = fmaf(nb, c[n][j], na * s[n][j]);
                    }
                }
                put<T, V>(dst + me.at[n].a, f[n]);
                put<T, V>(dst + me.at[n].b, f[n] + V);
            }
        }
    }
}

// Backward of the norm and the rotation: blocks that stay, each on tiles of one side, with the weight's gradient in registers.
template <typename T, int V, bool ADJACENT>
__global__ void __launch_bounds__(kThreads, kResident) rotary_backward_kernel(const __grid_constant__ RotaryParams p)
{
    extern __shared__ __align__(16) float table[];
    constexpr int kN = kUnits<V>, kAhead = 2;
    let_next_begin(p.overlap);
    const bool keys = blockIdx.x >= p.side[0].blocks;
    const Side &side = p.side[keys];
    const unsigned block = blockIdx.x - (keys ? p.side[0].blocks : 0u);
    const Lane<V> me(p, side, true);
    const float inverse_dim = 1.0f / float(p.dim);
    const int half = p.dim / 2;
    float dw[kN][2 * V] = {};
    const unsigned tiles = (p.rows + p.tile - 1) / p.tile;
    for (unsigned t = block; t < tiles; t += side.blocks) {
        const unsigned first = t * unsigned(p.tile), row = first + me.row_in_tile();
        const bool mine = row < p.rows, there = mine && row_there(p, row);
        float c[kN][V], s[kN][V];
        for (int h0 = 0; h0 < side.heads; h0 += me.stride * kAhead) {
            Chunk<T, V> x[kAhead][kN][2], y[kAhead][kN][2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int head = h0 + i * me.stride + me.first_head;
                if (there && head < side.heads) {
                    const T *src = vector_at<T>(side.x, row, p.length, head), *grad = vector_at<T>(side.dy, row, p.length, head);
#pragma unroll
                    for (int n = 0; n < kN; ++n)
                        if (me.has[n]) {
                            x[i][n][0].load(src + me.at[n].a);
                            x[i][n][1].load(src + me.at[n].b);
                            y[i][n][0].load(grad + me.at[n].a);
                            y[i][n][1].load(grad + me.at[n].b);
                        }
                }
            }
            if (h0 == 0) {
                __syncthreads();                      // the last tile's angles have been read
                fill_angles<V>(p, first, table);
                __syncthreads();
#pragma unroll
                for (int n = 0; n < kN; ++n)
                    if (me.has[n]) read_angles<V>(table + me.row_in_tile() * p.dim, half, me.lane + n * p.lanes, c[n], s[n]);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int head = h0 + i * me.stride + me.first_head;
                const bool work = mine && head < side.heads, live = work && there;
                float f[kN][2 * V], g[kN][2 * V], square = 0.0f, dot = 0.0f;
#pragma unroll
                for (int n = 0; n < kN; ++n) {
                    if (live && me.has[n]) {
                        x[i][n][0].get(f[n]);
                        x[i][n][1].get(f[n] + V);
                        y[i][n][0].get(g[n]);
                        y[i][n][1].get(g[n] + V);
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const int a = first_of<V, ADJACENT>(j), b = second_of<V, ADJACENT>(j);
                            const float ya = g[n][a], yb = g[n][b];
                            g[n][a] = fmaf(ya, c[n][j], yb * s[n][j]);
                            g[n][b] = fmaf(yb, c[n][j], -ya * s[n][j]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) f[n][e] = g[n][e] = 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) {
                        square = fmaf(f[n][e], f[n][e], square);
                        dot = fmaf(f[n][e] * me.w[n][e], g[n][e], dot);
                    }
                }
                square = group_sum(square, p.lanes);
                dot = group_sum(dot, p.lanes);
                if (!work) continue;
                const float r = 1.0f / sqrtf(fmaf(square, inverse_dim, p.eps));
                const float pull = dot * inverse_dim * r * r;
                T *dst = vector_at<T>(side.out, row, p.length, head);
#pragma unroll
                for (int n = 0; n < kN; ++n) {
                    if (!me.has[n]) continue;
                    if (there) {
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) {
                            dw[n][e] = fmaf(g[n][e], f[n][e] * r, dw[n][e]);
                            f[n][e] = r * fmaf(-f[n][e], pull, g[n][e] * me.w[n][e]);
                        }
                    }
                    put<T, V>(dst + me.at[n].a, f[n]);
                    put<T, V>(dst + me.at[n].b, f[n] + V);
                }
            }
        }
    }
    // the block's sums: groups of a warp by shuffles, then the warps in order
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
            float v = dw[n][e];
            for (int o = 16; o >= p.lanes; o /= 2) v += __shfl_xor_sync(~0u, v, o);
            if (int(threadIdx.x % 32) < p.lanes && me.has[n]) table[threadIdx.x / 32 * p.dim + (e < V ? me.at[n].a + e : me.at[n].b + e - V)] = v;
        }
    __syncthreads();
    for (int ch = threadIdx.x; ch < p.dim; ch += kThreads) {
        float v = table[ch];
        for (int w = 1; w < kWarps; ++w) v += table[w * p.dim + ch];
        side.partial[(unsigned long long)block * p.dim + ch] = v;
    }
}

struct WeightParams {
    const float *partial[2];
    void *grad[2];
    unsigned blocks[2];
    int dim, bf16;
};
// The blocks' sums of 32 channels of a side: a warp's share of the blocks each, the warps in order.
__global__ void __launch_bounds__(1024) rotary_weight_kernel(const WeightParams p)
{
    __shared__ float sum[32][33];
    const int side = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32, ch = blockIdx.x * 32 + lane;
    wait_for_previous();
    float v = 0.0f;
    if (ch < p.dim)
        for (unsigned b = warp; b < p.blocks[side]; b += 32) v += p.partial[side][(unsigned long long)b * p.dim + ch];
    sum[warp][lane] = v;
    __syncthreads();
    v = sum[lane][warp];                               // channel `warp` of the block's
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(~0u, v, o);
    const int out = blockIdx.x * 32 + warp;
    if (lane == 0 && out < p.dim) {
        if (p.bf16) static_cast<__nv_bfloat16 *>(p.grad[side])[out] = __float2bfloat16_rn(v);
        else static_cast<float *>(p.grad[side])[out] = v;
    }
}

// ---- host ---------------------------------------------------------------------------------------

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_rotary(const omni_rotary *r)
{
    if (!r) return OMNI_ERR_NULL;
    if (r->batch < 0 || r->length < 0 || r->heads < 1 || r->kv_heads < 1 || r->dim < 2 || r->dim % 2 || r->pairs < 1) return OMNI_ERR_BAD_CONFIG;
    if ((r->dtype != OMNI_F32 && r->dtype != OMNI_BF16) || (r->weight_dtype != OMNI_F32 && r->weight_dtype != OMNI_BF16) ||
        (r->position_type != OMNI_I32 && r->position_type != OMNI_I64) || r->axes < 1 || r->axes > OMNI_ROTARY_MAX_AXES)
        return OMNI_ERR_BAD_CONFIG;
    if (r->dim > OMNI_ROTARY_MAX_DIM) return OMNI_ERR_TOO_LARGE;
    if (2 * r->pairs > r->dim || !(r->eps >= 0.0f) || r->eps - r->eps != 0.0f) return OMNI_ERR_BAD_CONFIG;
    if (uint64_t(r->batch) * uint64_t(r->length) >= (1ull << 31) || r->heads > 65535 || r->kv_heads > 65535) return OMNI_ERR_TOO_LARGE;
    if (!r->frequency) return OMNI_ERR_NULL;
    for (int i = 0; i < r->pairs; ++i) {
        if (r->frequency[i] - r->frequency[i] != 0.0) return OMNI_ERR_BAD_CONFIG;
        if (r->axis && (r->axis[i] < 0 || r->axis[i] >= r->axes)) return OMNI_ERR_BAD_CONFIG;
    }
    if (!r->q_weight != !r->k_weight) return OMNI_ERR_NULL;
    const size_t weight = r->weight_dtype == OMNI_BF16 ? 2 : 4;
    if (!aligned(r->q_weight, weight) || !aligned(r->k_weight, weight) || !aligned(r->lengths, 4)) return OMNI_ERR_ALIGN;
    if (uint64_t(r->batch) * uint64_t(r->length) == 0) return OMNI_OK;
    if (!r->positions) return OMNI_ERR_NULL;
    return aligned(r->positions, r->position_type == OMNI_I64 ? 8 : 4) ? OMNI_OK : OMNI_ERR_ALIGN;
}

int check_view(const omni_rotary *r, const omni_attn_view *v, int heads, bool written)
{
    if (!v) return OMNI_ERR_NULL;
    if (uint64_t(r->batch) * uint64_t(r->length) == 0) return OMNI_OK;
    if (!v->data) return OMNI_ERR_NULL;
    if (!aligned(v->data, r->dtype == OMNI_BF16 ? 2 : 4)) return OMNI_ERR_ALIGN;
    const struct { int extent; uint64_t stride; } axis[3] = {{r->batch, v->batch}, {r->length, v->row}, {heads, v->head}};
    for (const auto &a : axis) {
        if (a.extent <= 1) continue;
        if (a.stride >= (1ull << 40)) return OMNI_ERR_TOO_LARGE;
        if (written && a.stride < uint64_t(r->dim)) return OMNI_ERR_BAD_CONFIG;      // rows that a result would write twice
    }
    return OMNI_OK;
}

View view_of(const omni_rotary *r, const omni_attn_view *v, int heads)
{
    return {v->data, r->batch > 1 ? v->batch : 0, r->length > 1 ? v->row : 0, heads > 1 ? v->head : 0};
}

// Whether every chunk of eight elements of an operand lies on a 16-byte boundary.
bool wide_view(const omni_rotary *r, const View &v)
{
    const size_t size = r->dtype == OMNI_BF16 ? 2 : 4;
    return aligned(v.data, 16) && v.batch * size % 16 == 0 && v.row * size % 16 == 0 && v.head * size % 16 == 0;
}

// The launch: rows of a tile, lanes of a head vector, blocks of either side.
struct Shape {
    int lanes, tile;
    unsigned blocks[2];
};

// A row's heads are dealt to a power of two of lane groups, so that a group has about `deep` heads of one row and its angles stay
// in registers; a tile is the rows that fill a block then.  Few rows: one a block, its heads on all groups.
Shape shape_of(const omni_rotary *r, bool wide, int deep, int sms, int resident)
{
    Shape s;
    const int units = wide ? r->dim / 16 : r->dim / 2;
    s.lanes = 1;
    while (s.lanes < units && s.lanes < 32) s.lanes *= 2;
    const uint64_t rows = uint64_t(r->batch) * uint64_t(r->length);
    const int groups = kThreads / s.lanes, fewest = r->heads < r->kv_heads ? r->heads : r->kv_heads;
    s.tile = 1;
    while (s.tile < groups && s.tile < kMaxTile && groups / s.tile * deep > fewest && rows >= uint64_t(s.tile) * 2 * sms) s.tile *= 2;
    const uint64_t tiles = (rows + s.tile - 1) / s.tile;
    s.blocks[0] = s.blocks[1] = unsigned(tiles);
    if (resident) {                                   // blocks that stay: shares by the work of a row, angles included
        const uint64_t all = uint64_t(sms) * resident, q = r->heads + 2, k = r->kv_heads + 2;
        uint64_t share = all * q / (q + k);
        share = share < 1 ? 1 : share > all - 1 ? all - 1 : share;
        s.blocks[0] = unsigned(tiles < share ? tiles : share);
        s.blocks[1] = unsigned(tiles < all - share ? tiles : all - share);
    }
    return s;
}

void fill(RotaryParams *p, const omni_rotary *r, const Shape &s, bool backwards)
{
    p->positions = r->positions;
    p->position_axis = r->position_axis;
    p->position_batch = r->position_batch;
    p->position_row = r->position_row;
    p->lengths = r->lengths;
    p->rows = unsigned(r->batch) * unsigned(r->length);
    p->length = unsigned(r->length);
    p->dim = r->dim;
    p->pairs = r->pairs;
    p->lanes = s.lanes;
    p->tile = s.tile;
    p->wide_positions = r->position_type == OMNI_I64;
    p->bf16_weight = r->weight_dtype == OMNI_BF16;
    p->interleaved = r->interleaved != 0;
    p->eps = r->eps;
    p->turn = backwards ? -1.0f : 1.0f;
    for (int i = 0; i < r->pairs; ++i) {
        p->frequency[i] = r->frequency[i];
        p->axis[i] = r->axis ? (unsigned char)r->axis[i] : 0;
    }
    p->side[0].heads = r->heads;
    p->side[1].heads = r->kv_heads;
    p->side[0].weight = r->q_weight;
    p->side[1].weight = r->k_weight;
    for (int i = 0; i < 2; ++i) p->side[i].blocks = s.blocks[i];
}

// Whole units of eight pairs: rotated and unrotated halves of multiples of eight, or any pairs that stand next to one another.
bool wide_units(const omni_rotary *r) { return r->dim % 16 == 0 && (r->interleaved || r->pairs % 8 == 0); }

template <typename T, bool NORM>
int enqueue_forward(omni_ctx *ctx, const RotaryParams &p, bool wide, cudaStream_t s)
{
    const unsigned grid = p.side[0].blocks + p.side[1].blocks;
    const size_t smem = size_t(p.tile) * p.dim * sizeof(float);
    if (!wide) rotary_forward_kernel<T, 1, false, NORM><<<grid, kThreads, smem, s>>>(p);
    else if (p.interleaved) rotary_forward_kernel<T, 8, true, NORM><<<grid, kThreads, smem, s>>>(p);
    else rotary_forward_kernel<T, 8, false, NORM><<<grid, kThreads, smem, s>>>(p);
    return context_launched(ctx, int(cudaGetLastError()));
}

template <typename T> int enqueue_backward(omni_ctx *ctx, const RotaryParams &p, bool wide, cudaStream_t s)
{
    const unsigned grid = p.side[0].blocks + p.side[1].blocks;
    const size_t smem = size_t(p.tile > kWarps ? p.tile : kWarps) * p.dim * sizeof(float);
    if (!wide) rotary_backward_kernel<T, 1, false><<<grid, kThreads, smem, s>>>(p);
    else if (p.interleaved) rotary_backward_kernel<T, 8, true><<<grid, kThreads, smem, s>>>(p);
    else rotary_backward_kernel<T, 8, false><<<grid, kThreads, smem, s>>>(p);
    return context_launched(ctx, int(cudaGetLastError()));
}

// One pass over both sides without sums: the forward call, and the gradient where there are no weights.
int rotate(omni_ctx *ctx, const omni_rotary *r, const omni_attn_view *const (&in)[2], const omni_attn_view *const (&out)[2], bool backwards,
           const ContextDevice &dev, void *stream)
{
    RotaryParams p;
    bool wide = wide_units(r);
    for (int i = 0; i < 2; ++i) {
        const int heads = i ? r->kv_heads : r->heads;
        p.side[i] = {view_of(r, in[i], heads), {}, view_of(r, out[i], heads), nullptr, nullptr, 0, 0};
        wide = wide && wide_view(r, p.side[i].x) && wide_view(r, p.side[i].out);
    }
    fill(&p, r, shape_of(r, wide, r->dtype == OMNI_BF16 ? 4 : 2, dev.sm_count, 0), backwards);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool norm = r->q_weight && !backwards;
    if (r->dtype == OMNI_BF16)
        return norm ? enqueue_forward<__nv_bfloat16, true>(ctx, p, wide, s) : enqueue_forward<__nv_bfloat16, false>(ctx, p, wide, s);
    return norm ? enqueue_forward<float, true>(ctx, p, wide, s) : enqueue_forward<float, false>(ctx, p, wide, s);
}


constexpr int kMostSms = 256;                         // what the workspace is sized for

uint64_t workspace_bytes(const omni_rotary *r)
{
    return r->q_weight ? uint64_t(kMostSms) * kResident * r->dim * sizeof(float) : 0;
}

}  // namespace
}  // namespace omni

using namespace omni;

extern "C" {

int omni_rotary_forward(omni_ctx *ctx, const omni_rotary *r, const omni_attn_view *q, const omni_attn_view *k, const omni_attn_view *q_out,
                        const omni_attn_view *k_out, void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_rotary(r);
    if (rc == OMNI_OK) rc = check_view(r, q, r->heads, false);
    if (rc == OMNI_OK) rc = check_view(r, k, r->kv_heads, false);
    if (rc == OMNI_OK) rc = check_view(r, q_out, r->heads, true);
    if (rc == OMNI_OK) rc = check_view(r, k_out, r->kv_heads, true);
    if (rc != OMNI_OK) return rc;
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK || r->batch == 0 || r->length == 0) return rc;
    return rotate(ctx, r, {q, k}, {q_out, k_out}, false, dev, stream);
}

int omni_rotary_workspace(const omni_rotary *r, uint64_t *bytes)
{
    if (!bytes) return OMNI_ERR_NULL;
    const int rc = check_rotary(r);
    if (rc == OMNI_OK) *bytes = workspace_bytes(r);
    return rc;
}

int omni_rotary_backward(omni_ctx *ctx, const omni_rotary *r, const omni_attn_view *q, const omni_attn_view *k, const omni_attn_view *dq_out,
                         const omni_attn_view *dk_out, const omni_attn_view *dq, const omni_attn_view *dk, void *dq_weight, void *dk_weight,
                         int32_t weight_grad_dtype, void *workspace, uint64_t bytes, void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_rotary(r);
    if (rc != OMNI_OK) return rc;
    const bool norm = r->q_weight != nullptr;
    if (norm) {
        rc = check_view(r, q, r->heads, false);
        if (rc == OMNI_OK) rc = check_view(r, k, r->kv_heads, false);
    }
    if (rc == OMNI_OK) rc = check_view(r, dq_out, r->heads, false);
    if (rc == OMNI_OK) rc = check_view(r, dk_out, r->kv_heads, false);
    if (rc == OMNI_OK) rc = check_view(r, dq, r->heads, true);
    if (rc == OMNI_OK) rc = check_view(r, dk, r->kv_heads, true);
    if (rc != OMNI_OK) return rc;
    if (norm) {
        if (weight_grad_dtype != OMNI_F32 && weight_grad_dtype != OMNI_BF16) return OMNI_ERR_BAD_CONFIG;
        if (!dq_weight || !dk_weight || !workspace) return OMNI_ERR_NULL;
        const size_t size = weight_grad_dtype == OMNI_BF16 ? 2 : 4;
        if (!aligned(dq_weight, size) || !aligned(dk_weight, size) || !aligned(workspace, 16)) return OMNI_ERR_ALIGN;
        if (bytes < workspace_bytes(r)) return OMNI_ERR_TOO_LARGE;
    }
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK) return rc;
    const bool empty = r->batch == 0 || r->length == 0;
    if (!norm) return empty ? OMNI_OK : rotate(ctx, r, {dq_out, dk_out}, {dq, dk}, true, dev, stream);

    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    WeightParams w;
    w.dim = r->dim;
    w.bf16 = weight_grad_dtype == OMNI_BF16;
    w.grad[0] = dq_weight;
    w.grad[1] = dk_weight;
    w.blocks[0] = w.blocks[1] = 0;                    // without rows the gradient is zeros
    w.partial[0] = w.partial[1] = static_cast<const float *>(workspace);
    if (!empty) {
        RotaryParams p;
        const omni_attn_view *const x[2] = {q, k}, *const dy[2] = {dq_out, dk_out}, *const dx[2] = {dq, dk};
        bool wide = wide_units(r);
        for (int i = 0; i < 2; ++i) {
            const int heads = i ? r->kv_heads : r->heads;
            p.side[i] = {view_of(r, x[i], heads), view_of(r, dy[i], heads), view_of(r, dx[i], heads), nullptr, nullptr, 0, 0};
            wide = wide && wide_view(r, p.side[i].x) && wide_view(r, p.side[i].dy) && wide_view(r, p.side[i].out);
        }
        const Shape shape = shape_of(r, wide, 2, dev.sm_count < kMostSms ? dev.sm_count : kMostSms, kResident);
        fill(&p, r, shape, false);
        p.overlap = dev.overlap;
        p.side[0].partial = static_cast<float *>(workspace);
        p.side[1].partial = p.side[0].partial + uint64_t(shape.blocks[0]) * r->dim;
        for (int i = 0; i < 2; ++i) {
            w.partial[i] = p.side[i].partial;
            w.blocks[i] = shape.blocks[i];
        }
        rc = r->dtype == OMNI_BF16 ? enqueue_backward<__nv_bfloat16>(ctx, p, wide, s) : enqueue_backward<float>(ctx, p, wide, s);
        if (rc != OMNI_OK) return rc;
    }
    Dependent launch(dev, dim3((r->dim + 31) / 32, 2), 1024, 0, s);
    if (empty) launch.cfg.numAttrs = 0;
    return context_launched(ctx, int(cudaLaunchKernelEx(&launch.cfg, rotary_weight_kernel, w)));
}

}  // extern "C"
