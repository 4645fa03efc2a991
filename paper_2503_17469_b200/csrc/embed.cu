// Embedding lookup with scaling, and its dense gradient by sorted tokens.
//
// Lookup: out_i = s * W[t_i].  Pure gather: the floor is the n rows written plus the distinct rows
// read.  A group of lanes owns a row, 8 elements (16 or 32 bytes) per lane and access.
//
// Gradient: dW_v = s * sum_{t_i = v} dy_i.  Scattered adds with atomics would leave the order of
// the sum to chance, so the tokens are sorted first and every row of the table is then written
// once, by an owner that adds its terms in order:
//   1. sort_tokens: CTA c owns the ids [512 c, 512 c + 512).  It walks all n tokens, counts its own
//      (per warp and id, in shared memory) and those of smaller ids, which gives its place in the sorted
//      order without a word between CTAs, then walks them again and writes (position, id) at its place.
//      Stable: warps take consecutive stretches of the tokens, lanes of a match rank by lane.
//   2. sum_runs: the sorted list is cut into blocks of 32, whatever the ids, so that a token that
//      fills a tenth of the batch is spread over as many owners as it needs.  A group of lanes adds a
//      block's rows in registers, and where the id changes writes the row -- or, for the run
//      that crosses the block's edge, a float partial to the workspace.  Rows without a token are set to zero by
//      further groups of the same launch.
//   3. join_runs: for each run that crosses an edge, the owner of its first block adds the partials
//      in block order and writes the row.
#include "context.h"
#include "vector.cuh"

namespace omni {
namespace {

constexpr int kIdsPerCta = 512;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kBlock = 32;          // sorted tokens per block
constexpr int kThreads = 256;
constexpr int kBatch = 4;           // rows in flight per group of lanes

struct Entry { int pos, id; };      // a token's place in the batch, and its id

template <typename I>
__device__ __forceinline__ int token_id(const void *tokens, long long i, int vocab, long long padding)
{
    const long long t = load_index<I>(tokens, i);
    return t >= 0 && t < vocab && t != padding ? int(t) : -1;
}

// ---- lookup -------------------------------------------------------------------------------------

// LANES lanes per row.  WIDE: groups of 8 elements (dim a multiple of 8, rows 16-byte aligned), else
// single elements.
template <typename I, typename T, typename O, bool WIDE>
__global__ void __launch_bounds__(kThreads) embed_lookup_kernel(const void *tokens, long long n, const T *table,
                                                                unsigned long long table_stride, int vocab, int dim,
                                                                float scale, O *out, unsigned long long out_stride, int lanes)
{
    const int per = kThreads / lanes, lane = threadIdx.x % lanes;
    const long long i = (long long)blockIdx.x * per + threadIdx.x / lanes;
    if (i >= n) return;
    const long long t = load_index<I>(tokens, i);
    const bool there = t >= 0 && t < vocab;
    const T *src = table + (there ? (unsigned long long)t : 0ull) * table_stride;
    O *dst = out + (unsigned long long)i * out_stride;
    constexpr int E = WIDE ? kGroup : 1;
    const int units = dim / E;
    for (int u = lane; u < units; u += lanes * kBatch) {
        float f[kBatch][E];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int w = u + b * lanes;
            if (w < units && there) {
                if constexpr (WIDE) load_group(src + w * E, f[b]);
                else f[b][0] = to_float(src[w]);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int w = u + b * lanes;
            if (w >= units) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) f[b][e] = there ? f[b][e] * scale : 0.0f;
            if constexpr (WIDE) store_group(dst + w * E, f[b]);
            else dst[w] = from_float<O>(f[b][0]);
        }
    }
}

// ---- sort ---------------------------------------------------------------------------------------

template <typename I>
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const void *tokens, long long n, int vocab,
                                                                   long long padding, Entry *sorted, int *start)
{
    extern __shared__ int hist[];   // [kSortWarps][kIdsPerCta]
    __shared__ int below_total, warp_sum[kIdsPerCta / 32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int lo = blockIdx.x * kIdsPerCta;
    for (int i = threadIdx.x; i < kSortWarps * kIdsPerCta; i += kSortThreads) hist[i] = 0;
    if (threadIdx.x == 0) below_total = 0;
    __syncthreads();
    const long long stretch = ((n + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
    const long long first = warp * stretch, last = first + stretch < n ? first + stretch : n;
    int *mine = hist + warp * kIdsPerCta;
    int below = 0;
    for (long long base = first; base < last; base += 32 * 4) {
        int id[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const long long i = base + b * 32 + lane;
            id[b] = i < last ? token_id<I>(tokens, i, vocab, padding) : -1;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            below += id[b] >= 0 && id[b] < lo;
            if (id[b] >= lo && id[b] < lo + kIdsPerCta) atomicAdd(&mine[id[b] - lo], 1);
        }
    }
    for (int o = 16; o > 0; o /= 2) below += __shfl_down_sync(~0u, below, o);
    if (lane == 0 && below) atomicAdd(&below_total, below);
    __syncthreads();
    // exclusive sums: over the warps of an id, then over the ids
    int total = 0, inc = 0;
    if (threadIdx.x < kIdsPerCta) {
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = hist[w * kIdsPerCta + threadIdx.x];
            hist[w * kIdsPerCta + threadIdx.x] = total;
            total += c;
        }
        inc = total;
        for (int o = 1; o < 32; o *= 2) {
            const int y = __shfl_up_sync(~0u, inc, o);
            if (lane >= o) inc += y;
        }
        if (lane == 31) warp_sum[warp] = inc;
    }
    __syncthreads();
    if (threadIdx.x < kIdsPerCta) {
        int at = below_total + inc - total;
        for (int w = 0; w < warp; ++w) at += warp_sum[w];
        const int id = lo + threadIdx.x;
        if (id < vocab) start[id] = at;
        if (id == vocab - 1) start[vocab] = at + total;
        for (int w = 0; w < kSortWarps; ++w) hist[w * kIdsPerCta + threadIdx.x] += at;
    }
    __syncthreads();
    for (long long base = first; base < last; base += 32 * 4) {
        int id[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const long long i = base + b * 32 + lane;
            id[b] = i < last ? token_id<I>(tokens, i, vocab, padding) : -1;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const bool in = id[b] >= lo && id[b] < lo + kIdsPerCta;
            const unsigned takers = __ballot_sync(~0u, in);
            if (!takers) continue;
            if (in) {
                const unsigned peers = __match_any_sync(takers, id[b]);
                const int rank = __popc(peers & ((1u << lane) - 1u));
                const int at = mine[id[b] - lo] + rank;
                sorted[at] = {int(base + b * 32 + lane), id[b]};
                __syncwarp(takers);
                if (rank == 0) mine[id[b] - lo] += __popc(peers);
                __syncwarp(takers);
            }
        }
    }
}

// ---- sums ---------------------------------------------------------------------------------------

template <typename G, bool WIDE>
__device__ __forceinline__ void put_row(G *dst, int col, float *acc, float scale, bool accumulate)
{
    constexpr int E = WIDE ? kGroup : 1;
    float o[E];
    if (accumulate) {
        if constexpr (WIDE) load_group(dst + col, o);
        else o[0] = to_float(dst[col]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = accumulate ? fmaf(scale, acc[e], o[e]) : scale * acc[e];
    if constexpr (WIDE) store_group(dst + col, o);
    else dst[col] = from_float<G>(o[0]);
}

struct RunParams {
    const Entry *sorted;
    const int *start;
    float *partial;             // [2 * blocks][padded dim]
    long long blocks;           // upper bound: of n tokens
    int vocab, dim, padded;     // padded: dim rounded up to 8
    int lanes, slices;          // lanes per group, column slices of lanes * E elements
    float scale;
    int accumulate;
    unsigned long long src_stride, dst_stride;
};

template <typename T, typename G, bool WIDE>
__global__ void __launch_bounds__(kThreads) sum_runs_kernel(RunParams p, const T *src, G *dst, long long run_groups)
{
    constexpr int E = WIDE ? kGroup : 1;
    const int per = kThreads / p.lanes, lane = threadIdx.x % p.lanes;
    const long long g = (long long)blockIdx.x * per + threadIdx.x / p.lanes;
    if (g >= run_groups) {
        // rows without a token: zeros
        const long long v = g - run_groups;
        if (p.accumulate || v >= p.vocab || p.start[v] != p.start[v + 1]) return;
        G *row = dst + (unsigned long long)v * p.dst_stride;
        float zero[E] = {};
        for (int col = lane * E; col < p.dim; col += p.lanes * E) {
            if constexpr (WIDE) store_group(row + col, zero);
            else row[col] = from_float<G>(0.0f);
        }
        return;
    }
    const long long block = g / p.slices;
    const int col = (int(g % p.slices) * p.lanes + lane) * E;
    const int total = p.start[p.vocab];
    const long long begin = block * kBlock;
    if (begin >= total || col >= p.dim) return;
    const int end = begin + kBlock < total ? int(begin) + kBlock : total;
    int cur = p.sorted[begin].id;
    bool open = begin > 0 && p.sorted[begin - 1].id == cur;     // the run began before this block
    const int next = end < total ? p.sorted[end].id : -1;
    float acc[E] = {};
    for (int i = int(begin); i < end; i += kBatch) {
        Entry en[kBatch];
        float f[kBatch][E];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) en[b] = i + b < end ? p.sorted[i + b] : Entry{-1, -1};
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            if (en[b].id >= 0) {
                const T *row = src + (unsigned long long)en[b].pos * p.src_stride;
                if constexpr (WIDE) load_group(row + col, f[b]);
                else f[b][0] = to_float(row[col]);
            }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (en[b].id < 0) continue;
            if (en[b].id != cur) {
                if (open) {
#pragma unroll
                    for (int e = 0; e < E; ++e) p.partial[(2 * block) * p.padded + col + e] = acc[e];
                } else {
                    put_row<G, WIDE>(dst + (unsigned long long)cur * p.dst_stride, col, acc, p.scale, p.accumulate);
                }
                open = false;
                cur = en[b].id;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += f[b][e];
        }
    }
    if (!open && next != cur) {
        put_row<G, WIDE>(dst + (unsigned long long)cur * p.dst_stride, col, acc, p.scale, p.accumulate);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) p.partial[(2 * block + (open ? 0 : 1)) * p.padded + col + e] = acc[e];
    }
}

// One group per (block, slice): if a run starts in the block and goes on in the next, add its partials.
template <typename G, bool WIDE>
__global__ void __launch_bounds__(kThreads) join_runs_kernel(RunParams p, G *dst, long long run_groups)
{
    constexpr int E = WIDE ? kGroup : 1;
    const int per = kThreads / p.lanes, lane = threadIdx.x % p.lanes;
    const long long g = (long long)blockIdx.x * per + threadIdx.x / p.lanes;
    if (g >= run_groups) return;
    const long long block = g / p.slices;
    const int col = (int(g % p.slices) * p.lanes + lane) * E;
    const int total = p.start[p.vocab];
    const long long edge = (block + 1) * kBlock;
    if (edge >= total || col >= p.dim) return;
    const int id = p.sorted[edge].id;
    if (p.sorted[edge - 1].id != id || p.start[id] / kBlock != block) return;
    const long long last = (p.start[id + 1] - 1) / kBlock;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = p.partial[(2 * block + 1) * p.padded + col + e];
#pragma unroll 4
    for (long long b = block + 1; b <= last; ++b) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += p.partial[(2 * b) * p.padded + col + e];
    }
    put_row<G, WIDE>(dst + (unsigned long long)id * p.dst_stride, col, acc, p.scale, p.accumulate);
}

// ---- host side ----------------------------------------------------------------------------------

unsigned long long round_up(unsigned long long x, unsigned long long m) { return (x + m - 1) / m * m; }
size_t element_size(int32_t dtype) { return dtype == OMNI_BF16 ? 2 : 4; }
bool known_dtype(int32_t d) { return d == OMNI_F32 || d == OMNI_BF16; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Rows that groups of 8 elements can be taken from.
bool wide_rows(const void *p, int32_t dtype, uint64_t stride)
{
    return aligned(p, 16) && stride * element_size(dtype) % 16 == 0;
}

// Lanes that share a row: enough to cover it with one access each, a warp at most.
int lanes_for(int dim, bool wide)
{
    const int units = wide ? dim / kGroup : dim;
    int lanes = 1;
    while (lanes < 32 && lanes < units) lanes *= 2;
    return lanes;
}

struct EmbedWorkspace { unsigned long long sorted, start, partial, bytes; };

EmbedWorkspace plan_workspace(uint64_t n, int32_t vocab, int32_t dim)
{
    EmbedWorkspace w;
    w.sorted = 0;
    w.start = round_up(n * sizeof(Entry), 256);
    w.partial = w.start + round_up((uint64_t(vocab) + 1) * sizeof(int), 256);
    const uint64_t blocks = (n + kBlock - 1) / kBlock;
    w.bytes = w.partial + 2 * blocks * round_up(dim, kGroup) * sizeof(float);
    return w;
}

int check_embed(const void *tokens, int32_t index_type, uint64_t n, const void *rows, int32_t rows_dtype,
                uint64_t rows_stride, int32_t vocab, int32_t dim, float scale, const void *table, int32_t table_dtype,
                uint64_t table_stride)
{
    if (index_type != OMNI_I32 && index_type != OMNI_I64) return OMNI_ERR_BAD_CONFIG;
    if (!known_dtype(rows_dtype) || !known_dtype(table_dtype) || vocab < 1 || dim < 1) return OMNI_ERR_BAD_CONFIG;
    if (rows_stride < uint64_t(dim) || table_stride < uint64_t(dim)) return OMNI_ERR_BAD_CONFIG;
    if (!(scale - scale == 0.0f)) return OMNI_ERR_BAD_CONFIG;   // not finite
    if (!table || (n > 0 && (!tokens || !rows))) return OMNI_ERR_NULL;
    if (n >= (1ull << 31)) return OMNI_ERR_TOO_LARGE;
    if (!aligned(tokens, index_type == OMNI_I64 ? 8 : 4) || !aligned(rows, element_size(rows_dtype)) ||
        !aligned(table, element_size(table_dtype)))
        return OMNI_ERR_ALIGN;
    return OMNI_OK;
}

// Calls f with a null pointer of the element type `dtype` names.
template <typename F> int with_type(int32_t dtype, F f)
{
    return dtype == OMNI_BF16 ? f(static_cast<__nv_bfloat16 *>(nullptr)) : f(static_cast<float *>(nullptr));
}
template <typename F> int with_index(int32_t type, F f)
{
    return type == OMNI_I64 ? f(static_cast<long long *>(nullptr)) : f(static_cast<int *>(nullptr));
}
template <typename F> int with_flag(bool flag, F f)
{
    return flag ? f(std::integral_constant<bool, true>{}) : f(std::integral_constant<bool, false>{});
}

}  // namespace
}  // namespace omni

using namespace omni;

extern "C" {

int omni_embed_forward(omni_ctx *ctx, const void *tokens, int32_t index_type, uint64_t n, const void *table,
                       int32_t table_dtype, uint64_t table_stride, int32_t vocab, int32_t dim, float scale, void *out,
                       int32_t out_dtype, uint64_t out_stride, void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_embed(tokens, index_type, n, out, out_dtype, out_stride, vocab, dim, scale, table, table_dtype, table_stride);
    if (rc != OMNI_OK) return rc;
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK || n == 0) return rc;
    const bool wide = dim % kGroup == 0 && wide_rows(table, table_dtype, table_stride) && wide_rows(out, out_dtype, out_stride);
    const int lanes = lanes_for(dim, wide), per = kThreads / lanes;
    const unsigned grid = unsigned((n + per - 1) / per);
    return with_index(index_type, [&](auto *ip) {
        return with_type(table_dtype, [&](auto *tp) {
            return with_type(out_dtype, [&](auto *op) {
                return with_flag(wide, [&](auto w) {
                    using I = std::remove_pointer_t<decltype(ip)>;
                    using T = std::remove_pointer_t<decltype(tp)>;
                    using O = std::remove_pointer_t<decltype(op)>;
                    embed_lookup_kernel<I, T, O, decltype(w)::value><<<grid, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
                        tokens, (long long)n, static_cast<const T *>(table), table_stride, vocab, dim, scale,
                        static_cast<O *>(out), out_stride, lanes);
                    return context_launched(ctx, int(cudaGetLastError()));
                });
            });
        });
    });
}

int omni_embed_workspace(uint64_t n, int32_t vocab, int32_t dim, uint64_t *bytes)
{
    if (!bytes) return OMNI_ERR_NULL;
    if (vocab < 1 || dim < 1) return OMNI_ERR_BAD_CONFIG;
    if (n >= (1ull << 31)) return OMNI_ERR_TOO_LARGE;
    *bytes = plan_workspace(n, vocab, dim).bytes;
    return OMNI_OK;
}

int omni_embed_backward(omni_ctx *ctx, const void *tokens, int32_t index_type, uint64_t n, const void *grad_out,
                        int32_t grad_out_dtype, uint64_t grad_out_stride, int32_t vocab, int32_t dim, float scale,
                        int64_t padding, void *grad, int32_t grad_dtype, uint64_t grad_stride, int32_t accumulate,
                        void *workspace, uint64_t workspace_bytes, void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_embed(tokens, index_type, n, grad_out, grad_out_dtype, grad_out_stride, vocab, dim, scale, grad,
                         grad_dtype, grad_stride);
    if (rc != OMNI_OK) return rc;
    if (!workspace) return OMNI_ERR_NULL;
    if (!aligned(workspace, 16)) return OMNI_ERR_ALIGN;
    const EmbedWorkspace w = plan_workspace(n, vocab, dim);
    if (workspace_bytes < w.bytes) return OMNI_ERR_TOO_LARGE;
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    Entry *sorted = reinterpret_cast<Entry *>(ws + w.sorted);
    int *start = reinterpret_cast<int *>(ws + w.start);
    const int smem = kSortWarps * kIdsPerCta * int(sizeof(int));
    rc = with_index(index_type, [&](auto *ip) {
        using I = std::remove_pointer_t<decltype(ip)>;
        const int r = context_shared(ctx, reinterpret_cast<const void *>(sort_tokens_kernel<I>), smem);
        if (r != OMNI_OK) return r;
        sort_tokens_kernel<I><<<(vocab + kIdsPerCta - 1) / kIdsPerCta, kSortThreads, smem, s>>>(tokens, (long long)n, vocab,
                                                                                               padding, sorted, start);
        return context_launched(ctx, int(cudaGetLastError()));
    });
    if (rc != OMNI_OK) return rc;
    const bool wide = dim % kGroup == 0 && wide_rows(grad_out, grad_out_dtype, grad_out_stride) &&
                      wide_rows(grad, grad_dtype, grad_stride);
    RunParams p;
    p.sorted = sorted;
    p.start = start;
    p.partial = reinterpret_cast<float *>(ws + w.partial);
    p.blocks = (n + kBlock - 1) / kBlock;
    p.vocab = vocab;
    p.dim = dim;
    p.padded = int(round_up(dim, kGroup));
    p.lanes = lanes_for(dim, wide);
    const int cols = p.lanes * (wide ? kGroup : 1);
    p.slices = (dim + cols - 1) / cols;
    p.scale = scale;
    p.accumulate = accumulate != 0;
    p.src_stride = grad_out_stride;
    p.dst_stride = grad_stride;
    const int per = kThreads / p.lanes;
    const long long run_groups = p.blocks * p.slices;
    const long long groups = run_groups + (accumulate ? 0 : vocab);
    return with_type(grad_out_dtype, [&](auto *tp) {
        return with_type(grad_dtype, [&](auto *gp) {
            return with_flag(wide, [&](auto wd) {
                using T = std::remove_pointer_t<decltype(tp)>;
                using G = std::remove_pointer_t<decltype(gp)>;
                constexpr bool W = decltype(wd)::value;
                if (groups == 0) return int(OMNI_OK);
                sum_runs_kernel<T, G, W><<<unsigned((groups + per - 1) / per), kThreads, 0, s>>>(
                    p, static_cast<const T *>(grad_out), static_cast<G *>(grad), run_groups);
                const int r = context_launched(ctx, int(cudaGetLastError()));
                if (r != OMNI_OK || p.blocks < 2) return r;
                join_runs_kernel<G, W><<<unsigned((run_groups + per - 1) / per), kThreads, 0, s>>>(p, static_cast<G *>(grad),
                                                                                                  run_groups);
                return context_launched(ctx, int(cudaGetLastError()));
            });
        });
    });
}

}  // extern "C"
