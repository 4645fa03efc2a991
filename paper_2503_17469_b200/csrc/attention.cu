// C ABI of attention: argument checks, tensor maps, launches.
#include <cmath>
#include <cstring>

#include "attention_backward.cuh"
#include "attention_forward.cuh"
#include "context.h"
#include "vector.cuh"

namespace omni {
namespace {

constexpr int64_t kSms = 148;

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
uint64_t round_up(uint64_t x, uint64_t m) { return (x + m - 1) / m * m; }

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, through the runtime (the library does not link libcuda).
int encoder(omni_ctx *ctx, EncodeTiled *out)
{
    static EncodeTiled found = nullptr;     // the same address whoever looks it up first
    if (!found) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
        if (e != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn)
            return context_launched(ctx, e != cudaSuccess ? int(e) : int(cudaErrorSymbolNotFound));
        found = reinterpret_cast<EncodeTiled>(fn);
    }
    *out = found;
    return OMNI_OK;
}

// View as (column, head, row, batch) with boxes of 64 columns x 128 rows of one head.
int make_map(omni_ctx *ctx, EncodeTiled encode, CUtensorMap *map, const omni_attn_view &v, int dim, int heads, int len,
             int batch)
{
    const cuuint64_t extent[4] = {cuuint64_t(dim), cuuint64_t(heads), cuuint64_t(len), cuuint64_t(batch)};
    // the stride of an extent of one is never used, but has to be a legal one
    const cuuint64_t strides[3] = {heads > 1 ? v.head * 2 : 16, len > 1 ? v.row * 2 : 16, batch > 1 ? v.batch * 2 : 16};
    const cuuint32_t box[4] = {64, 1, kRows, 1}, step[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, v.data, extent, strides, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? OMNI_OK : context_launched(ctx, int(cudaErrorInvalidValue));
}

int check_shape(const omni_attn *a)
{
    if (!a) return OMNI_ERR_NULL;
    if (a->batch < 0 || a->q_len < 0 || a->kv_len < 0 || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads != 0)
        return OMNI_ERR_BAD_CONFIG;
    if (a->dim < 8 || a->dim % 8 != 0 || !(a->scale > 0.0f) || !std::isfinite(a->scale)) return OMNI_ERR_BAD_CONFIG;
    if (a->dim > OMNI_ATTN_MAX_DIM || a->batch > 65535 || a->heads > 65535 || a->q_len > (1 << 30) || a->kv_len > (1 << 30))
        return OMNI_ERR_TOO_LARGE;
    const int64_t rows = a->q_len > a->kv_len ? a->q_len : a->kv_len;
    if ((rows / kRows + 1) * a->heads * a->batch >= (1ll << 30)) return OMNI_ERR_TOO_LARGE;      // blocks of a launch
    if (!aligned(a->q_lengths, 4) || !aligned(a->kv_lengths, 4)) return OMNI_ERR_ALIGN;
    return OMNI_OK;
}

// A tensor of `len` rows per sequence: present, 16-byte aligned, strides of whole 16 bytes within what a tensor map takes.
int check_view(const omni_attn_view *v, int dim, int heads, int len, int batch)
{
    if (!v) return OMNI_ERR_NULL;
    if (len == 0 || batch == 0) return OMNI_OK;
    if (!v->data) return OMNI_ERR_NULL;
    if (!aligned(v->data, 16)) return OMNI_ERR_ALIGN;
    const uint64_t strides[3] = {v->head, v->row, v->batch};
    const int extents[3] = {heads, len, batch};
    for (int i = 0; i < 3; ++i) {
        if (extents[i] == 1) continue;
        if (strides[i] % 8 != 0) return OMNI_ERR_ALIGN;
        if (strides[i] < uint64_t(dim)) return OMNI_ERR_BAD_CONFIG;
        if (strides[i] >= (1ull << 38)) return OMNI_ERR_TOO_LARGE;
    }
    return OMNI_OK;
}

AttnShape shape_of(const omni_attn *a)
{
    return {a->batch, a->heads, a->kv_heads, a->dim, a->q_len, a->kv_len, a->causal != 0, a->scale, a->q_lengths, a->kv_lengths};
}
OutView out_of(const omni_attn_view *v)
{
    return {static_cast<__nv_bfloat16 *>(v->data), (long long)v->batch, (long long)v->row, (long long)v->head};
}

// One launch of a kernel that takes its parameter block by value, with its shared memory opted in.
// `after`: it begins while the call's previous kernel ends.
template <typename P>
int launch(omni_ctx *ctx, void (*kernel)(P), dim3 grid, int threads, int smem, cudaStream_t s, const P &p, const ContextDevice *after = nullptr)
{
    const void *fn = reinterpret_cast<const void *>(kernel);
    int rc = context_shared(ctx, fn, smem);
    if (rc != OMNI_OK) return rc;
    void *args[] = {const_cast<P *>(&p)};
    if (!after) return context_launched(ctx, int(cudaLaunchKernel(fn, grid, dim3(threads), args, smem, s)));
    const Dependent d(*after, grid, threads, smem, s);
    return context_launched(ctx, int(cudaLaunchKernelExC(&d.cfg, fn, args)));
}

// Blocks per tile: where the tiles do not fill half of the SMs (148), the walks along the other axis, `steps` tiles long at
// most, are dealt out until they fill them all once, two steps a block at least.  Whole walks against dealt out, us a call:
// one query on 8192 keys, 8 heads on 1, forward 113.7 / 26.8, backward 84.2 / 36.0; 4096 x 4096, 2 heads on 1, causal 63.3 / 30.8
// and 116.2 / 45.1; 1025 queries on 11 keys, 8 heads on 2, three sequences, backward 68.0 / 28.8.  Below eight steps the
// joining kernel costs more than it gives (512 x 512, 8 heads: forward 15.3 / 19.5), and so does dealing out from a tile
// per SM on or filling the SMs twice (777 x 777, 12 heads on 4, two sequences: forward 18.5 / 33.1; 256 x 8192: 30.8 / 45.1).
// The rule looks at the number of tiles, not at the longest walk: a padded batch whose one long sequence keeps an SM busy after the
// others are done is not dealt out (6 x 777, 12 heads on 4 of 80, backward, every walk in parts and joined: 68 against 53 us).
int splits_of(int64_t tiles, int64_t steps)
{
    if (tiles < 1 || 2 * tiles > kSms || steps < 8) return 1;
    const int64_t fill = kSms / tiles, most = steps / 2;
    return int(fill < most ? fill : most);
}
int64_t row_tiles(int64_t rows, int tile = kRows) { return (rows + tile - 1) / tile; }
int forward_splits(const omni_attn *a)
{
    return splits_of(row_tiles(a->q_len, 2 * kRows) * a->heads * a->batch, row_tiles(a->kv_len));
}
int query_splits(const omni_attn *a) { return splits_of(row_tiles(a->q_len) * a->heads * a->batch, row_tiles(a->kv_len)); }
int key_splits(const omni_attn *a)
{
    return splits_of(row_tiles(a->kv_len) * a->kv_heads * a->batch, row_tiles(a->q_len) * (a->heads / a->kv_heads));
}
// Floats of the parts, and what describes them; `at` moves on behind them.
uint64_t part_floats(int splits, const omni_attn *a, int len, int heads)
{
    return splits > 1 ? uint64_t(splits) * a->batch * len * heads * a->dim : 0;
}
Parts take_parts(float *&at, int splits, const omni_attn *a, int len, int heads)
{
    const Parts p = {splits, at, (long long)a->batch * len * heads, len, heads};
    at += part_floats(splits, a, len, heads);
    return p;
}
int q_pad_of(const omni_attn *a) { return int(round_up(uint64_t(a->q_len), kRows)); }

}  // namespace
}  // namespace omni

using namespace omni;

extern "C" {

int omni_attn_forward(omni_ctx *ctx, const omni_attn *a, const omni_attn_view *q, const omni_attn_view *k,
                      const omni_attn_view *v, const omni_attn_view *out, float *lse, void *workspace, uint64_t workspace_bytes,
                      void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_shape(a);
    if (rc != OMNI_OK) return rc;
    const omni_attn_view *qs[2] = {q, out}, *ks[2] = {k, v};
    for (const omni_attn_view *x : qs)
        if ((rc = check_view(x, a->dim, a->heads, a->q_len, a->batch)) != OMNI_OK) return rc;
    for (const omni_attn_view *x : ks)
        if ((rc = check_view(x, a->dim, a->kv_heads, a->kv_len, a->batch)) != OMNI_OK) return rc;
    if (a->q_len > 0 && a->batch > 0 && !lse) return OMNI_ERR_NULL;
    uint64_t need = 0;
    if ((rc = omni_attn_forward_workspace(a, &need)) != OMNI_OK) return rc;
    if (need > 0 && !workspace) return OMNI_ERR_NULL;
    if (!aligned(lse, 4) || !aligned(workspace, 16)) return OMNI_ERR_ALIGN;
    if (workspace_bytes < need) return OMNI_ERR_TOO_LARGE;
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK || a->q_len == 0 || a->batch == 0) return rc;
    EncodeTiled encode;
    if ((rc = encoder(ctx, &encode)) != OMNI_OK) return rc;
    AttnForwardParams p;
    std::memset(&p, 0, sizeof p);
    if ((rc = make_map(ctx, encode, &p.q, *q, a->dim, a->heads, a->q_len, a->batch)) != OMNI_OK) return rc;
    if (a->kv_len > 0) {      // without keys no kernel touches their maps
        if ((rc = make_map(ctx, encode, &p.k, *k, a->dim, a->kv_heads, a->kv_len, a->batch)) != OMNI_OK) return rc;
        if ((rc = make_map(ctx, encode, &p.v, *v, a->dim, a->kv_heads, a->kv_len, a->batch)) != OMNI_OK) return rc;
    }
    p.s = shape_of(a);
    p.out = out_of(out);
    p.lse = lse;
    p.status = dev.status;
    p.q_tiles = (a->q_len + 2 * kRows - 1) / (2 * kRows);
    float *at = static_cast<float *>(workspace);
    p.parts = take_parts(at, forward_splits(a), a, a->q_len, a->heads);
    p.part_lse = at;
    const dim3 grid(unsigned(p.q_tiles) * a->heads * a->batch * p.parts.splits);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = a->dim <= 64 ? launch(ctx, attention_forward_kernel<64>, grid, kForwardThreads, ForwardShared<64>::kBytes, s, p)
                      : launch(ctx, attention_forward_kernel<128>, grid, kForwardThreads, ForwardShared<128>::kBytes, s, p);
    if (rc != OMNI_OK || p.parts.splits == 1) return rc;
    return launch(ctx, attention_forward_join_kernel, dim3(unsigned((p.parts.rows * (a->dim / 8) + 255) / 256)), 256, 0, s, p, &dev);
}

int omni_attn_forward_workspace(const omni_attn *a, uint64_t *bytes)
{
    if (!bytes) return OMNI_ERR_NULL;
    const int rc = check_shape(a);
    if (rc != OMNI_OK) return rc;
    const int splits = forward_splits(a);
    *bytes = splits > 1 ? (part_floats(splits, a, a->q_len, a->heads) + uint64_t(splits) * a->batch * a->heads * a->q_len) * sizeof(float) : 0;
    return OMNI_OK;
}

int omni_attn_workspace(const omni_attn *a, uint64_t *bytes)
{
    if (!bytes) return OMNI_ERR_NULL;
    const int rc = check_shape(a);
    if (rc != OMNI_OK) return rc;
    *bytes = (2ull * a->batch * a->heads * q_pad_of(a) + part_floats(query_splits(a), a, a->q_len, a->heads) +
              2 * part_floats(key_splits(a), a, a->kv_len, a->kv_heads)) * sizeof(float);
    return OMNI_OK;
}

int omni_attn_backward(omni_ctx *ctx, const omni_attn *a, const omni_attn_view *q, const omni_attn_view *k,
                       const omni_attn_view *v, const omni_attn_view *out, const float *lse, const omni_attn_view *dout,
                       const omni_attn_view *dq, const omni_attn_view *dk, const omni_attn_view *dv, void *workspace,
                       uint64_t workspace_bytes, void *stream)
{
    if (!ctx) return OMNI_ERR_NULL;
    int rc = check_shape(a);
    if (rc != OMNI_OK) return rc;
    const omni_attn_view *qs[4] = {q, out, dout, dq}, *ks[4] = {k, v, dk, dv};
    for (const omni_attn_view *x : qs)
        if ((rc = check_view(x, a->dim, a->heads, a->q_len, a->batch)) != OMNI_OK) return rc;
    for (const omni_attn_view *x : ks)
        if ((rc = check_view(x, a->dim, a->kv_heads, a->kv_len, a->batch)) != OMNI_OK) return rc;
    uint64_t need = 0;
    rc = omni_attn_workspace(a, &need);
    if (rc != OMNI_OK) return rc;
    if (need > 0 && (!lse || !workspace)) return OMNI_ERR_NULL;
    if (!aligned(lse, 4) || !aligned(workspace, 16)) return OMNI_ERR_ALIGN;
    if (workspace_bytes < need) return OMNI_ERR_TOO_LARGE;
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK || a->batch == 0 || (a->q_len == 0 && a->kv_len == 0)) return rc;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int q_pad = q_pad_of(a);

    AttnBackwardParams p;
    std::memset(&p, 0, sizeof p);
    p.s = shape_of(a);
    p.row_lse = static_cast<float *>(workspace);
    p.row_delta = p.row_lse + uint64_t(a->batch) * a->heads * q_pad;
    p.q_pad = q_pad;
    p.q_tiles = q_pad / kRows;
    p.dq = out_of(dq);
    p.dk = out_of(dk);
    p.dv = out_of(dv);
    p.status = dev.status;
    if (a->q_len > 0) {
        const AttnRowsParams r = {p.s, out_of(out), out_of(dout), lse, const_cast<float *>(p.row_lse),
                                  const_cast<float *>(p.row_delta), q_pad, dev.overlap};
        rc = launch(ctx, attention_rows_kernel, dim3(q_pad / 16, a->heads, a->batch), 256, 0, s, r);
        if (rc != OMNI_OK) return rc;
    }
    EncodeTiled encode;
    if ((rc = encoder(ctx, &encode)) != OMNI_OK) return rc;
    if (a->q_len > 0 && a->kv_len > 0) {         // without a pair of a query and a key no kernel touches the maps
        const struct { CUtensorMap *map; const omni_attn_view *view; int heads, len; } maps[4] = {
            {&p.q, q, a->heads, a->q_len}, {&p.dout, dout, a->heads, a->q_len},
            {&p.k, k, a->kv_heads, a->kv_len}, {&p.v, v, a->kv_heads, a->kv_len}};
        for (const auto &m : maps)
            if ((rc = make_map(ctx, encode, m.map, *m.view, a->dim, m.heads, m.len, a->batch)) != OMNI_OK) return rc;
    }
    float *at = static_cast<float *>(workspace) + 2ull * a->batch * a->heads * q_pad;
    p.parts_dq = take_parts(at, query_splits(a), a, a->q_len, a->heads);
    p.parts_dk = take_parts(at, key_splits(a), a, a->kv_len, a->kv_heads);
    p.parts_dv = take_parts(at, key_splits(a), a, a->kv_len, a->kv_heads);
    p.key_blocks = int(row_tiles(a->kv_len)) * a->kv_heads * a->batch * p.parts_dk.splits;
    const dim3 grid(unsigned(p.key_blocks) + unsigned(p.q_tiles) * a->heads * a->batch * p.parts_dq.splits);
    rc = a->dim <= 64 ? launch(ctx, attention_backward_kernel<64>, grid, kBackwardThreads, BackwardShared<64>::kBytes, s, p, a->q_len > 0 ? &dev : nullptr)
                      : launch(ctx, attention_backward_kernel<128>, grid, kBackwardThreads, BackwardShared<128>::kBytes, s, p, a->q_len > 0 ? &dev : nullptr);
    const int64_t rows = (p.parts_dq.splits > 1 ? p.parts_dq.rows : 0) + (p.parts_dk.splits > 1 ? 2 * p.parts_dk.rows : 0);
    if (rc != OMNI_OK || rows == 0) return rc;
    return launch(ctx, attention_backward_join_kernel, dim3(unsigned((rows * (a->dim / 8) + 255) / 256)), 256, 0, s, p, &dev);
}

}  // extern "C"
