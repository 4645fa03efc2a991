// Attention, backward.  With L the kept log-sum-exp and D_i = sum over columns of dO_i O_i:
//   P = exp(scale Q K^T - L), dP = dO V^T, dS = P (dP - D)
//   dV = P^T dO, dK = scale dS^T Q, dQ = scale dS K
// P and dP are computed again, twice: once by the owner of a key tile, which adds up dK and dV over
// the queries (and over the query heads that share the key head), and once by the owner of a query
// tile, which adds up dQ over the keys.  Seven products instead of five, but every sum has one owner and one order:
// no float atomics, no zeroed and re-read dQ in float, the same bits from the same call.
//
// Both kernels work on 128 x 64 pieces.  Two pairs of warpgroups take the pieces in turn, a thread per 32
// columns of a row, while the tensor core works on the pieces before and after.
//   dK, dV: S^T = K Q^T and dP^T = V dO^T (128 keys x 64 queries).  P^T goes back to tensor memory over
//     S^T as the A operand of dV += P^T dO; dS^T goes to shared memory as that of dK += dS^T Q.
//   dQ:     S = Q K^T and dP = dO V^T (128 queries x 64 keys); dS over S as the A operand of dQ += dS K.
// P and dS are rounded to bfloat16 for the products; all sums are float.
//
// Warps 0-7 and 8-15: pieces in turn (the first four of each the first 32 columns), 16: loads, 17: MMA.
#pragma once
#include <type_traits>

#include "attention.cuh"

namespace omni {

constexpr int kBackwardThreads = 576;
constexpr int kLoadWarp = 16, kMmaWarp = 17;
constexpr int kHalf = 32;           // columns of a thread
constexpr int kPiece = 64;

struct AttnBackwardParams {
    CUtensorMap q, k, v, dout;      // boxes of 128 rows for the operands a block keeps, of 64 for those it streams
    AttnShape s;
    const float *row_lse, *row_delta;   // [batch * heads][q_pad]: -L in powers of two (-inf: no row), -D
    int q_pad, q_tiles;
    OutView dq, dk, dv;
    unsigned *status;
};

struct AttnRowsParams {
    AttnShape s;
    OutView out, dout;
    const float *lse;
    float *row_lse, *row_delta;
    int q_pad;
};

// -D and minus the log-sum-exp in powers of two, for every query row and the padding up to whole tiles.
// 16 lanes a row.  Reads O and dO once.
__global__ void __launch_bounds__(256) attention_rows_kernel(const AttnRowsParams p)
{
    const int lane = threadIdx.x % 16, i = blockIdx.x * 16 + threadIdx.x / 16, head = blockIdx.y, b = blockIdx.z;
    const int q_length = p.s.q_lengths ? min(max(p.s.q_lengths[b], 0), p.s.q_len) : p.s.q_len;
    float sum = 0.0f;
    if (i < q_length)
        for (int c = lane * 8; c < p.s.dim; c += 128) {
            float o[8], d[8];
            const __nv_bfloat16 *po = p.out.data + b * p.out.batch + (long long)i * p.out.row + head * p.out.head + c;
            const __nv_bfloat16 *pd = p.dout.data + b * p.dout.batch + (long long)i * p.dout.row + head * p.dout.head + c;
            widen(*reinterpret_cast<const uint4 *>(po), o);
            widen(*reinterpret_cast<const uint4 *>(pd), d);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(o[e], d[e], sum);
        }
    for (int o = 8; o > 0; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane != 0) return;
    const long long at = ((long long)b * p.s.heads + head) * p.q_pad + i;
    const float lse = i < q_length ? p.lse[((long long)b * p.s.heads + head) * p.s.q_len + i] : -INFINITY;
    const bool there = lse != -INFINITY;
    p.row_lse[at] = there ? -lse * kAttnLog2e : -INFINITY;
    p.row_delta[at] = there ? -sum : 0.0f;
}

// ---- dK, dV -------------------------------------------------------------------------------------

template <int DP> struct KeysShared {
    static constexpr int kStages = 4;
    static constexpr int kTile = kRows * DP * 2, kPieceTile = kPiece * DP * 2, kDs = kRows * kPiece * 2;
    static constexpr int kK = 0, kV = kTile, kQ = 2 * kTile, kDo = kQ + kStages * kPieceTile, kS = kDo + kStages * kPieceTile;
    static constexpr int kStats = kS + 2 * kDs;                    // [stages][2][64] float
    static constexpr int kBars = kStats + kStages * 2 * kPiece * 4;
    // barriers, and what is left of the block's 227 KB for rounding the base up to 1024
    static constexpr int kBytes = kBars + 256 + (DP == 128 ? 768 : 1024);
    static_assert(kBytes <= 227 * 1024, "shared memory of a block");
};

template <int DP>
__global__ void __launch_bounds__(kBackwardThreads, 1) attention_keys_kernel(const __grid_constant__ AttnBackwardParams p)
{
    using L = KeysShared<DP>;
    constexpr int ST = L::kStages;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(smem + L::kBars);
    unsigned long long *kv_full = bars, *full = bars + 1, *empty = full + ST, *s_full = empty + ST, *ds_ready = s_full + 2;
    unsigned long long *done = ds_ready + 2;
    volatile int *give_up = reinterpret_cast<int *>(done + 1);
    unsigned *tmem_cell = reinterpret_cast<unsigned *>(done + 2);
    const float *stats = reinterpret_cast<const float *>(smem + L::kStats);

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Place at_tile = place_of(p.s.kv_heads, p.s.batch);
    const int kv_head = at_tile.head, b = at_tile.batch, group = p.s.heads / p.s.kv_heads;
    const int k0 = at_tile.tile * kRows;
    const Lengths len = lengths_of(p.s, b);

    // query pieces that see some key of this tile: from the one with the first row i >= k0 - shift
    const int first_row = p.s.causal ? max(0, k0 - len.shift) : 0;
    const int piece0 = first_row / kPiece;
    const int pieces = k0 < len.kv && first_row < len.q ? (len.q + kPiece - 1) / kPiece - piece0 : 0;
    const int n = pieces * group;

    if (threadIdx.x == 0) {
        mbar_init(kv_full, 1);
        for (int i = 0; i < ST; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int t = 0; t < 2; ++t) { mbar_init(s_full + t, 1); mbar_init(ds_ready + t, 2 * kRows); }
        mbar_init(done, 1);
        *give_up = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) tmem_alloc(tmem_cell, 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const unsigned tmem = *tmem_cell;
    const unsigned dv_at = tmem, dk_at = tmem + DP, s_at = tmem + 2 * DP, dp_at = s_at + 2 * kPiece;

    if (warp == kLoadWarp) {
        if (lane == 0 && n > 0) {
            prefetch_map(&p.q); prefetch_map(&p.k); prefetch_map(&p.v); prefetch_map(&p.dout);
            mbar_expect_tx(kv_full, 2 * L::kTile);
            load_tile<DP, kRows>(smem + L::kK, &p.k, kv_head, k0, b, kv_full);
            load_tile<DP, kRows>(smem + L::kV, &p.v, kv_head, k0, b, kv_full);
            int armed = 0;
            const unsigned long long policy = policy_evict_last();
            for (int h = 0; h < n; ++h) {
                const int st = h % ST, head = kv_head * group + h / pieces, row = (piece0 + h % pieces) * kPiece;
                if (!bounded_wait(empty + st, ((h / ST) & 1) ^ 1, give_up, p.status)) break;
                mbar_expect_tx(full + st, 2 * L::kPieceTile + 2 * kPiece * 4);
                load_tile<DP, kPiece>(smem + L::kQ + st * L::kPieceTile, &p.q, head, row, b, full + st);
                load_tile<DP, kPiece>(smem + L::kDo + st * L::kPieceTile, &p.dout, head, row, b, full + st);
                const long long at = ((long long)b * p.s.heads + head) * p.q_pad + row;
                float *to = reinterpret_cast<float *>(smem + L::kStats) + st * 2 * kPiece;
                bulk_load(to, p.row_lse + at, kPiece * 4, full + st, policy);
                bulk_load(to + kPiece, p.row_delta + at, kPiece * 4, full + st, policy);
                ++armed;
            }
            mbar_wait(kv_full, 0);
            for (int h = max(0, armed - ST); h < armed; ++h) mbar_wait(full + h % ST, (h / ST) & 1);
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        const unsigned k = smem_addr(smem + L::kK), v = smem_addr(smem + L::kV), ds = smem_addr(smem + L::kS);
        bool ok = n == 0 || warp_wait(kv_full, 0, give_up, p.status);
        // scores of piece h into its half of tensor memory
        auto scores = [&](int h) {
            const int st = h % ST, row = (piece0 + h % pieces) * kPiece;
            const bool w = warp_wait(full + st, (h / ST) & 1, give_up, p.status);
            if (!w) return false;
            if (p.s.q_lengths && len.q - row < kPiece) {
                zero_rows<DP, kPiece>(smem + L::kQ + st * L::kPieceTile, len.q - row);
                zero_rows<DP, kPiece>(smem + L::kDo + st * L::kPieceTile, len.q - row);
            }
            fence_after_sync();
            if (lane == 0) {
                const unsigned q = smem_addr(smem + L::kQ + st * L::kPieceTile), d = smem_addr(smem + L::kDo + st * L::kPieceTile);
                mma_along<DP, kRows, kPiece, kPiece>(s_at + (h & 1) * kPiece, k, q, false);
                mma_along<DP, kRows, kPiece, kPiece>(dp_at + (h & 1) * kPiece, v, d, false);
                mma_commit(s_full + (h & 1));
            }
            __syncwarp();
            return true;
        };
        for (int h = 0; h < 2 && h < n && ok; ++h) ok = scores(h);
        for (int h = 0; h < n && ok; ++h) {
            const int st = h % ST, t = h & 1;
            ok = warp_wait(ds_ready + t, (h / 2) & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            if (lane == 0) {
                const unsigned q = smem_addr(smem + L::kQ + st * L::kPieceTile), d = smem_addr(smem + L::kDo + st * L::kPieceTile);
                mma_tmem_across<DP, kPiece, kPiece, kHalf>(dv_at, s_at + t * kPiece, d, h > 0);
#pragma unroll
                for (int s = 0; s < kPiece / 16; ++s)
                    mma_ss(dk_at, tile_desc(ds + t * L::kDs + s * 32, 1024, 16), tile_desc(q + s * 2048, 1024, kPiece * 128),
                           mma_kind(DP, false, true), h > 0 || s > 0);
                mma_commit(empty + st);
            }
            __syncwarp();
            if (h + 2 < n) ok = scores(h + 2);     // over P of piece h: MMAs run in the order of issue
        }
        if (lane == 0) {
            mma_commit(done);
            mbar_wait(done, 0);
        }
        __syncwarp();
    } else {
        const int t = warp / 8, half = warp / 4 % 2, row = threadIdx.x % kRows, j = k0 + row;
        const unsigned lanes = unsigned(warp % 4) * 32u << 16;
        const unsigned s_row = s_at + t * kPiece + half * kHalf + lanes, dp_row = dp_at + t * kPiece + half * kHalf + lanes;
        const float2 unit = {p.s.scale * kAttnLog2e, p.s.scale * kAttnLog2e};
        // queries that see this key: i >= from
        const int from = j >= len.kv ? INT_MAX : p.s.causal ? j - len.shift : 0;
        unsigned char *ds_row = smem + L::kS + t * L::kDs + row * 128;
        bool ok = true;
        for (int h = t; h < n; h += 2) {
            const int st = h % ST, i0 = (piece0 + h % pieces) * kPiece + half * kHalf;
            ok = warp_wait(s_full + t, (h / 2) & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            const float4 *lse = reinterpret_cast<const float4 *>(stats + st * 2 * kPiece + half * kHalf);
            const float4 *delta = lse + kPiece / 4;
            uint32_t s[kHalf], dp[kHalf], pk[kHalf / 2], dk[kHalf / 2];
            tmem_load2(s, s_row, dp, dp_row);
            auto piece = [&](auto edge) {
#pragma unroll
                for (int c = 0; c < kHalf; c += 4) {
                    const float4 l = lse[c / 4], d = delta[c / 4];
                    const float2 x0 = fma2({__uint_as_float(s[c]), __uint_as_float(s[c + 1])}, unit, {l.x, l.y});
                    const float2 x1 = fma2({__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])}, unit, {l.z, l.w});
                    float2 p0 = {exp2_fast(x0.x), exp2_fast(x0.y)}, p1 = {exp2_fast(x1.x), exp2_fast(x1.y)};
                    float2 d0 = mul2(p0, add2({__uint_as_float(dp[c]), __uint_as_float(dp[c + 1])}, {d.x, d.y}));
                    float2 d1 = mul2(p1, add2({__uint_as_float(dp[c + 2]), __uint_as_float(dp[c + 3])}, {d.z, d.w}));
                    if constexpr (decltype(edge)::value) {
                        if (i0 + c < from) p0.x = d0.x = 0.0f;
                        if (i0 + c + 1 < from) p0.y = d0.y = 0.0f;
                        if (i0 + c + 2 < from) p1.x = d1.x = 0.0f;
                        if (i0 + c + 3 < from) p1.y = d1.y = 0.0f;
                    }
                    pk[c / 2] = pack2(p0.x, p0.y);
                    pk[c / 2 + 1] = pack2(p1.x, p1.y);
                    dk[c / 2] = pack2(d0.x, d0.y);
                    dk[c / 2 + 1] = pack2(d1.x, d1.y);
                }
            };
            if (__any_sync(~0u, from > i0)) piece(std::true_type{});
            else piece(std::false_type{});
            tmem_store(s_row, pk);
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<uint4 *>(ds_row + (((half * 4 + g) ^ (row & 7)) * 16)) =
                    make_uint4(dk[g * 4], dk[g * 4 + 1], dk[g * 4 + 2], dk[g * 4 + 3]);
            tmem_wait_store();
            fence_async_proxy();
            fence_before_sync();
            mbar_arrive(ds_ready + t);
        }
        // warps 0-7 write dV, warps 8-15 dK, half of the columns each four
        if (n > 0 && ok) ok = warp_wait(done, 0, give_up, p.status);
        ok = __all_sync(~0u, ok && *give_up == 0);
        fence_after_sync();
        const OutView &o = t == 0 ? p.dv : p.dk;
        const int c0 = half * (DP / 2);
        __nv_bfloat16 *dst = o.data + b * o.batch + (long long)j * o.row + kv_head * o.head;
        const bool mine = ok && j < p.s.kv_len;
        if (n > 0 && ok)
            store_row<DP / 2>((t == 0 ? dv_at : dk_at) + lanes + c0, t == 0 ? 1.0f : p.s.scale, dst + c0, p.s.dim - c0, mine);
        else if (mine && half == 0)
            store_zeros(dst, p.s.dim);
    }
    fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) tmem_free(tmem, 512);
}

// ---- dQ -----------------------------------------------------------------------------------------

template <int DP> struct QueriesShared {
    static constexpr int kStages = 4;
    static constexpr int kTile = kRows * DP * 2, kPieceTile = kPiece * DP * 2;
    static constexpr int kQ = 0, kDo = kTile, kK = 2 * kTile, kV = kK + kStages * kPieceTile;
    static constexpr int kBars = kV + kStages * kPieceTile;
    static constexpr int kBytes = kBars + 256 + 1024;
};

template <int DP>
__global__ void __launch_bounds__(kBackwardThreads, 1) attention_queries_kernel(const __grid_constant__ AttnBackwardParams p)
{
    using L = QueriesShared<DP>;
    constexpr int ST = L::kStages;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(smem + L::kBars);
    unsigned long long *q_full = bars, *full = bars + 1, *empty = full + ST, *s_full = empty + ST, *ds_ready = s_full + 2;
    unsigned long long *done = ds_ready + 2;
    volatile int *give_up = reinterpret_cast<int *>(done + 1);
    unsigned *tmem_cell = reinterpret_cast<unsigned *>(done + 2);

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Place at_tile = place_of(p.s.heads, p.s.batch);
    const int head = at_tile.head, b = at_tile.batch, kv_head = head / (p.s.heads / p.s.kv_heads);
    const int q0 = (p.q_tiles - 1 - at_tile.tile) * kRows;
    const Lengths len = lengths_of(p.s, b);
    const int last = min(q0 + kRows, len.q) - 1;
    const int seen = last < q0 ? 0 : p.s.causal ? min(len.kv, last + len.shift + 1) : len.kv;
    const int n = seen > 0 ? (seen + kPiece - 1) / kPiece : 0;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int i = 0; i < ST; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int t = 0; t < 2; ++t) { mbar_init(s_full + t, 1); mbar_init(ds_ready + t, 2 * kRows); }
        mbar_init(done, 1);
        *give_up = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) tmem_alloc(tmem_cell, 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const unsigned tmem = *tmem_cell;
    const unsigned dq_at = tmem, s_at = tmem + DP, dp_at = s_at + 2 * kPiece;

    if (warp == kLoadWarp) {
        if (lane == 0 && n > 0) {
            prefetch_map(&p.q); prefetch_map(&p.k); prefetch_map(&p.v); prefetch_map(&p.dout);
            mbar_expect_tx(q_full, 2 * L::kTile);
            load_tile<DP, kRows>(smem + L::kQ, &p.q, head, q0, b, q_full);
            load_tile<DP, kRows>(smem + L::kDo, &p.dout, head, q0, b, q_full);
            int armed = 0;
            for (int h = 0; h < n; ++h) {
                const int st = h % ST;
                if (!bounded_wait(empty + st, ((h / ST) & 1) ^ 1, give_up, p.status)) break;
                mbar_expect_tx(full + st, 2 * L::kPieceTile);
                load_tile<DP, kPiece>(smem + L::kK + st * L::kPieceTile, &p.k, kv_head, h * kPiece, b, full + st);
                load_tile<DP, kPiece>(smem + L::kV + st * L::kPieceTile, &p.v, kv_head, h * kPiece, b, full + st);
                ++armed;
            }
            mbar_wait(q_full, 0);
            for (int h = max(0, armed - ST); h < armed; ++h) mbar_wait(full + h % ST, (h / ST) & 1);
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        const unsigned q = smem_addr(smem + L::kQ), d = smem_addr(smem + L::kDo);
        bool ok = n == 0 || warp_wait(q_full, 0, give_up, p.status);
        auto scores = [&](int h) {
            const int st = h % ST;
            const bool w = warp_wait(full + st, (h / ST) & 1, give_up, p.status);
            if (!w) return false;
            if (p.s.kv_lengths && len.kv - h * kPiece < kPiece)
                zero_rows<DP, kPiece>(smem + L::kK + st * L::kPieceTile, len.kv - h * kPiece);
            fence_after_sync();
            if (lane == 0) {
                const unsigned k = smem_addr(smem + L::kK + st * L::kPieceTile), v = smem_addr(smem + L::kV + st * L::kPieceTile);
                mma_along<DP, kRows, kPiece, kPiece>(s_at + (h & 1) * kPiece, q, k, false);
                mma_along<DP, kRows, kPiece, kPiece>(dp_at + (h & 1) * kPiece, d, v, false);
                mma_commit(s_full + (h & 1));
            }
            __syncwarp();
            return true;
        };
        for (int h = 0; h < 2 && h < n && ok; ++h) ok = scores(h);
        for (int h = 0; h < n && ok; ++h) {
            const int st = h % ST, t = h & 1;
            ok = warp_wait(ds_ready + t, (h / 2) & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            if (lane == 0) {
                mma_tmem_across<DP, kPiece, kPiece, kHalf>(dq_at, s_at + t * kPiece, smem_addr(smem + L::kK + st * L::kPieceTile), h > 0);
                mma_commit(empty + st);
            }
            __syncwarp();
            if (h + 2 < n) ok = scores(h + 2);     // over dS of piece h: MMAs run in the order of issue
        }
        if (lane == 0) {
            mma_commit(done);
            mbar_wait(done, 0);
        }
        __syncwarp();
    } else {
        const int t = warp / 8, half = warp / 4 % 2, row = threadIdx.x % kRows, i = q0 + row;
        const unsigned lanes = unsigned(warp % 4) * 32u << 16;
        const unsigned s_row = s_at + t * kPiece + half * kHalf + lanes, dp_row = dp_at + t * kPiece + half * kHalf + lanes;
        const float2 unit = {p.s.scale * kAttnLog2e, p.s.scale * kAttnLog2e};
        const int limit = i >= len.q ? 0 : p.s.causal ? min(len.kv, i + len.shift + 1) : len.kv;
        const long long at = ((long long)b * p.s.heads + head) * p.q_pad + i;
        const float lse = p.row_lse[at], delta = p.row_delta[at];
        bool ok = true;
        for (int h = t; h < n; h += 2) {
            ok = warp_wait(s_full + t, (h / 2) & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            const int open = limit - h * kPiece - half * kHalf;
            uint32_t s[kHalf], dp[kHalf], pk[kHalf / 2];
            tmem_load2(s, s_row, dp, dp_row);
            auto piece = [&](auto edge) {
#pragma unroll
                for (int c = 0; c < kHalf; c += 2) {
                    const float2 x = fma2({__uint_as_float(s[c]), __uint_as_float(s[c + 1])}, unit, {lse, lse});
                    const float2 pr = {exp2_fast(x.x), exp2_fast(x.y)};
                    float2 dr = mul2(pr, add2({__uint_as_float(dp[c]), __uint_as_float(dp[c + 1])}, {delta, delta}));
                    if constexpr (decltype(edge)::value) {
                        if (c >= open) dr.x = 0.0f;
                        if (c + 1 >= open) dr.y = 0.0f;
                    }
                    pk[c / 2] = pack2(dr.x, dr.y);
                }
            };
            if (__any_sync(~0u, open < kHalf)) piece(std::true_type{});
            else piece(std::false_type{});
            tmem_store(s_row, pk);
            tmem_wait_store();
            fence_before_sync();
            mbar_arrive(ds_ready + t);
        }
        if (n > 0 && ok) ok = warp_wait(done, 0, give_up, p.status);
        ok = __all_sync(~0u, ok && *give_up == 0);
        fence_after_sync();
        // every warpgroup a quarter of the columns
        const int c0 = (2 * t + half) * (DP / 4);
        __nv_bfloat16 *dst = p.dq.data + b * p.dq.batch + (long long)i * p.dq.row + head * p.dq.head;
        const bool mine = ok && i < p.s.q_len, empty = limit <= 0;
        if (n > 0 && ok) store_row<DP / 4>(dq_at + lanes + c0, p.s.scale, dst + c0, p.s.dim - c0, mine && !empty);
        if (c0 == 0 && mine && empty) store_zeros(dst, p.s.dim);
    }
    fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) tmem_free(tmem, 512);
}

}  // namespace omni
