// Attention, backward.  With L the kept log-sum-exp and D_i = sum over columns of dO_i O_i:
//   P = exp(scale Q K^T - L), dP = dO V^T, dS = P (dP - D)
//   dV = P^T dO, dK = scale dS^T Q, dQ = scale dS K
// P and dP are computed again, twice: once by the owner of a key tile, which adds up dK and dV over
// the queries (and over the query heads that share the key head), and once by the owner of a query
// tile, which adds up dQ over the keys.  Seven products instead of five, but every sum has one owner and one order:
// no float atomics, no zeroed and re-read dQ in float, the same bits from the same call.
//
// Both walk 128 x 128 tiles of S and dP in tensor memory.  (64 columns a tile would leave room for two of each, but an MMA
// m128 n64 k16 with both operands in shared memory takes 48 cycles, n128 64: measured.)  The elementwise work comes in two phases, P from S and dS from P and dP, sixteen warps at 32 columns of a row per thread,
// and each phase runs beside products of the same or the next tile:
//   dK, dV: S^T = K Q^T and dP^T = V dO^T (128 keys x 128 queries).  P^T goes back to tensor memory over S^T as the A
//     operand of dV += P^T dO, dS^T over dP^T as that of dK += dS^T Q.
//     Order of the products: S0 dP0 | dV0 S1 dK0 dP1 | dV1 S2 dK1 dP2 | ...
//   dQ:     S = Q K^T and dP = dO V^T (128 queries x 128 keys), two tiles of S; dS over S as the A operand of dQ += dS K.
//     Order: S0 dP0 S1 | dP1 dQ0 S2 | dP2 dQ1 S3 | ...
// An operand in tensor memory is overwritten by a product that is issued after the one that reads it; one thread
// issues all of a block's, and the tensor core takes them in that order.
// What bounds it: the chain of one tile, S, P, dV and the next S over P, 2900 cycles a step with dK and dV where the four
// products take 2048, and 2200 a step with dQ where the three take 1536; then the power cap.  Measured: 8192 rows, 16 heads on 8 of
// 128, causal, 744 us (924 TFLOP/s at five products) in a burst, where the clock is at 1.73 GHz, and 870 us a call in a
// long run.  By clock stamps, in thousands of cycles an SM: 33280 steps of dK and dV 652 and as many of dQ 494; beside their steps
// 512 blocks of keys, 16 each, 55 and 1024 blocks of queries, 11 each, 77 (set-up 2.3, first loads and scores 3.0-3.7, last product and
// stores 4.0-8.4, on to the next 1.7); mean 1277, busiest SM 1286.
// Where a padded batch leaves few blocks the longest decides: 6 x 777, 12 heads on 4 of 80, causal, lasts the 21 steps that the
// first key tile has to do (three heads, seven query tiles), 77 thousand cycles, 42 of 52 us a call; the mean SM works 33.
// Tried: P and dS through shared memory 1018 against 940 us then; P over dP, so that S is free earlier (Q's copies then come late) 541
// against 455 us of dK, dV; a third place for Q 744 against 747; exponentials by a polynomial 451-472 against 455.
// P and dS are rounded to bfloat16 for the products; all sums are float.
//
// Warps 0-15: elementwise (four warps cover the 128 rows, each four another 32 columns), 16: loads, 17: MMA.
#pragma once
#include "attention.cuh"

namespace omni {

constexpr int kLoadWarp = 16, kMmaWarp = 17, kBackwardThreads = 18 * 32;
constexpr int kElementWarps = 16;
constexpr int kCols = 32;           // columns of a thread

struct AttnBackwardParams {
    CUtensorMap q, k, v, dout;
    AttnShape s;
    const float *row_lse, *row_delta;   // [batch * heads][q_pad]: -L in powers of two (-inf: no row), -D
    int q_pad, q_tiles;
    int key_blocks;                 // blocks that own keys; the others own queries
    OutView dq, dk, dv;
    Parts parts_dq, parts_dk, parts_dv;
    unsigned *status;
};

struct AttnRowsParams {
    AttnShape s;
    OutView out, dout;
    const float *lse;
    float *row_lse, *row_delta;
    int q_pad;
    bool overlap;                   // the next kernel may begin early
};

// -D and minus the log-sum-exp in powers of two, for every query row and the padding up to whole tiles.
// 16 lanes a row.  Reads O and dO once.
__global__ void __launch_bounds__(256) attention_rows_kernel(const AttnRowsParams p)
{
    let_next_begin(p.overlap);
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
    static constexpr int kStages = DP == 128 ? 2 : 3;
    static constexpr int kTile = kRows * DP * 2;
    static constexpr int kK = 0, kV = kTile, kQ = 2 * kTile, kDo = kQ + kStages * kTile;
    static constexpr int kStats = kDo + kStages * kTile;           // [stages][2][128] float
    static constexpr int kBars = kStats + kStages * 2 * kRows * 4;
    static constexpr int kBytes = kBars + 256 + 1024;              // barriers, and the base rounded up to 1024
    static_assert(kBytes <= 227 * 1024, "shared memory of a block");
};

template <int DP> __device__ __forceinline__ void attention_keys(const AttnBackwardParams &p, int block)
{
    using L = KeysShared<DP>;
    constexpr int ST = L::kStages;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(smem + L::kBars);
    unsigned long long *kv_full = bars, *q_full = bars + 1, *q_empty = q_full + ST, *do_full = q_empty + ST, *do_empty = do_full + ST;
    unsigned long long *s_full = do_empty + ST, *p_ready = s_full + 1, *dp_full = p_ready + 1, *ds_ready = dp_full + 1, *done = ds_ready + 1;
    unsigned long long *own = done + 1;
    volatile int *give_up = reinterpret_cast<int *>(own + 1);
    unsigned *tmem_cell = reinterpret_cast<unsigned *>(own + 2);
    const float *stats = reinterpret_cast<const float *>(smem + L::kStats);

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int splits = p.parts_dk.splits;
    const Place at_tile = place_of(block, p.s.kv_heads * splits, p.s.batch);
    const int kv_head = at_tile.head / splits, part = at_tile.head % splits, b = at_tile.batch, group = p.s.heads / p.s.kv_heads;
    const int k0 = at_tile.tile * kRows;
    const Lengths len = lengths_of(p.s, b);

    // query tiles that see some key of this tile: from the one with the first row i >= k0 - shift
    const int first_row = p.s.causal ? max(0, k0 - len.shift) : 0;
    const int tile0 = first_row / kRows;
    const int tiles = k0 < len.kv && first_row < len.q ? (len.q + kRows - 1) / kRows - tile0 : 0;
    int h0, h1;                                                     // this block's steps, (query head, tile) one after the other
    stretch_of(tiles * group, part, splits, &h0, &h1);
    const int n = h1 - h0;
    if (n == 0) {                                                   // no query sees these keys
        wait_for_previous();                                        // a grid that is complete has to mean that both kernels are
        const int rows = min(kRows, p.s.kv_len - k0);
        if (splits > 1) {
            zero_parts(p.parts_dk, part, b, kv_head, k0, rows, p.s.dim);
            zero_parts(p.parts_dv, part, b, kv_head, k0, rows, p.s.dim);
        } else {
            zero_tile(p.dk, b, kv_head, k0, rows, p.s.dim);
            zero_tile(p.dv, b, kv_head, k0, rows, p.s.dim);
        }
        return;
    }

    if (threadIdx.x == 0) {
        mbar_init(kv_full, 1);
        for (int i = 0; i < ST; ++i) {
            mbar_init(q_full + i, 1); mbar_init(q_empty + i, 1);
            mbar_init(do_full + i, 1); mbar_init(do_empty + i, 1);
        }
        mbar_init(s_full, 1); mbar_init(p_ready, kElementWarps);
        mbar_init(dp_full, 1); mbar_init(ds_ready, kElementWarps);
        mbar_init(done, 1); mbar_init(own, 1);
        *give_up = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) tmem_alloc(tmem_cell, 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const unsigned tmem = *tmem_cell;
    const unsigned dv_at = tmem, dk_at = tmem + DP, s_at = tmem + 2 * DP, dp_at = s_at + kRows;

    if (warp == kLoadWarp) {
        Loader load = {own, 0, give_up, p.status};
        if (lane == 0) {
            prefetch_map(&p.q); prefetch_map(&p.k); prefetch_map(&p.v); prefetch_map(&p.dout);
            mbar_expect_tx(kv_full, 2 * L::kTile);
            load_tile<DP>(smem + L::kK, &p.k, kv_head, k0, b, kv_full);
            load_tile<DP>(smem + L::kV, &p.v, kv_head, k0, b, kv_full);
        }
        int q_armed = 0, do_armed = 0;
        const unsigned long long policy = policy_evict_last();
        for (int h = 0; h < n; ++h) {
            const int st = h % ST, head = kv_head * group + (h0 + h) / tiles, row = (tile0 + (h0 + h) % tiles) * kRows;
            const int valid = p.s.q_lengths ? len.q - row : kRows, unseeing = p.s.causal ? -len.shift - row : 0;
            const unsigned free_parity = ((h / ST) & 1) ^ 1;
            if (!load.wait(q_empty + st, free_parity)) break;
            if (!load.tile<DP>(smem + L::kQ + st * L::kTile, &p.q, head, row, b, q_full + st, valid, 2 * kRows * 4, unseeing)) break;
            if (lane == 0) {
                if (h == 0) wait_for_previous();                   // the row values are the previous kernel's
                const long long at = ((long long)b * p.s.heads + head) * p.q_pad + row;
                float *to = reinterpret_cast<float *>(smem + L::kStats) + st * 2 * kRows;
                bulk_load(to, p.row_lse + at, kRows * 4, q_full + st, policy);
                bulk_load(to + kRows, p.row_delta + at, kRows * 4, q_full + st, policy);
            }
            ++q_armed;
            if (!load.wait(do_empty + st, free_parity)) break;
            if (!load.tile<DP>(smem + L::kDo + st * L::kTile, &p.dout, head, row, b, do_full + st, valid, 0, unseeing)) break;
            ++do_armed;
        }
        wait_for_previous();                                       // also when it gave up before the first row values
        // the block may not end with a copy in flight, not even when it gave up
        mbar_wait(kv_full, 0);
        for (int h = max(0, q_armed - ST); h < q_armed; ++h) mbar_wait(q_full + h % ST, (h / ST) & 1);
        for (int h = max(0, do_armed - ST); h < do_armed; ++h) mbar_wait(do_full + h % ST, (h / ST) & 1);
        __syncwarp();
    } else if (warp == kMmaWarp) {
        if (elect_one()) {
            const unsigned k = smem_addr(smem + L::kK), v = smem_addr(smem + L::kV);
            const unsigned q0 = smem_addr(smem + L::kQ), do0 = smem_addr(smem + L::kDo);
            auto wait = [&](unsigned long long *bar, unsigned parity) { return bounded_wait(bar, parity, give_up, p.status); };
            auto scores = [&](int h) {
                const int st = h % ST;
                if (!wait(q_full + st, (h / ST) & 1)) return false;
                fence_after_sync();
                mma_along<DP>(s_at, k, q0 + st * L::kTile);
                mma_commit(s_full);
                return true;
            };
            auto slopes = [&](int h) {
                const int st = h % ST;
                if (!wait(do_full + st, (h / ST) & 1)) return false;
                fence_after_sync();
                mma_along<DP>(dp_at, v, do0 + st * L::kTile);
                mma_commit(dp_full);
                return true;
            };
            bool ok = wait(kv_full, 0) && scores(0) && slopes(0);
            for (int h = 0; h < n && ok; ++h) {
                const int st = h % ST;
                if (!(ok = wait(p_ready, h & 1))) break;
                fence_after_sync();
                mma_tmem_across<DP, kRows, kCols>(dv_at, s_at, do0 + st * L::kTile, h > 0);
                mma_commit(do_empty + st);
                if (h + 1 < n && !(ok = scores(h + 1))) break;
                if (!(ok = wait(ds_ready, h & 1))) break;
                fence_after_sync();
                mma_tmem_across<DP, kRows, kCols>(dk_at, dp_at, q0 + st * L::kTile, h > 0);
                mma_commit(q_empty + st);
                if (h + 1 < n) ok = slopes(h + 1);
            }
            mma_commit(done);
            mbar_wait(done, 0);
        }
        __syncwarp();
    } else {
        const int c0 = warp / 4 * kCols, row = threadIdx.x % kRows, j = k0 + row;
        const unsigned lanes = unsigned(warp % 4) * 32u << 16;
        const unsigned s_row = s_at + c0 + lanes, dp_row = dp_at + c0 + lanes;
        const float2 unit = {p.s.scale * kAttnLog2e, p.s.scale * kAttnLog2e};
        // queries that see this key: i >= from
        const int from = j >= len.kv ? INT_MAX : p.s.causal ? j - len.shift : 0;
        bool ok = true;
        for (int h = 0; h < n; ++h) {
            const int i0 = (tile0 + (h0 + h) % tiles) * kRows + c0;
            const float4 *lse = reinterpret_cast<const float4 *>(stats + h % ST * 2 * kRows + c0), *delta = lse + kRows / 4;
            // the row values came with Q: their copy is waited for here too
            ok = warp_wait(q_full + h % ST, (h / ST) & 1, give_up, p.status) && warp_wait(s_full, h & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            const bool edge = __any_sync(~0u, from > i0);
            uint32_t x[kCols], out[kCols / 2];
            float2 pr[kCols / 2];
            tmem_load(x, s_row);
#pragma unroll
            for (int c = 0; c < kCols; c += 4) {
                const float4 l = lse[c / 4];
                const float2 a = fma2({__uint_as_float(x[c]), __uint_as_float(x[c + 1])}, unit, {l.x, l.y});
                const float2 d = fma2({__uint_as_float(x[c + 2]), __uint_as_float(x[c + 3])}, unit, {l.z, l.w});
                pr[c / 2] = {exp2_fast(a.x), exp2_fast(a.y)};
                pr[c / 2 + 1] = {exp2_fast(d.x), exp2_fast(d.y)};
            }
            if (edge) {
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    if (i0 + c < from) pr[c / 2].x = 0.0f;
                    if (i0 + c + 1 < from) pr[c / 2].y = 0.0f;
                }
            }
#pragma unroll
            for (int c = 0; c < kCols / 2; ++c) out[c] = pack2(pr[c].x, pr[c].y);
            tmem_store(s_row, out);
            tmem_wait_store();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready);

            ok = warp_wait(dp_full, h & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            tmem_load(x, dp_row);
#pragma unroll
            for (int c = 0; c < kCols; c += 4) {
                const float4 d = delta[c / 4];
                const float2 a = mul2(pr[c / 2], add2({__uint_as_float(x[c]), __uint_as_float(x[c + 1])}, {d.x, d.y}));
                const float2 e = mul2(pr[c / 2 + 1], add2({__uint_as_float(x[c + 2]), __uint_as_float(x[c + 3])}, {d.z, d.w}));
                pr[c / 2] = a;
                pr[c / 2 + 1] = e;
            }
            if (edge) {                                             // 0 x NaN would not be 0
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    if (i0 + c < from) pr[c / 2].x = 0.0f;
                    if (i0 + c + 1 < from) pr[c / 2].y = 0.0f;
                }
            }
#pragma unroll
            for (int c = 0; c < kCols / 2; ++c) out[c] = pack2(pr[c].x, pr[c].y);
            tmem_store(dp_row, out);
            tmem_wait_store();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_ready);
        }
        // warps 0-7 write dV, warps 8-15 dK, half of the columns each four
        if (ok) ok = warp_wait(done, 0, give_up, p.status);
        ok = __all_sync(~0u, ok && *give_up == 0);
        fence_after_sync();
        const bool values = warp < 8;
        const OutView &o = values ? p.dv : p.dk;
        const int half = warp / 4 % 2, d0 = half * (DP / 2);
        const unsigned from_tmem = (values ? dv_at : dk_at) + lanes + d0;
        const float gain = values ? 1.0f : p.s.scale;
        // a key behind the length has P = 0 throughout, but a row of dO may hold NaN
        const bool mine = ok && j < p.s.kv_len, seen = j < len.kv;
        const int cols = min(DP / 2, p.s.dim - d0);
        if (splits > 1) {
            float *dst = (values ? p.parts_dv : p.parts_dk).at(part, b, j, kv_head, p.s.dim) + d0;
            if (ok) store_row<DP / 2>(from_tmem, gain, dst, cols, mine && seen);
            if (mine && !seen)
                for (int c = 0; c < cols; ++c) dst[c] = 0.0f;
        } else {
            __nv_bfloat16 *dst = o.data + b * o.batch + (long long)j * o.row + kv_head * o.head + d0;
            if (ok) store_row<DP / 2>(from_tmem, gain, dst, cols, mine && seen);
            if (mine && !seen) store_zeros(dst, cols);
        }
    }
    fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) tmem_free(tmem, 512);
}

// ---- dQ -----------------------------------------------------------------------------------------

template <int DP> struct QueriesShared {
    static constexpr int kKStages = 3, kVStages = 2;
    static constexpr int kTile = kRows * DP * 2;
    static constexpr int kQ = 0, kDo = kTile, kK = 2 * kTile, kV = kK + kKStages * kTile;
    static constexpr int kBars = kV + kVStages * kTile;
    static constexpr int kBytes = kBars + 256 + 1024;      // barriers, and the base rounded up to 1024
    static_assert(kBytes <= 227 * 1024, "shared memory of a block");
};

template <int DP> __device__ __forceinline__ void attention_queries(const AttnBackwardParams &p, int block)
{
    using L = QueriesShared<DP>;
    constexpr int KS = L::kKStages, VS = L::kVStages;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(smem + L::kBars);
    unsigned long long *q_full = bars, *k_full = bars + 1, *k_empty = k_full + KS, *v_full = k_empty + KS, *v_empty = v_full + VS;
    unsigned long long *s_full = v_empty + VS, *dp_full = s_full + 2, *dp_read = dp_full + 1, *ds_ready = dp_read + 1, *done = ds_ready + 1;
    unsigned long long *own = done + 1;
    volatile int *give_up = reinterpret_cast<int *>(own + 1);
    unsigned *tmem_cell = reinterpret_cast<unsigned *>(own + 2);

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int splits = p.parts_dq.splits;
    const Place at_tile = place_of(block, p.s.heads * splits, p.s.batch);
    const int head = at_tile.head / splits, part = at_tile.head % splits, b = at_tile.batch, kv_head = head / (p.s.heads / p.s.kv_heads);
    const int q0 = (p.q_tiles - 1 - at_tile.tile) * kRows;
    const Lengths len = lengths_of(p.s, b);
    const int last = min(q0 + kRows, len.q) - 1;
    const int seen = last < q0 ? 0 : p.s.causal ? min(len.kv, last + len.shift + 1) : len.kv;
    int h0, h1;                                                     // this block's key tiles
    stretch_of(seen > 0 ? (seen + kRows - 1) / kRows : 0, part, splits, &h0, &h1);
    const int n = h1 - h0;
    if (n == 0) {                                                   // no query of the tile sees a key
        wait_for_previous();                                        // as in attention_keys
        if (splits > 1) zero_parts(p.parts_dq, part, b, head, q0, min(kRows, p.s.q_len - q0), p.s.dim);
        else zero_tile(p.dq, b, head, q0, min(kRows, p.s.q_len - q0), p.s.dim);
        return;
    }

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int i = 0; i < KS; ++i) { mbar_init(k_full + i, 1); mbar_init(k_empty + i, 1); }
        for (int i = 0; i < VS; ++i) { mbar_init(v_full + i, 1); mbar_init(v_empty + i, 1); }
        mbar_init(s_full, 1); mbar_init(s_full + 1, 1);
        mbar_init(dp_full, 1); mbar_init(dp_read, kElementWarps); mbar_init(ds_ready, kElementWarps);
        mbar_init(done, 1); mbar_init(own, 1);
        *give_up = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) tmem_alloc(tmem_cell, 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const unsigned tmem = *tmem_cell;
    const unsigned dq_at = tmem, s_at = tmem + DP, dp_at = s_at + 2 * kRows;

    if (warp == kLoadWarp) {
        Loader load = {own, 0, give_up, p.status};
        if (lane == 0) {
            prefetch_map(&p.q); prefetch_map(&p.k); prefetch_map(&p.v); prefetch_map(&p.dout);
            mbar_expect_tx(q_full, 2 * L::kTile);
            load_tile<DP>(smem + L::kQ, &p.q, head, q0, b, q_full);
            load_tile<DP>(smem + L::kDo, &p.dout, head, q0, b, q_full);
        }
        int k_armed = 0, v_armed = 0;
        for (int h = 0; h < n; ++h) {
            const int ks = h % KS, vs = h % VS;
            if (!load.wait(k_empty + ks, ((h / KS) & 1) ^ 1)) break;
            if (!load.tile<DP>(smem + L::kK + ks * L::kTile, &p.k, kv_head, (h0 + h) * kRows, b, k_full + ks,
                               p.s.kv_lengths ? len.kv - (h0 + h) * kRows : kRows))
                break;
            ++k_armed;
            if (!load.wait(v_empty + vs, ((h / VS) & 1) ^ 1)) break;
            load.tile<DP>(smem + L::kV + vs * L::kTile, &p.v, kv_head, (h0 + h) * kRows, b, v_full + vs, kRows);
            ++v_armed;
        }
        mbar_wait(q_full, 0);
        for (int h = max(0, k_armed - KS); h < k_armed; ++h) mbar_wait(k_full + h % KS, (h / KS) & 1);
        for (int h = max(0, v_armed - VS); h < v_armed; ++h) mbar_wait(v_full + h % VS, (h / VS) & 1);
        __syncwarp();
    } else if (warp == kMmaWarp) {
        if (elect_one()) {
            const unsigned q = smem_addr(smem + L::kQ), d = smem_addr(smem + L::kDo);
            const unsigned k0 = smem_addr(smem + L::kK), v0 = smem_addr(smem + L::kV);
            auto wait = [&](unsigned long long *bar, unsigned parity) { return bounded_wait(bar, parity, give_up, p.status); };
            auto scores = [&](int h) {
                const int st = h % KS;
                if (!wait(k_full + st, (h / KS) & 1)) return false;
                fence_after_sync();
                mma_along<DP>(s_at + (h & 1) * kRows, q, k0 + st * L::kTile);
                mma_commit(s_full + (h & 1));
                return true;
            };
            auto slopes = [&](int h) {
                const int st = h % VS;
                if (!wait(v_full + st, (h / VS) & 1)) return false;
                fence_after_sync();
                mma_along<DP>(dp_at, d, v0 + st * L::kTile);
                mma_commit(dp_full);
                mma_commit(v_empty + st);
                return true;
            };
            bool ok = wait(q_full, 0) && scores(0) && slopes(0) && (n < 2 || scores(1));
            for (int h = 0; h < n && ok; ++h) {
                const int st = h % KS;
                if (h + 1 < n && !(ok = wait(dp_read, h & 1) && slopes(h + 1))) break;
                if (!(ok = wait(ds_ready, h & 1))) break;
                fence_after_sync();
                mma_tmem_across<DP, kRows, kCols>(dq_at, s_at + (h & 1) * kRows, k0 + st * L::kTile, h > 0);
                mma_commit(k_empty + st);
                if (h + 2 < n) ok = scores(h + 2);
            }
            mma_commit(done);
            mbar_wait(done, 0);
        }
        __syncwarp();
    } else {
        const int c0 = warp / 4 * kCols, row = threadIdx.x % kRows, i = q0 + row;
        const unsigned lanes = unsigned(warp % 4) * 32u << 16;
        const unsigned s_row = s_at + c0 + lanes, dp_row = dp_at + c0 + lanes;
        const float2 unit = {p.s.scale * kAttnLog2e, p.s.scale * kAttnLog2e};
        const int limit = i >= len.q ? 0 : p.s.causal ? min(len.kv, i + len.shift + 1) : len.kv;
        const long long at = ((long long)b * p.s.heads + head) * p.q_pad + i;
        wait_for_previous();                                        // the row values are the previous kernel's
        const float2 lse = {p.row_lse[at], p.row_lse[at]}, delta = {p.row_delta[at], p.row_delta[at]};
        bool ok = true;
        for (int h = 0; h < n; ++h) {
            const unsigned s_here = s_row + (h & 1) * kRows;
            ok = warp_wait(s_full + (h & 1), (h / 2) & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            const int open = limit - (h0 + h) * kRows - c0;
            uint32_t x[kCols], out[kCols / 2];
            float2 pr[kCols / 2];
            tmem_load(x, s_here);
#pragma unroll
            for (int c = 0; c < kCols; c += 2) {
                const float2 a = fma2({__uint_as_float(x[c]), __uint_as_float(x[c + 1])}, unit, lse);
                pr[c / 2] = {exp2_fast(a.x), exp2_fast(a.y)};
            }
            ok = warp_wait(dp_full, h & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            tmem_load(x, dp_row);
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(dp_read);
#pragma unroll
            for (int c = 0; c < kCols; c += 2)
                pr[c / 2] = mul2(pr[c / 2], add2({__uint_as_float(x[c]), __uint_as_float(x[c + 1])}, delta));
            if (__any_sync(~0u, open < kCols)) {
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    if (c >= open) pr[c / 2].x = 0.0f;
                    if (c + 1 >= open) pr[c / 2].y = 0.0f;
                }
            }
#pragma unroll
            for (int c = 0; c < kCols / 2; ++c) out[c] = pack2(pr[c].x, pr[c].y);
            tmem_store(s_here, out);
            tmem_wait_store();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_ready);
        }
        if (ok) ok = warp_wait(done, 0, give_up, p.status);
        ok = __all_sync(~0u, ok && *give_up == 0);
        fence_after_sync();
        // every four warps a quarter of the columns
        const int d0 = warp / 4 * (DP / 4);
        const bool mine = ok && i < p.s.q_len, empty = limit <= 0;
        if (splits > 1) {
            // a row that sees no key has P = 0 throughout, but a row of Q may hold NaN
            float *dst = p.parts_dq.at(part, b, i, head, p.s.dim) + d0;
            if (ok) store_row<DP / 4>(dq_at + lanes + d0, p.s.scale, dst, p.s.dim - d0, mine && !empty);
            if (mine && empty)
                for (int c = 0; c < DP / 4 && d0 + c < p.s.dim; ++c) dst[c] = 0.0f;
        } else {
            __nv_bfloat16 *dst = p.dq.data + b * p.dq.batch + (long long)i * p.dq.row + head * p.dq.head;
            if (ok) store_row<DP / 4>(dq_at + lanes + d0, p.s.scale, dst + d0, p.s.dim - d0, mine && !empty);
            if (d0 == 0 && mine && empty) store_zeros(dst, p.s.dim);
        }
    }
    fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) tmem_free(tmem, 512);
}

// Both in one launch: neither waits for the other, and the shorter blocks of dQ fill the SMs that the last of dK, dV leave.
template <int DP>
__global__ void __launch_bounds__(kBackwardThreads, 1) attention_backward_kernel(const __grid_constant__ AttnBackwardParams p)
{
    if (int(blockIdx.x) < p.key_blocks) attention_keys<DP>(p, int(blockIdx.x));
    else attention_queries<DP>(p, int(blockIdx.x) - p.key_blocks);
}
template <int DP> struct BackwardShared {
    static constexpr int kBytes = KeysShared<DP>::kBytes > QueriesShared<DP>::kBytes ? KeysShared<DP>::kBytes : QueriesShared<DP>::kBytes;
};

// The gradients whose walks were dealt out, from their parts: a thread per 8 columns of a row.
__global__ void __launch_bounds__(256) attention_backward_join_kernel(const __grid_constant__ AttnBackwardParams p)
{
    wait_for_previous();
    const int groups = p.s.dim / 8;
    long long at = (long long)blockIdx.x * 256 + threadIdx.x;
#pragma unroll
    for (int side = 0; side < 3; ++side) {
        const Parts &o = side == 0 ? p.parts_dq : side == 1 ? p.parts_dk : p.parts_dv;
        const OutView &v = side == 0 ? p.dq : side == 1 ? p.dk : p.dv;
        const long long mine = o.splits > 1 ? o.rows * groups : 0;
        if (at >= mine) { at -= mine; continue; }
        const long long row = at / groups;
        const int c = int(at % groups) * 8, head = int(row % o.heads), i = int(row / o.heads % o.len), b = int(row / o.heads / o.len);
        float sum[8];
        join_parts(o, b, i, head, p.s.dim, c, sum, [](int) { return 1.0f; });
        store_group(v.data + b * v.batch + (long long)i * v.row + head * v.head + c, sum);
        return;
    }
}

}  // namespace omni
