// Attention, forward: O = softmax(scale Q K^T + mask) V in one pass over the keys, and the row's log-sum-exp.
//
// A CTA owns 256 query rows of one head as two tiles of 128, and streams key and value tiles of 128.
// Per tile pair: S = Q K^T (tensor memory, float), a thread per row takes the row's running maximum m
// and sum l, writes P = 2^(S - m) as bfloat16 over S, and O += P V with P straight from tensor memory.
// The two tiles take turns: while the threads of one are at their exponentials, the tensor
// core works for the other; the product with V starts on the first quarter of P.
// What bounds it: S, its exponentials and its product with V follow one another (all 512 columns are taken, so the next S
// goes over P), 1900 + 1150 cycles per tile pair and step where the products alone take 2048.  Measured: 2 x 4096 rows, 16 heads on
// 4 of 128, causal, 130 us (1057 TFLOP/s of seen pairs) in a burst, where the clock is at 1.75 GHz, and 146 us a call in a
// long run.  By clock stamps, in thousands of cycles an SM: 8704 steps 179; 512 blocks, 3.5 an SM, 39 more, 11 each (set-up 2.1,
// first loads and scores 2.9, the end with its stores of 16 bytes a row 4.8, on to the next 1.4); mean 217, busiest SM 228.
// Tried: P through shared memory (S free earlier, but an MMA with both operands there takes all its bandwidth) 171 against
// 147 us then; two threads a row 154; exponentials in part by a polynomial on the multiply-add units 137-156 against 135.
// O stays in tensor memory; it is rescaled only when a row's maximum has grown by more than
// 2^8 since its reference (the sum and O carry the same reference, so the result does not change, and
// 2^8 times a tile's sum is far from float's range).  m, l and O are float; P is rounded to bfloat16, as the
// tensor core multiplies that type.
//
// Warps 0-3: rows of tile 0, 4-7: rows of tile 1, 8: loads, 9: MMA.
#pragma once
#include "attention.cuh"

namespace omni {

struct AttnForwardParams {
    CUtensorMap q, k, v;
    AttnShape s;
    int q_tiles;                    // pairs of tiles
    OutView out;
    float *lse;
    Parts parts;                    // of out, each divided by its own sum
    float *part_lse;                // [splits][batch][heads][q_len]
    unsigned *status;
};

// Three warpgroups at 168 registers; the third, of which two warps have work, hands most of its share to the other two.
constexpr int kForwardThreads = 384;
constexpr int kForwardFew = 80, kForwardMany = 208;    // 128 x 80 + 256 x 208 <= 384 x 168
constexpr float kRescaleAbove = 8.0f;
constexpr int kParts = 4, kPart = kRows / kParts;      // of P: its product starts when the first is there

template <int DP> struct ForwardShared {
    static constexpr int kStages = DP == 128 ? 2 : 4;
    static constexpr int kTile = kRows * DP * 2;
    static constexpr int kQ = 0, kK = 2 * kTile, kV = kK + kStages * kTile, kBars = kV + kStages * kTile;
    static constexpr int kBytes = kBars + 512 + 1024;      // barriers, and the base rounded up to 1024
};

template <int DP>
__global__ void __launch_bounds__(kForwardThreads, 1) attention_forward_kernel(const __grid_constant__ AttnForwardParams p)
{
    using L = ForwardShared<DP>;
    constexpr int ST = L::kStages;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    unsigned long long *bars = reinterpret_cast<unsigned long long *>(smem + L::kBars);
    unsigned long long *q_full = bars, *k_full = bars + 1, *k_empty = k_full + ST, *v_full = k_empty + ST, *v_empty = v_full + ST;
    unsigned long long *s_full = v_empty + ST, *p_ready = s_full + 2, *o_full = p_ready + 2 * kParts, *drained = o_full + 2, *own = drained + 1;
    volatile int *give_up = reinterpret_cast<int *>(own + 1);
    unsigned *tmem_cell = reinterpret_cast<unsigned *>(own + 2);

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int splits = p.parts.splits;
    const Place at = place_of(int(blockIdx.x), p.s.heads * splits, p.s.batch);
    const int head = at.head / splits, part = at.head % splits, b = at.batch, kv_head = head / (p.s.heads / p.s.kv_heads);
    const int q0 = (p.q_tiles - 1 - at.tile) * 2 * kRows;
    const Lengths len = lengths_of(p.s, b);

    // key tiles that some row of each query tile sees
    int tiles[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int first = q0 + t * kRows, last = min(first + kRows, len.q) - 1;
        const int seen = last < first ? 0 : p.s.causal ? min(len.kv, last + len.shift + 1) : len.kv;
        tiles[t] = seen > 0 ? (seen + kRows - 1) / kRows : 0;
    }
    int j0, j1;                                                       // this block's key tiles
    stretch_of(max(tiles[0], tiles[1]), part, splits, &j0, &j1);
    const int n = j1 - j0;
#pragma unroll
    for (int t = 0; t < 2; ++t) tiles[t] = min(max(tiles[t] - j0, 0), n);
    float *lse = splits > 1 ? p.part_lse + (long long)part * p.s.batch * p.s.heads * p.s.q_len : p.lse;
    lse += ((long long)b * p.s.heads + head) * p.s.q_len;
    if (n == 0) {                                                     // no row sees a key
        const int rows = min(2 * kRows, p.s.q_len - q0);
        if (splits > 1) zero_parts(p.parts, part, b, head, q0, rows, p.s.dim);
        else zero_tile(p.out, b, head, q0, rows, p.s.dim);
        for (int i = threadIdx.x; i < rows; i += blockDim.x) lse[q0 + i] = -INFINITY;
        return;
    }

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int i = 0; i < ST; ++i) {
            mbar_init(k_full + i, 1); mbar_init(k_empty + i, 1);
            mbar_init(v_full + i, 1); mbar_init(v_empty + i, 1);
        }
        for (int t = 0; t < 2; ++t) { mbar_init(s_full + t, 1); mbar_init(o_full + t, 1); }
        for (int i = 0; i < 2 * kParts; ++i) mbar_init(p_ready + i, 4);   // [tile][part]
        mbar_init(drained, 1); mbar_init(own, 1);
        *give_up = 0;
        fence_barrier_init();
    }
    if (warp == 9) tmem_alloc(tmem_cell, 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const unsigned tmem = *tmem_cell;
    const unsigned s_at = tmem, o_at = tmem + 2 * kRows;             // S0 S1 | O0 O1

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kForwardFew));
        if (warp == 8) {
            Loader load = {own, 0, give_up, p.status};
            if (lane == 0) {
                prefetch_map(&p.q); prefetch_map(&p.k); prefetch_map(&p.v);
                const int q_tiles = tiles[1] > 0 ? 2 : 1;
                mbar_expect_tx(q_full, q_tiles * L::kTile);
                for (int t = 0; t < q_tiles; ++t) load_tile<DP>(smem + L::kQ + t * L::kTile, &p.q, head, q0 + t * kRows, b, q_full);
            }
            int kj = 0, vj = 0;                                       // copies armed
            for (int j = 0; j < n; ++j) {
                const int st = j % ST;
                const unsigned free_parity = ((j / ST) & 1) ^ 1;
                if (!load.wait(k_empty + st, free_parity)) break;
                load.tile<DP>(smem + L::kK + st * L::kTile, &p.k, kv_head, (j0 + j) * kRows, b, k_full + st, kRows);
                ++kj;
                if (!load.wait(v_empty + st, free_parity)) break;
                if (!load.tile<DP>(smem + L::kV + st * L::kTile, &p.v, kv_head, (j0 + j) * kRows, b, v_full + st,
                                   p.s.kv_lengths ? len.kv - (j0 + j) * kRows : kRows))
                    break;
                ++vj;
            }
            // the block may not end with a copy in flight, not even when it gave up
            mbar_wait(q_full, 0);
            for (int j = max(0, kj - ST); j < kj; ++j) mbar_wait(k_full + j % ST, (j / ST) & 1);
            for (int j = max(0, vj - ST); j < vj; ++j) mbar_wait(v_full + j % ST, (j / ST) & 1);
        } else if (warp == 9 && elect_one()) {
            const unsigned q = smem_addr(smem + L::kQ), k = smem_addr(smem + L::kK), v = smem_addr(smem + L::kV);
            auto wait = [&](unsigned long long *bar, unsigned parity) { return bounded_wait(bar, parity, give_up, p.status); };
            bool ok = wait(q_full, 0) && wait(k_full, 0);
            fence_after_sync();
            if (ok) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (tiles[t] > 0) {
                        mma_along<DP>(s_at + t * kRows, q + t * L::kTile, k);
                        mma_commit(s_full + t);
                    }
                mma_commit(k_empty);
            }
            for (int j = 0; j < n && ok; ++j) {
                const int st = j % ST, next = (j + 1) % ST;
                ok = wait(v_full + st, (j / ST) & 1) && (j + 1 >= n || wait(k_full + next, ((j + 1) / ST) & 1));
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (j >= tiles[t]) continue;
#pragma unroll
                    for (int part = 0; part < kParts; ++part) {
                        ok = ok && wait(p_ready + kParts * t + part, j & 1);
                        if (!ok) break;
                        fence_after_sync();
                        mma_tmem_across<DP, kPart, kPart>(o_at + t * DP, s_at + t * kRows + part * kPart / 2,
                                                                 v + st * L::kTile + part * kPart * 128, j > 0 || part > 0);
                    }
                    if (!ok) break;
                    // the next scores go over P: the tensor core takes MMAs in order
                    if (j + 1 < tiles[t]) {
                        mma_along<DP>(s_at + t * kRows, q + t * L::kTile, k + next * L::kTile);
                        mma_commit(s_full + t);
                    } else {
                        mma_commit(o_full + t);
                    }
                }
                if (!ok) break;
                if (j + 1 < n) mma_commit(k_empty + next);
                mma_commit(v_empty + st);
            }
            mma_commit(drained);
            mbar_wait(drained, 0);
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kForwardMany));
        const int t = warp / 4, row = threadIdx.x % kRows, i = q0 + t * kRows + row;
        const unsigned lanes = unsigned(warp % 4) * 32u << 16;
        const unsigned s_row = s_at + t * kRows + lanes, o_row = o_at + t * DP + lanes;
        // keys this row sees: [0, limit)
        const int limit = i >= len.q ? 0 : p.s.causal ? min(len.kv, i + len.shift + 1) : len.kv;
        const float unit = p.s.scale * kAttnLog2e;
        float m = -INFINITY, l = 0.0f;                                // in powers of two
        bool ok = true;
        for (int j = 0; j < tiles[t]; ++j) {
            ok = warp_wait(s_full + t, j & 1, give_up, p.status);
            if (!ok) break;
            fence_after_sync();
            uint32_t x[2][64];
            tmem_load2(x[0], s_row, x[1], s_row + 64);
            const int open = limit - (j0 + j) * kRows;                       // columns of this tile that the row sees
            if (__any_sync(~0u, open < kRows)) {
#pragma unroll
                for (int c = 0; c < kRows; ++c)
                    if (c >= open) x[c / 64][c % 64] = __float_as_uint(-INFINITY);
            }
            float top[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) top[c] = __uint_as_float(x[0][c]);
#pragma unroll
            for (int c = 4; c < kRows; c += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    top[e] = c + 4 + e < kRows ? max3(top[e], __uint_as_float(x[c / 64][c % 64 + e]), __uint_as_float(x[(c + 4) / 64][(c + 4) % 64 + e]))
                                               : fmaxf(top[e], __uint_as_float(x[c / 64][c % 64 + e]));
            const float tile_max = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * unit;
            const bool grow = tile_max > m + kRescaleAbove;           // also the first finite one
            if (__any_sync(~0u, grow)) {
                const float factor = grow ? exp2_fast(m - tile_max) : 1.0f;
                if (grow) { m = tile_max; l *= factor; }
                if (j > 0) {
#pragma unroll
                    for (int c = 0; c < DP / 32; ++c) {
                        uint32_t o[32];
                        tmem_load(o, o_row + c * 32);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                        tmem_store(o_row + c * 32, o);
                    }
                }
            }
            const float ref = m == -INFINITY ? 0.0f : m;
            const float2 unit2 = {unit, unit}, ref2 = {-ref, -ref};
            float2 sum[2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
#pragma unroll
            for (int h = 0; h < kParts; ++h) {
                uint32_t packed[kPart / 2];
#pragma unroll
                for (int c = 0; c < kPart; c += 2) {
                    const float2 z = fma2({__uint_as_float(x[(h * kPart + c) / 64][(h * kPart + c) % 64]), __uint_as_float(x[(h * kPart + c) / 64][(h * kPart + c) % 64 + 1])}, unit2, ref2);
                    const float2 e = {exp2_fast(z.x), exp2_fast(z.y)};
                    sum[c / 2 % 2] = add2(sum[c / 2 % 2], e);
                    packed[c / 2] = pack2(e.x, e.y);
                }
                tmem_store(s_row + h * kPart / 2, packed);
                tmem_wait_store();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready + kParts * t + h);
            }
            l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        }
        if (ok && tiles[t] > 0) ok = warp_wait(o_full + t, 0, give_up, p.status);
        fence_after_sync();
        const bool mine = i < p.s.q_len && ok;
        const bool empty = l == 0.0f, write = mine && !empty;         // empty: the row sees no key
        if (splits > 1) {
            float *dst = p.parts.at(part, b, i, head, p.s.dim);
            if (tiles[t] > 0 && ok) store_row<DP>(o_row, 1.0f / l, dst, p.s.dim, write);
            if (mine && empty)
                for (int c = 0; c < p.s.dim; ++c) dst[c] = 0.0f;
        } else {
            __nv_bfloat16 *dst = p.out.data + b * p.out.batch + (long long)i * p.out.row + head * p.out.head;
            if (tiles[t] > 0 && ok) store_row<DP>(o_row, 1.0f / l, dst, p.s.dim, write);
            if (mine && empty) store_zeros(dst, p.s.dim);
        }
        if (mine) lse[i] = (m + log2f(l)) * kAttnLn2;
    }
    fence_before_sync();
    __syncthreads();
    if (warp == 9) tmem_free(tmem, 512);
}

// out and lse from the parts, a thread per 8 columns: out = sum of exp(lse_k - lse) out_k.
__global__ void __launch_bounds__(256) attention_forward_join_kernel(const __grid_constant__ AttnForwardParams p)
{
    wait_for_previous();
    const int groups = p.s.dim / 8;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= p.parts.rows * groups) return;
    const long long row = at / groups;
    const int c = int(at % groups) * 8, head = int(row % p.s.heads);
    const int i = int(row / p.s.heads % p.s.q_len), b = int(row / p.s.heads / p.s.q_len);
    const long long cell = ((long long)b * p.s.heads + head) * p.s.q_len + i, step = (long long)p.s.batch * p.s.heads * p.s.q_len;
    float top = -INFINITY, total = 0.0f;
    bool nan = false;
    for (int k = 0; k < p.parts.splits; ++k) {
        const float x = p.part_lse[k * step + cell];
        nan = nan || x != x;
        top = fmaxf(top, x);
    }
    for (int k = 0; k < p.parts.splits; ++k) total += top == -INFINITY ? 0.0f : expf(p.part_lse[k * step + cell] - top);
    const float lse = nan ? NAN : top + logf(total);
    float sum[8];
    join_parts(p.parts, b, i, head, p.s.dim, c, sum, [&](int k) { return top == -INFINITY ? 0.0f : expf(p.part_lse[k * step + cell] - lse); });
    store_group(p.out.data + b * p.out.batch + (long long)i * p.out.row + head * p.out.head + c, sum);
    if (c == 0) p.lse[cell] = lse;
}

}  // namespace omni
