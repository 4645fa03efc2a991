// Norms of the query and key heads with the rotation by positions, forward and backward, in one pass.
//
// Per head vector x, with weights w: n_c = w_c x_c r, r = (mean_c x_c^2 + eps)^(-1/2); without weights n = x.  A pair (a, b) of n is
// turned by the angle position * frequency:
//   y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin.
// Backward, from x and dy: dn is dy turned back, dw_c = sum of dn_c x_c r over all rows and heads of the side, and with g = w dn
//   dx = r (g - x r^2 mean_c(g_c x_c)).
// Without weights the gradient is the rotation by the opposite angle.  Floors: one read and one write of the heads; backward two reads.
//
// A group of lanes has a head vector, up to sixteen elements a lane, fetched ahead into shared memory by asynchronous copies: no registers
// wait for them, and no barrier stands between rows.  An angle belongs to a row, so a group keeps its row's angles in registers for all
// heads.  Angles are taken in whole numbers of 2^-64 turns and turned into sines by Taylor's series after the nearest quadrant:
// about 35 instructions a pair, where products in 64-bit floats and the library's function took about 100.
// Forward: blocks of rows, more of them than fit at once; blocks that stay, with the turns dealt out evenly, took 66-75 us where these
// take 58.  Backward: blocks that stay, so that a weight's gradient is summed in registers and 296 partial sums are joined by a second launch;
// the turns of all rows (of a padded batch those before the lengths alone) are dealt to the warps in equal parts.
// Measured: 4 x 4096, 32 heads on 8 of 128 bfloat16, forward 58 us (floor 51); backward 2 x 8192, 16 heads on 8 of 128, 61 us (floor 46): the
// kernel 53, bound by latency that 16 warps an SM, at 128 registers, do not cover (issue 58 %, DRAM 61 %), the join 5; 6 x 1777 of 80, float,
// padded, a quarter of the rows there, 36 us; a single token of 16 sequences 4.6 us.
// Heads or halves that no 16-byte access fits take 8 or 4 bytes at a time, the lanes of a head side by side (sixteen elements in a row
// to a lane: up to twice the time, from the pieces of sectors that are stored): 4751 rows of 16 heads on 4 of 84 bfloat16 18 us (floor 5), backward 29
// (7), 2 x 4096 of 16 on 8 of 250 float 90 (60) and 143 (90).  Element by element those took 37, 51, 91 and 138.
// Tried forward: a group that has a row's queries and keys with one set of angles 61 us where two groups take 58 (1 + 1 heads of 128, 27990 rows, 16
// instead of 20).
// Tried for the backward kernel: loads by registers 111 us; angles of a tile in shared memory between barriers 68-82; weights and angles read from
// shared memory at each turn for a third block an SM 84 (spills); groups of five lanes for a head of 80 39 instead of 36.
#include "context.h"
#include "vector.cuh"

#include <cmath>
#include <initializer_list>
#include <type_traits>
#include <utility>

namespace omni {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxPairs = OMNI_ROTARY_MAX_DIM / 2;
constexpr int kMostSequences = 1024;                  // of a padded batch whose absent rows are passed over
constexpr int kResident = 2;                          // backward blocks an SM

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
    unsigned magic, shift;                            // row / length = (mulhi(magic, row) + row) >> shift
    int dim, pairs, axes;
    int lanes, split;                                 // lanes of a head vector, groups of lanes that share a row's heads (forward): powers of two
    unsigned bundles;                                 // backward: rows in bundles of 32 / lanes
    int batch, padded;                                // sequences; backward walks the bundles before their lengths alone
    int wide_positions, bf16_weight, interleaved, overlap;
    int backwards;                                    // the opposite angle
    float eps;
    unsigned long long frequency[kMaxPairs];          // turns per position, a fraction of 2^64
    unsigned char axis[kMaxPairs];
};

// Where the two parts of UNIT pairs stand (UNIT elements each).  The elements that are not rotated are pairs of angle zero behind the others.
struct Place { int a, b; };
template <int UNIT> __device__ __forceinline__ Place place(const RotaryParams &p, int unit)
{
    const int first = unit * UNIT;
    if (p.interleaved) return {2 * first, 2 * first + UNIT};
    const int rest = p.dim / 2 - p.pairs;
    return first < p.pairs ? Place{first, first + p.pairs} : Place{first + p.pairs, first + p.pairs + rest};
}

// Sums over a group of lanes; spelled out, so that the steps are branches of the whole warp.
__device__ __forceinline__ float group_sum(float x, int lanes)
{
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        if (o >= lanes) break;
        x += __shfl_xor_sync(~0u, x, o);
    }
    return x;
}
__device__ __forceinline__ float2 group_sum(float2 x, int lanes)
{
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        if (o >= lanes) break;
        const float a = __shfl_xor_sync(~0u, x.x, o), b = __shfl_xor_sync(~0u, x.y, o);
        x = make_float2(x.x + a, x.y + b);
    }
    return x;
}

// A row of the batch, and where its heads start in an operand.
struct RowAt {
    unsigned batch, i;
    bool mine, there;                                 // a row of the call; not behind its sequence's length
    __device__ __forceinline__ RowAt(const RotaryParams &p, unsigned row) : mine(row < p.rows)
    {
        batch = (__umulhi(p.magic, row) + row) >> p.shift;
        i = row - batch * p.length;
        there = mine && (!p.lengths || int(i) < p.lengths[batch]);
    }
    template <typename T> __device__ __forceinline__ T *in(const View &v) const { return static_cast<T *>(v.data) + batch * v.batch + i * v.row; }
};

// Cosine and sine of an angle in 2^-32 turns: the quadrant nearest to it, and Taylor's series of the rest, which is within pi / 4
// (next terms below 2^-29).
__device__ __forceinline__ void cos_sin(uint32_t angle, float *c, float *s)
{
    const uint32_t quadrant = (angle + (1u << 29)) >> 30;
    const float x = float(int(angle - (quadrant << 30))) * 1.4629180792671596e-9f, y = x * x;        // 2 pi / 2^32
    const float odd = fmaf(fmaf(fmaf(fmaf(y, 1.0f / 362880.0f, -1.0f / 5040.0f), y, 1.0f / 120.0f), y, -1.0f / 6.0f) * y, x, x);
    const float even = fmaf(fmaf(fmaf(fmaf(fmaf(y, -1.0f / 3628800.0f, 1.0f / 40320.0f), y, -1.0f / 720.0f), y, 1.0f / 24.0f), y, -0.5f), y, 1.0f);
    const float a = quadrant & 1 ? odd : even, b = quadrant & 1 ? even : odd;
    *c = (quadrant + 1) & 2 ? -a : a;
    *s = quadrant & 2 ? -b : b;
}

// A block's copy of the pairs' frequencies (0, which gives cosine 1 and sine 0, for those that are not rotated) and axes: asked of the
// parameters, every lane another, they are slow.
struct Pairs {
    static constexpr int kCount = kMaxPairs + 1;      // the last is never turned
    unsigned long long frequency[kCount];
    unsigned char axis[kCount];
    __device__ __forceinline__ void fill(const RotaryParams &p)
    {
        for (int i = threadIdx.x; i < kCount; i += kThreads) {
            frequency[i] = i < p.pairs ? p.frequency[i] : 0;
            axis[i] = i < p.pairs ? p.axis[i] : 0;
        }
    }
};

__device__ __forceinline__ unsigned long long position_at(const RotaryParams &p, const RowAt &row, int axis)
{
    if (!row.mine) return 0;
    const unsigned long long at = row.batch * p.position_batch + row.i * p.position_row + axis * p.position_axis;
    const unsigned long long x = p.wide_positions ? load_index<long long>(p.positions, at) : load_index<int>(p.positions, at);
    return p.backwards ? -x : x;
}

// A row's angles, pair by pair; `position` is that of `axis`, fetched ahead.  A position times the turns per position, in whole numbers
// modulo 2^64, is what is left of the angle after its whole turns: however far the position, it is off by
// 2^-65 turns per position, and by the 2^-32 of the part that is used.
struct Angles {
    const RotaryParams &p;
    const Pairs &pairs;
    const RowAt &row;
    unsigned long long position;
    int axis;
    __device__ __forceinline__ void at(int pair, float *c, float *s)
    {
        if (p.axes > 1 && pairs.axis[pair] != axis) position = position_at(p, row, axis = pairs.axis[pair]);
        cos_sin(uint32_t(position * pairs.frequency[pair] >> 32), c, s);
    }
};

// Forward: how a block's threads share its rows: `lanes` of a head vector; `split` groups of them have the heads of one row in turn.
struct Share {
    int lane, row, first, turns;                      // heads first, first + split, ...; every group takes as many turns, for the shuffles
    __device__ __forceinline__ Share(const RotaryParams &p, int heads)
    {
        const int group = threadIdx.x / p.lanes;
        lane = threadIdx.x % p.lanes;
        row = group / p.split;
        first = group % p.split;
        turns = (heads + p.split - 1) / p.split;
    }
};
__device__ __forceinline__ unsigned rows_of_block(const RotaryParams &p) { return kThreads / (p.lanes * p.split); }

// Backward, of a padded batch: how many bundles (the rows of a warp's groups) lie before each sequence, counting those that begin
// before its length.
struct Sequences {
    int before[kMostSequences + 1];
    __device__ __forceinline__ void fill(const RotaryParams &p)
    {
        if (threadIdx.x >= 32) return;
        const int lane = threadIdx.x, each = (p.batch + 31) / 32, first = min(lane * each, p.batch), last = min(first + each, p.batch);
        const unsigned rows = 32 / p.lanes;
        int sum = 0;
        for (int b = first; b < last; ++b) {
            before[b] = sum;                          // of this lane's
            sum += (min(unsigned(max(p.lengths[b], 0)), p.length) + rows - 1) / rows;        // unsigned: may pass 31 bits
        }
        int ahead = sum;
        for (int o = 1; o < 32; o *= 2) {
            const int other = __shfl_up_sync(~0u, ahead, o);
            if (lane >= o) ahead += other;
        }
        if (lane == 31) before[p.batch] = ahead;
        for (int b = first; b < last; ++b) before[b] += ahead - sum;
    }
};

// Backward: a warp's share of a side: a group of lanes has a row, the warp's groups a bundle of rows, and a turn is one head of each.  The turns of all
// bundles are dealt to the side's warps in equal parts, wherever in a bundle they begin.  PADDED: of the bundles before the sequences' lengths alone.
constexpr unsigned kNoRow = 0x7fffffffu;              // behind all rows
template <bool PADDED> struct Walk {
    unsigned number;                                  // of the bundle
    int sequence, head, left;                         // its sequence; turns that are left
    __device__ __forceinline__ Walk(const RotaryParams &p, const Sequences *seq, unsigned block, unsigned blocks, int heads) : sequence(0)
    {
        const unsigned long long bundles = PADDED ? unsigned(seq->before[p.batch]) : p.bundles;
        const unsigned long long all = bundles * heads, warps = (unsigned long long)blocks * kWarps;
        const unsigned long long me = (unsigned long long)block * kWarps + threadIdx.x / 32;
        const unsigned long long first = all * me / warps;
        left = int(all * (me + 1) / warps - first);
        number = unsigned(first / heads);
        head = int(first - (unsigned long long)number * heads);
        if (!PADDED || left == 0) return;
        int high = p.batch;                           // the last sequence that begins at or before the bundle
        while (high - sequence > 1) {
            const int middle = (sequence + high) / 2;
            if (seq->before[middle] <= int(number)) sequence = middle;
            else high = middle;
        }
    }
    // the group's row
    __device__ __forceinline__ unsigned row(const RotaryParams &p, const Sequences *seq) const
    {
        const unsigned rows = 32 / p.lanes, group = threadIdx.x % 32 / p.lanes;
        if constexpr (PADDED) {
            const unsigned i = (number - unsigned(seq->before[sequence])) * rows + group;
            return i < p.length ? sequence * p.length + i : kNoRow;
        } else {
            return number * rows + group;
        }
    }
    __device__ __forceinline__ void next(const RotaryParams &p, const Sequences *seq, int heads, int by = 1)
    {
        left -= by;
        head += by;
        if (head < heads) return;
        head = 0;
        ++number;
        if constexpr (PADDED)
            while (sequence < p.batch - 1 && seq->before[sequence + 1] <= int(number)) ++sequence;
    }
    __device__ __forceinline__ unsigned next_row(const RotaryParams &p, const Sequences *seq, int heads) const
    {
        Walk then = *this;
        then.next(p, seq, heads, heads - head);
        return left > heads - head ? then.row(p, seq) : kNoRow;
    }
};

// Backward, of a padded batch: f(a row behind its length) by each group, over all rows.
template <typename F> __device__ __forceinline__ void absent_rows(const RotaryParams &p, const Side &side, unsigned block, F f)
{
    for (unsigned n = block * kWarps + threadIdx.x / 32; n < p.bundles; n += side.blocks * kWarps) {
        const RowAt row(p, n * unsigned(32 / p.lanes) + threadIdx.x % 32 / p.lanes);
        if (row.mine && !row.there) f(row);
    }
}

__device__ __forceinline__ float weight_at(const RotaryParams &p, const Side &side, int c)
{
    return p.bf16_weight ? to_float(static_cast<const __nv_bfloat16 *>(side.weight)[c]) : static_cast<const float *>(side.weight)[c];
}

// A block's sums of the weight's gradient: f(channel) of each lane's elements, groups of a warp by shuffles, then the warps in order.
__device__ __forceinline__ float warp_groups_sum(float v, int lanes)
{
    for (int o = 16; o >= lanes; o /= 2) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
__device__ __forceinline__ void put_partial(const RotaryParams &p, const float *sums, float *partial)
{
    for (int ch = threadIdx.x; ch < p.dim; ch += kThreads) {
        float v = sums[ch];
        for (int w = 1; w < kWarps; ++w) v += sums[w * p.dim + ch];
        partial[ch] = v;
    }
}

// ---- wide accesses: a lane has sixteen elements, fetched ahead by asynchronous copies into slots of its own ----------------------

// Which sixteen: eight pairs whose halves are both whole groups of eight; eight pairs of neighbours; or, with halves that do not begin on a
// group, sixteen elements in a row, whose partners are read one by one from the slots of the lanes that have them.
enum Layout { kHalves, kNeighbours, kGathered };
template <Layout L> __device__ __forceinline__ Place wide_place(const RotaryParams &p, int unit)
{
    return L == kHalves ? place<8>(p, unit) : Place{16 * unit, 16 * unit + 8};
}

// A lane's two chunks of eight, as it reads and writes them.  GRAIN: bytes of an access.  16: a chunk is eight elements in a row.  Below, where
// operands or halves do not begin on groups of eight, it is runs of a few, the lanes of a head side by side, so that an access of a
// warp still is a few whole pieces of memory; some runs may not exist, and count as zeros.
template <typename T, Layout L, int GRAIN> struct Lane {
    // elements of an access and of a run, runs of a chunk
    enum : int { kLeast = GRAIN / int(sizeof(T)), kEach = GRAIN == 16 ? kGroup : L == kNeighbours && kLeast < 2 ? 2 : kLeast, kRuns = kGroup / kEach };
    bool has;
    int unit, start, to_b;                            // the place of the first element; 16: from there to the other chunk
    int step, turned_runs, runs[2];                   // from run to run; those of pairs that are turned; those of either chunk that exist
    int pairs, half;                                  // what is not turned is dealt in two halves, from 2 * pairs on
    __device__ __forceinline__ Lane(const RotaryParams &p, int lane) : unit(lane), pairs(p.pairs)
    {
        if constexpr (GRAIN == 16) {
            has = lane * 16 < p.dim;
            if (!has) unit = 0;
            const Place at = wide_place<L>(p, unit);
            start = at.a;
            to_b = at.b - at.a;
        } else {
            start = lane * kEach;
            step = p.lanes * kEach;
            const auto before = [&](int end) { return max(0, min(int(kRuns), (end - start + step - 1) / step)); };       // runs that begin before `end`
            if constexpr (L == kNeighbours) {
                runs[0] = before(p.dim);
                runs[1] = max(0, min(int(kRuns), (p.dim - start - kRuns * step + step - 1) / step));
            } else {
                const int rest = (p.dim - 2 * pairs) / kEach;
                half = (rest + 1) / 2 * kEach;
                turned_runs = before(pairs);
                runs[0] = before(pairs + half);
                runs[1] = max(turned_runs, before(p.dim - pairs - half));
            }
            has = runs[0] > 0;
        }
    }
    // from `start` to run i of a chunk
    __device__ __forceinline__ int offset(int chunk, int i) const
    {
        if constexpr (GRAIN == 16) return chunk ? to_b : 0;
        else if constexpr (L == kNeighbours) return (chunk * kRuns + i) * step;
        else return i * step + (i < turned_runs ? chunk ? pairs : 0 : chunk ? pairs + half : pairs);
    }
    __device__ __forceinline__ bool there(int chunk, int i) const { return GRAIN == 16 || i < runs[chunk]; }
    // Of the sixteen elements in the order of the chunks, element x: its place in the head vector, and whether it exists.
    __device__ __forceinline__ int element(int x) const { return start + offset(x / kGroup, x % kGroup / kEach) + x % kEach; }
    __device__ __forceinline__ bool exists(int x) const { return there(x / kGroup, x % kGroup / kEach); }
    // Pair j of the eight.
    __device__ __forceinline__ int pair(int j) const
    {
        if constexpr (GRAIN == 16) return unit * 8 + j;
        else if constexpr (L == kNeighbours) return min(element(2 * j) / 2, pairs);
        else return min(start + j / kEach * step + j % kEach, pairs);
    }
    // How many of its leading pairs are turned; eight as well if only such exist.
    __device__ __forceinline__ int turned() const
    {
        if constexpr (GRAIN == 16) {
            return L == kGathered ? 2 * pairs - start : pairs - unit * 8;
        } else {
            int n = 0, all = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool is = exists(L == kNeighbours ? 2 * j : j);
                n += is && pair(j) < pairs;
                all += is;
            }
            return n == all ? 8 : n;
        }
    }
    __device__ __forceinline__ void put(T *to, const float *f) const
    {
#pragma unroll
        for (int chunk = 0; chunk < 2; ++chunk) {
            if constexpr (GRAIN == 16) {
                store_group(to + offset(chunk, 0), f + 8 * chunk);
            } else {
#pragma unroll
                for (int i = 0; i < kRuns; ++i) {
                    if (!there(chunk, i)) break;
                    put_run(to + offset(chunk, i), f + 8 * chunk + i * kEach);
                }
            }
        }
    }
    static __device__ __forceinline__ uint32_t word(const float *f)
    {
        if constexpr (sizeof(T) == 4) return __float_as_uint(f[0]);
        const __nv_bfloat162 x = __floats2bfloat162_rn(f[0], f[1]);
        return *reinterpret_cast<const uint32_t *>(&x);
    }
    static __device__ __forceinline__ void put_run(T *to, const float *f)
    {
#pragma unroll
        for (int e = 0; e < kEach; e += kLeast) {
            if constexpr (GRAIN == 8) *reinterpret_cast<uint2 *>(to + e) = make_uint2(word(f + e), word(f + e + kLeast / 2));
            else *reinterpret_cast<uint32_t *>(to + e) = word(f + e);
        }
    }
};

// Eight elements in shared memory: pieces of 16 bytes, each piece of all threads side by side.
template <typename T> constexpr int kPieces = int(sizeof(T)) / 2;
__device__ __forceinline__ void copy_async(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
template <int GRAIN> __device__ __forceinline__ void copy_async_grain(uint32_t to, const void *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(GRAIN) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// CHUNKS chunks of eight elements a stage.  The start is on 128 bytes, so that a warp's 512 are four whole lines: backward 61 us, 65 without.
template <typename T, int CHUNKS, int STAGES> struct Ring {
    static constexpr int kStage = CHUNKS * kPieces<T> * kThreads * 16;
    static constexpr int kBytes = STAGES * kStage;
    char *base;
    uint32_t shared;
    __device__ __forceinline__ explicit Ring(char *at) : base(at + threadIdx.x * 16), shared(uint32_t(__cvta_generic_to_shared(base))) {}
    __device__ __forceinline__ void fetch(int stage, int chunk, const T *from) const
    {
#pragma unroll
        for (int i = 0; i < kPieces<T>; ++i)
            copy_async(shared + stage * kStage + (chunk * kPieces<T> + i) * kThreads * 16, reinterpret_cast<const char *>(from) + 16 * i);
    }
    // A lane's two chunks, from the first one's start on.
    template <Layout L, int GRAIN> __device__ __forceinline__ void fetch(int stage, int chunk, const T *from, const Lane<T, L, GRAIN> &lane) const
    {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if constexpr (GRAIN == 16) {
                fetch(stage, chunk + c, from + lane.offset(c, 0));
            } else {
                const uint32_t to = shared + stage * kStage + (chunk + c) * kPieces<T> * kThreads * 16;
#pragma unroll
                for (int i = 0; i < lane.kRuns; ++i) {
                    if (!lane.there(c, i)) break;
#pragma unroll
                    for (int e = 0; e < lane.kEach; e += lane.kLeast) {
                        const int o = (i * lane.kEach + e) * int(sizeof(T));
                        copy_async_grain<GRAIN>(to + o / 16 * kThreads * 16 + o % 16, from + lane.offset(c, i) + e);
                    }
                }
            }
        }
    }
    // Zeros in place of what is not there: a turn's sums need no cases then.
    __device__ __forceinline__ void clear(int stage) const
    {
#pragma unroll
        for (int i = 0; i < CHUNKS * kPieces<T>; ++i) *reinterpret_cast<uint4 *>(base + stage * kStage + i * kThreads * 16) = make_uint4(0, 0, 0, 0);
    }
    // Where element j of the group's head vector stands in a stage, from the start of the block's slots on; `first`: the group's first thread.
    static __device__ __forceinline__ int element(int first, int chunk, int j)
    {
        const int piece = (chunk + j / 8 % 2) * kPieces<T> + j % 8 * int(sizeof(T)) / 16;
        return (piece * kThreads + first + j / 16) * 16 + j * int(sizeof(T)) % 16;
    }
    __device__ __forceinline__ float at(int stage, int offset) const
    {
        return to_float(*reinterpret_cast<const T *>(base - threadIdx.x * 16 + stage * kStage + offset));
    }
    __device__ __forceinline__ void get(int stage, int chunk, float *f) const
    {
        const char *const at = base + stage * kStage + chunk * kPieces<T> * kThreads * 16;
        if constexpr (sizeof(T) == 2) {
            widen(*reinterpret_cast<const uint4 *>(at), f);
        } else {
            const float4 x = *reinterpret_cast<const float4 *>(at), y = *reinterpret_cast<const float4 *>(at + kThreads * 16);
            f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
            f[4] = y.x; f[5] = y.y; f[6] = y.z; f[7] = y.w;
        }
    }
};

// A unit's 16 elements, in the order of its two chunks, as two pairs (of first or of second elements) of consecutive rotations.
template <Layout L> __device__ __forceinline__ float2 firsts(const float *f, int i)
{
    return L == kNeighbours ? make_float2(f[4 * i], f[4 * i + 2]) : make_float2(f[2 * i], f[2 * i + 1]);
}
template <Layout L> __device__ __forceinline__ float2 seconds(const float *f, int i)
{
    return L == kNeighbours ? make_float2(f[4 * i + 1], f[4 * i + 3]) : make_float2(f[8 + 2 * i], f[8 + 2 * i + 1]);
}
template <Layout L> __device__ __forceinline__ void put_pairs(float *f, int i, float2 a, float2 b)
{
    if (L == kNeighbours) {
        f[4 * i] = a.x; f[4 * i + 2] = a.y; f[4 * i + 1] = b.x; f[4 * i + 3] = b.y;
    } else {
        f[2 * i] = a.x; f[2 * i + 1] = a.y; f[8 + 2 * i] = b.x; f[8 + 2 * i + 1] = b.y;
    }
}
__device__ __forceinline__ float2 minus(float2 a) { return make_float2(-a.x, -a.y); }

// The side's weights in shared memory.
struct Weights {
    float w[OMNI_ROTARY_MAX_DIM];
    __device__ __forceinline__ void fill(const RotaryParams &p, const Side &side)
    {
        for (int i = threadIdx.x; i < p.dim; i += kThreads) w[i] = weight_at(p, side, i);
    }
};
__device__ __forceinline__ float2 two(const float *f, int i) { return *reinterpret_cast<const float2 *>(f + i); }
// Those of a lane's sixteen elements, in the order of the chunks.
template <typename T, Layout L, int GRAIN> __device__ __forceinline__ void weights_of(const Weights &weights, const Lane<T, L, GRAIN> &lane, float *w)
{
#pragma unroll
    for (int x = 0; x < 16; ++x) w[x] = lane.exists(x) ? weights.w[lane.element(x)] : 0.0f;
}

// What a pair's other element adds to one that is not turned is nothing, whatever it is (a product with a sine of 0 would carry infinities and
// NaN over): of two consecutive pairs or elements, of which `turned` counts those that are.
__device__ __forceinline__ float2 still(float2 x, int turned) { return make_float2(turned > 0 ? x.x : 0.0f, turned > 1 ? x.y : 0.0f); }

// Gathered: what turns element i, the element it is turned with, and the sign of that one's sine.
struct Partner {
    int pair, with;
    float sign;
    __device__ __forceinline__ Partner(const RotaryParams &p, int i, bool back)
    {
        pair = i < p.pairs ? i : i < 2 * p.pairs ? i - p.pairs : p.pairs;        // those that are not turned: a frequency of 0
        with = i < p.pairs ? i + p.pairs : i < 2 * p.pairs ? i - p.pairs : i;
        sign = (i < p.pairs) == back ? 1.0f : -1.0f;
    }
};
// The offsets of sixteen partners in a stage, two to a word.
template <typename R> __device__ __forceinline__ void partner_offsets(const RotaryParams &p, int first, int chunk, int from, uint32_t *offset)
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        offset[e] = uint32_t(R::element(first, chunk, Partner(p, from + 2 * e, false).with)) |
                    uint32_t(R::element(first, chunk, Partner(p, from + 2 * e + 1, false).with)) << 16;
}
template <typename R> __device__ __forceinline__ float2 partners(const R &ring, int stage, uint32_t offset)
{
    return make_float2(ring.at(stage, int(offset & 0xffffu)), ring.at(stage, int(offset >> 16)));
}

template <typename T> constexpr int kForwardStages = sizeof(T) == 2 ? 6 : 4;
template <typename T> using ForwardRing = Ring<T, 2, kForwardStages<T>>;

// Forward: a group of lanes has a row of one side.  With weights they are folded into the angles, and a result is
// y_a = r ((w_a cos) x_a - (w_b sin) x_b), y_b = r ((w_b cos) x_b + (w_a sin) x_a).
template <typename T, Layout L, bool NORM, int GRAIN>
__global__ void __launch_bounds__(kThreads, L == kGathered ? 2 : 3) rotary_forward_wide_kernel(const __grid_constant__ RotaryParams p)
{
    extern __shared__ __align__(128) char shared[];
    __shared__ Pairs pairs;
    __shared__ __align__(16) Weights weights;
    constexpr int kStages = kForwardStages<T>;
    const ForwardRing<T> ring(shared);
    const bool keys = blockIdx.x >= p.side[0].blocks;
    const Side &side = p.side[keys];
    const Share me(p, side.heads);
    const RowAt row(p, (blockIdx.x - (keys ? p.side[0].blocks : 0u)) * rows_of_block(p) + me.row);
    const Lane<T, L, GRAIN> mine(p, me.lane);
    const bool has = mine.has;
    const int from = mine.start;
    const T *src = row.in<T>(side.x) + me.first * side.x.head + from;
    T *dst = row.in<T>(side.out) + me.first * side.out.head + from;
    const unsigned long long src_step = p.split * side.x.head, dst_step = p.split * side.out.head;
    int ahead = row.there && has ? me.first : side.heads;               // the next head to be fetched
    const auto fetch = [&](int stage) {
        if (ahead < side.heads) {
            ring.fetch(stage, 0, src, mine);
            src += src_step;
            ahead += p.split;
        } else {
            ring.clear(stage);
        }
        copies_commit();
    };
    if constexpr (GRAIN < 16)
        for (int j = 0; j < kStages; ++j) ring.clear(j);
#pragma unroll
    for (int j = 0; j < kStages - 1; ++j) fetch(j);
    pairs.fill(p);
    if constexpr (NORM) weights.fill(p, side);
    __syncthreads();
    constexpr int kCoefficients = L == kGathered ? 8 : 4;
    // cos and sin, with weights those times w_a and w_b, sb with its sign; gathered: of an element and of its partner
    float2 ca[kCoefficients], sa[kCoefficients], cb[4], sb[4];
    uint32_t offset[8];
    const int first_pair = L == kGathered ? Partner(p, from, false).pair : mine.pair(0);
    Angles angles{p, pairs, row, position_at(p, row, pairs.axis[first_pair]), pairs.axis[first_pair]};
    if constexpr (L == kGathered) {
        partner_offsets<ForwardRing<T>>(p, int(threadIdx.x) - me.lane, 0, from, offset);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const Partner x(p, from + 2 * e, false), y(p, from + 2 * e + 1, false);
            angles.at(x.pair, &ca[e].x, &sa[e].x);
            angles.at(y.pair, &ca[e].y, &sa[e].y);
            sa[e] = mul2(sa[e], make_float2(x.sign, y.sign));
            if constexpr (NORM) {
                ca[e] = mul2(ca[e], two(weights.w, from + 2 * e));
                sa[e] = mul2(sa[e], make_float2(weights.w[x.with], weights.w[y.with]));
            }
        }
    } else {
        float w[16];
        if constexpr (NORM) weights_of(weights, mine, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 c, s;
            angles.at(mine.pair(2 * i), &c.x, &s.x);
            angles.at(mine.pair(2 * i + 1), &c.y, &s.y);
            const float2 wa = firsts<L>(w, i), wb = seconds<L>(w, i);
            ca[i] = NORM ? mul2(c, wa) : c;
            cb[i] = NORM ? mul2(c, wb) : c;
            sa[i] = NORM ? mul2(s, wa) : s;
            sb[i] = minus(NORM ? mul2(s, wb) : s);
        }
    }
    const float inverse_dim = 1.0f / float(p.dim);
    const int turned = mine.turned();                  // gathered: elements
    int stage = 0, head = row.mine && has ? me.first : side.heads;
    for (int j = 0; j < me.turns; ++j, head += p.split, dst += dst_step) {
        copies_wait<kStages - 2>();
        float f[16];
        float2 with[8];
        if constexpr (L == kGathered) __syncwarp();   // other lanes' copies have arrived, and they are done with the turn before
        ring.get(stage, 0, f);
        ring.get(stage, 1, f + 8);
        if constexpr (L == kGathered)
#pragma unroll
            for (int e = 0; e < 8; ++e) with[e] = partners(ring, stage, offset[e]);
        // into the slot that the turn before this one has used up
        fetch(stage == 0 ? kStages - 1 : stage - 1);
        stage = stage == kStages - 1 ? 0 : stage + 1;
        float2 r = {1.0f, 1.0f};
        if constexpr (NORM) {
            float2 sum = {0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fma2(make_float2(f[2 * e], f[2 * e + 1]), make_float2(f[2 * e], f[2 * e + 1]), sum);
            const float squares = group_sum(sum.x + sum.y, p.lanes);
            r.x = r.y = row.there ? rsqrtf(fmaf(squares, inverse_dim, p.eps)) : 0.0f;
        }
        const auto turn = [&](auto some) {             // some of them are not
            constexpr bool kSome = decltype(some)::value;
            if constexpr (L == kGathered) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 other = kSome ? still(with[e], turned - 2 * e) : with[e];
                    float2 y = fma2(make_float2(f[2 * e], f[2 * e + 1]), ca[e], mul2(other, sa[e]));
                    if constexpr (NORM) y = mul2(y, r);
                    f[2 * e] = y.x;
                    f[2 * e + 1] = y.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 a = firsts<L>(f, i), b = seconds<L>(f, i);
                    const float2 to_a = kSome ? still(b, turned - 2 * i) : b, to_b = kSome ? still(a, turned - 2 * i) : a;
                    float2 ya = fma2(a, ca[i], mul2(to_a, sb[i])), yb = fma2(b, cb[i], mul2(to_b, sa[i]));
                    if constexpr (NORM) {
                        ya = mul2(ya, r);
                        yb = mul2(yb, r);
                    }
                    put_pairs<L>(f, i, ya, yb);
                }
            }
        };
        if (turned >= (L == kGathered ? 16 : 8)) turn(std::false_type());
        else turn(std::true_type());
        if (head < side.heads) mine.put(dst, f);
    }
}

template <typename T> constexpr int kBackwardStages = sizeof(T) == 2 ? 4 : 3;
template <typename T> using BackwardRing = Ring<T, 4, kBackwardStages<T>>;

// Backward of the norm and the rotation: blocks that stay, each on rows of one side, with the weight's gradient in registers.  Two an
// SM: a turn holds x, dy, angles, weights and sums of sixteen elements each, 120 registers and more.
template <typename T, Layout L, bool PADDED, int GRAIN>
__global__ void __launch_bounds__(kThreads, kResident) rotary_backward_wide_kernel(const __grid_constant__ RotaryParams p)
{
    extern __shared__ __align__(128) char shared[];
    __shared__ Pairs pairs;
    __shared__ __align__(16) Weights weights;
    constexpr int kStages = kBackwardStages<T>;
    const BackwardRing<T> ring(shared);
    let_next_begin(p.overlap);
    const bool keys = blockIdx.x >= p.side[0].blocks;
    const Side &side = p.side[keys];
    const unsigned block = blockIdx.x - (keys ? p.side[0].blocks : 0u);
    const int heads = side.heads, lane = threadIdx.x % p.lanes;
    const Lane<T, L, GRAIN> own(p, lane);
    const bool has = own.has;
    const int from = own.start;
    const float inverse_dim = 1.0f / float(p.dim);
    __shared__ Sequences sequences[1];
    const Sequences *const seq = sequences;
    if constexpr (PADDED) {
        sequences->fill(p);
        __syncthreads();
    }
    // what is fetched next: the loads run ahead of the sums, over the bundles' ends
    Walk<PADDED> now(p, seq, block, side.blocks, heads), ahead = now;
    const T *src = nullptr, *grad = nullptr;
    bool ahead_there = false, ahead_new = true;
    const auto fetch = [&](int stage) {
        if (ahead.left > 0) {
            if (ahead_new) {
                const RowAt row(p, ahead.row(p, seq));
                ahead_there = row.there && has;
                src = row.in<T>(side.x) + ahead.head * side.x.head + from;
                grad = row.in<T>(side.dy) + ahead.head * side.dy.head + from;
            }
            if (ahead_there) {
                ring.fetch(stage, 0, src, own);
                ring.fetch(stage, 2, grad, own);
            } else {
                ring.clear(stage);
            }
            src += side.x.head;
            grad += side.dy.head;
            ahead.next(p, seq, heads);
            ahead_new = ahead.head == 0;
        }
        copies_commit();
    };
    if constexpr (GRAIN < 16)
        for (int j = 0; j < kStages; ++j) ring.clear(j);
#pragma unroll
    for (int j = 0; j < kStages - 1; ++j) fetch(j);
    pairs.fill(p);
    weights.fill(p, side);
    __syncthreads();
    constexpr int kCoefficients = L == kGathered ? 8 : 4;
    float2 wa[4], wb[4], da[4] = {}, db[4] = {};
    uint32_t offset[8];
    if constexpr (L == kGathered) partner_offsets<BackwardRing<T>>(p, int(threadIdx.x) - lane, 2, from, offset);
    {
        float w[16];
        weights_of(weights, own, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            wa[i] = firsts<L>(w, i);
            wb[i] = seconds<L>(w, i);
        }
    }
    const int first_pair = L == kGathered ? Partner(p, from, true).pair : own.pair(0);
    unsigned long long position = position_at(p, RowAt(p, now.row(p, seq)), pairs.axis[first_pair]);
    float2 c[kCoefficients], s[kCoefficients];        // gathered: of an element and of its partner, with its sign
    const int turned = own.turned();                   // gathered: elements
    T *dst = nullptr;
    bool mine = false, there = false, fresh = true;
    int stage = 0;
    while (now.left > 0) {
        if (fresh) {
            const RowAt row(p, now.row(p, seq));
            mine = row.mine && has;
            there = row.there && has;
            dst = row.in<T>(side.out) + now.head * side.out.head + from;
            Angles angles{p, pairs, row, position, pairs.axis[first_pair]};
            position = position_at(p, RowAt(p, now.next_row(p, seq, heads)), pairs.axis[first_pair]);
            if constexpr (L == kGathered) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const Partner x(p, from + 2 * e, true), y(p, from + 2 * e + 1, true);
                    angles.at(x.pair, &c[e].x, &s[e].x);
                    angles.at(y.pair, &c[e].y, &s[e].y);
                    s[e] = mul2(s[e], make_float2(x.sign, y.sign));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    angles.at(own.pair(2 * i), &c[i].x, &s[i].x);
                    angles.at(own.pair(2 * i + 1), &c[i].y, &s[i].y);
                }
            }
        }
        copies_wait<kStages - 2>();
        float f[16], g[16];
        if constexpr (L == kGathered) __syncwarp();   // other lanes' copies have arrived, and they are done with the turn before
        ring.get(stage, 0, f);
        ring.get(stage, 1, f + 8);
        ring.get(stage, 2, g);
        ring.get(stage, 3, g + 8);
        const auto turn = [&](auto some) {             // back; some of them are not turned
            constexpr bool kSome = decltype(some)::value;
            if constexpr (L == kGathered) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 with = partners(ring, stage, offset[e]);
                    const float2 n = fma2(make_float2(g[2 * e], g[2 * e + 1]), c[e], mul2(kSome ? still(with, turned - 2 * e) : with, s[e]));
                    g[2 * e] = n.x;
                    g[2 * e + 1] = n.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 a = firsts<L>(g, i), b = seconds<L>(g, i);
                    const float2 to_a = kSome ? still(b, turned - 2 * i) : b, to_b = kSome ? still(a, turned - 2 * i) : a;
                    put_pairs<L>(g, i, fma2(a, c[i], mul2(to_a, s[i])), fma2(b, c[i], mul2(to_b, minus(s[i]))));
                }
            }
        };
        if (turned >= (L == kGathered ? 16 : 8)) turn(std::false_type());
        else turn(std::true_type());
        // into the slot that the turn before this one has used up
        fetch(stage == 0 ? kStages - 1 : stage - 1);
        stage = stage == kStages - 1 ? 0 : stage + 1;
        float2 square = {0.0f, 0.0f}, dot = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = firsts<L>(f, i), b = seconds<L>(f, i);
            const float2 na = firsts<L>(g, i), nb = seconds<L>(g, i);
            square = fma2(b, b, fma2(a, a, square));
            dot = fma2(mul2(b, wb[i]), nb, fma2(mul2(a, wa[i]), na, dot));
        }
        const float2 sums = group_sum(make_float2(square.x + square.y, dot.x + dot.y), p.lanes);
        // 0 where nothing is there: infinite without eps, it would make a NaN of the zeros
        const float scale = there ? rsqrtf(fmaf(sums.x, inverse_dim, p.eps)) : 0.0f, pull = -sums.y * inverse_dim * scale * scale;
        const float2 r = {scale, scale}, q = {pull, pull};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = firsts<L>(f, i), b = seconds<L>(f, i);
            const float2 na = firsts<L>(g, i), nb = seconds<L>(g, i);
            da[i] = fma2(na, mul2(a, r), da[i]);
            db[i] = fma2(nb, mul2(b, r), db[i]);
            put_pairs<L>(f, i, mul2(r, fma2(a, q, mul2(na, wa[i]))), mul2(r, fma2(b, q, mul2(nb, wb[i]))));
        }
        if (mine) own.put(dst, f);
        dst += side.out.head;
        now.next(p, seq, heads);
        fresh = now.head == 0;
    }
    if constexpr (PADDED)
        absent_rows(p, side, block, [&](const RowAt &row) {
            T *to = row.in<T>(side.out) + from;
            const float zeros[16] = {};
            for (int head = 0; has && head < heads; ++head, to += side.out.head) own.put(to, zeros);
        });
    copies_wait<0>();
    __syncthreads();
    float *const sums = reinterpret_cast<float *>(shared);
    float dw[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) put_pairs<L>(dw, i, da[i], db[i]);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float v = warp_groups_sum(dw[e], p.lanes);
        if (int(threadIdx.x % 32) < p.lanes && has && own.exists(e)) sums[threadIdx.x / 32 * p.dim + own.element(e)] = v;
    }
    __syncthreads();
    put_partial(p, sums, side.partial + (unsigned long long)block * p.dim);
}

// ---- bfloat16 that no access of two elements fits: element by element, up to four pairs a lane in registers ----------------------

constexpr int kOwn = kMaxPairs / 32;                  // pairs of a lane
struct Own {
    Place at[kOwn];
    bool has[kOwn], turned[kOwn];
    float w[kOwn][2];
    __device__ __forceinline__ Own(const RotaryParams &p, const Side &side, int lane, bool norm)
    {
#pragma unroll
        for (int n = 0; n < kOwn; ++n) {
            const int unit = lane + n * p.lanes;
            has[n] = unit < p.dim / 2;
            turned[n] = unit < p.pairs;
            at[n] = place<1>(p, has[n] ? unit : 0);
            w[n][0] = norm ? weight_at(p, side, at[n].a) : 1.0f;
            w[n][1] = norm ? weight_at(p, side, at[n].b) : 1.0f;
        }
    }
};

template <bool NORM> __global__ void __launch_bounds__(kThreads) rotary_forward_kernel(const __grid_constant__ RotaryParams p)
{
    using T = __nv_bfloat16;
    __shared__ Pairs pairs;
    constexpr int kAhead = 4;                         // heads in flight
    const bool keys = blockIdx.x >= p.side[0].blocks;
    const Side &side = p.side[keys];
    const Share me(p, side.heads);
    const RowAt row(p, (blockIdx.x - (keys ? p.side[0].blocks : 0u)) * rows_of_block(p) + me.row);
    const Own own(p, side, me.lane, NORM);
    const T *const src = row.in<T>(side.x);
    T *const dst = row.in<T>(side.out);
    const float inverse_dim = 1.0f / float(p.dim);
    float c[kOwn], s[kOwn];
    for (int j0 = 0; j0 < me.turns; j0 += kAhead) {
        T x[kAhead][kOwn][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int head = me.first + (j0 + i) * p.split;
#pragma unroll
            for (int n = 0; n < kOwn; ++n)
                if (row.there && head < side.heads && own.has[n]) {
                    x[i][n][0] = src[head * side.x.head + own.at[n].a];
                    x[i][n][1] = src[head * side.x.head + own.at[n].b];
                }
        }
        if (j0 == 0) {                                // the first loads are under way
            pairs.fill(p);
            __syncthreads();
            Angles angles{p, pairs, row, position_at(p, row, pairs.axis[me.lane]), pairs.axis[me.lane]};
#pragma unroll
            for (int n = 0; n < kOwn; ++n) angles.at(min(me.lane + n * p.lanes, kMaxPairs - 1), &c[n], &s[n]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int head = me.first + (j0 + i) * p.split;
            const bool work = row.mine && head < side.heads;
            float f[kOwn][2], sum = 0.0f, r = 1.0f;
#pragma unroll
            for (int n = 0; n < kOwn; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    f[n][e] = work && row.there && own.has[n] ? to_float(x[i][n][e]) : 0.0f;
                    sum = fmaf(f[n][e], f[n][e], sum);
                }
            if constexpr (NORM) r = rsqrtf(fmaf(group_sum(sum, p.lanes), inverse_dim, p.eps));
            if (!work) continue;
            T *const at = dst + head * side.out.head;
#pragma unroll
            for (int n = 0; n < kOwn; ++n) {
                if (!own.has[n]) continue;
                const float a = NORM ? f[n][0] * r * own.w[n][0] : f[n][0], b = NORM ? f[n][1] * r * own.w[n][1] : f[n][1];
                at[own.at[n].a] = from_float<T>(!row.there ? 0.0f : own.turned[n] ? fmaf(a, c[n], -b * s[n]) : a);
                at[own.at[n].b] = from_float<T>(!row.there ? 0.0f : own.turned[n] ? fmaf(b, c[n], a * s[n]) : b);
            }
        }
    }
}

template <bool PADDED> __global__ void __launch_bounds__(kThreads, kResident) rotary_backward_kernel(const __grid_constant__ RotaryParams p)
{
    using T = __nv_bfloat16;
    __shared__ Pairs pairs;
    __shared__ float sums[kWarps * OMNI_ROTARY_MAX_DIM];
    constexpr int kAhead = 2;
    let_next_begin(p.overlap);
    const bool keys = blockIdx.x >= p.side[0].blocks;
    const Side &side = p.side[keys];
    const unsigned block = blockIdx.x - (keys ? p.side[0].blocks : 0u);
    const int heads = side.heads, lane = threadIdx.x % p.lanes;
    const Own own(p, side, lane, true);
    const float inverse_dim = 1.0f / float(p.dim);
    __shared__ Sequences sequences[1];
    const Sequences *const seq = sequences;
    pairs.fill(p);
    if constexpr (PADDED) sequences->fill(p);
    __syncthreads();
    float dw[kOwn][2] = {}, c[kOwn], s[kOwn];
    bool fresh = true;
    for (Walk<PADDED> now(p, seq, block, side.blocks, heads); now.left > 0;) {
        const RowAt row(p, now.row(p, seq));
        const T *const src = row.in<T>(side.x) + now.head * side.x.head, *const grad = row.in<T>(side.dy) + now.head * side.dy.head;
        T *const dst = row.in<T>(side.out) + now.head * side.out.head;
        const int turns = min(min(kAhead, now.left), heads - now.head);
        T x[kAhead][kOwn][2], y[kAhead][kOwn][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int n = 0; n < kOwn; ++n)
                if (row.there && i < turns && own.has[n]) {
                    x[i][n][0] = src[i * side.x.head + own.at[n].a];
                    x[i][n][1] = src[i * side.x.head + own.at[n].b];
                    y[i][n][0] = grad[i * side.dy.head + own.at[n].a];
                    y[i][n][1] = grad[i * side.dy.head + own.at[n].b];
                }
        if (fresh) {
            Angles angles{p, pairs, row, position_at(p, row, pairs.axis[lane]), pairs.axis[lane]};
#pragma unroll
            for (int n = 0; n < kOwn; ++n) angles.at(min(lane + n * p.lanes, kMaxPairs - 1), &c[n], &s[n]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (i >= turns) break;
            float f[kOwn][2], g[kOwn][2], square = 0.0f, dot = 0.0f;
#pragma unroll
            for (int n = 0; n < kOwn; ++n) {
                f[n][0] = f[n][1] = g[n][0] = g[n][1] = 0.0f;
                if (row.there && own.has[n]) {
                    const float ya = to_float(y[i][n][0]), yb = to_float(y[i][n][1]);
                    f[n][0] = to_float(x[i][n][0]);
                    f[n][1] = to_float(x[i][n][1]);
                    g[n][0] = own.turned[n] ? fmaf(ya, c[n], yb * s[n]) : ya;
                    g[n][1] = own.turned[n] ? fmaf(yb, c[n], -ya * s[n]) : yb;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    square = fmaf(f[n][e], f[n][e], square);
                    dot = fmaf(f[n][e] * own.w[n][e], g[n][e], dot);
                }
            }
            const float2 both = group_sum(make_float2(square, dot), p.lanes);
            if (!row.mine) continue;
            const float r = rsqrtf(fmaf(both.x, inverse_dim, p.eps)), pull = both.y * inverse_dim * r * r;
            T *const at = dst + i * side.out.head;
#pragma unroll
            for (int n = 0; n < kOwn; ++n) {
                if (!own.has[n]) continue;
                float dx[2] = {0.0f, 0.0f};
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (row.there) {
                        dw[n][e] = fmaf(g[n][e], f[n][e] * r, dw[n][e]);
                        dx[e] = r * fmaf(-f[n][e], pull, g[n][e] * own.w[n][e]);
                    }
                at[own.at[n].a] = from_float<T>(dx[0]);
                at[own.at[n].b] = from_float<T>(dx[1]);
            }
        }
        now.next(p, seq, heads, turns);
        fresh = now.head == 0;
    }
    if constexpr (PADDED)
        absent_rows(p, side, block, [&](const RowAt &row) {
            T *to = row.in<T>(side.out);
            for (int head = 0; head < heads; ++head, to += side.out.head)
#pragma unroll
                for (int n = 0; n < kOwn; ++n)
                    if (own.has[n]) to[own.at[n].a] = to[own.at[n].b] = from_float<T>(0.0f);
        });
#pragma unroll
    for (int n = 0; n < kOwn; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float v = warp_groups_sum(dw[n][e], p.lanes);
            if (int(threadIdx.x % 32) < p.lanes && own.has[n]) sums[threadIdx.x / 32 * p.dim + (e ? own.at[n].b : own.at[n].a)] = v;
        }
    __syncthreads();
    put_partial(p, sums, side.partial + (unsigned long long)block * p.dim);
}

struct WeightParams {
    const float *partial[2];
    void *grad[2];
    unsigned blocks[2];
    int dim, bf16;
};
// The blocks' sums of eight channels of a side: a thread's share of the blocks each, lanes and warps in order.
constexpr int kJoin = 8;
__global__ void __launch_bounds__(1024) rotary_weight_kernel(const WeightParams p)
{
    __shared__ float sum[32][kJoin];
    const int side = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32, ch = blockIdx.x * kJoin + threadIdx.x % kJoin;
    const float *const partial = side ? p.partial[1] : p.partial[0];
    const unsigned blocks = side ? p.blocks[1] : p.blocks[0];
    wait_for_previous();
    float v = 0.0f;
    if (ch < p.dim)
        for (unsigned b = threadIdx.x / kJoin; b < blocks; b += 1024 / kJoin) v += partial[(unsigned long long)b * p.dim + ch];
    for (int o = kJoin; o < 32; o *= 2) v += __shfl_xor_sync(~0u, v, o);
    if (lane < kJoin) sum[warp][lane] = v;
    __syncthreads();
    if (warp > 0) return;
    v = 0.0f;
    for (int w = lane / kJoin; w < 32; w += 32 / kJoin) v += sum[w][lane % kJoin];
    for (int o = kJoin; o < 32; o *= 2) v += __shfl_xor_sync(~0u, v, o);
    if (lane < kJoin && ch < p.dim) {
        if (p.bf16) static_cast<__nv_bfloat16 *>(side ? p.grad[1] : p.grad[0])[ch] = __float2bfloat16_rn(v);
        else static_cast<float *>(side ? p.grad[1] : p.grad[0])[ch] = v;
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
        if (a.stride >= (1ull << 40) || (written && a.stride > (1ull << 57) / unsigned(a.extent))) return OMNI_ERR_TOO_LARGE;
        if (written && a.stride < uint64_t(r->dim)) return OMNI_ERR_BAD_CONFIG;      // rows that a result would write twice
    }
    return OMNI_OK;
}

// Whether what a call writes is written once.  Two head vectors of dim elements share one if their distance, a sum of one multiple of each stride, is below dim
// either way.  The strides are tried from the largest on, and of each the multiples that the smaller ones can still bring back: where the smaller
// ones' extents fit into a stride, as in any slice of a larger tensor, that is three multiples at most.
class Distances {
    struct Axis { int64_t stride, low, high; } axis[6];      // multiples from low to high
    int64_t low[7], high[7], dim;                     // what the axes from i on add at least and at most
    int count = 0, steps = 1 << 16;                   // layouts that take more are refused

    bool meet(int i, int64_t from, bool apart)
    {
        if (from + low[i] >= dim || from + high[i] <= -dim) return false;
        if (i == count) return apart;
        if (--steps < 0) return true;
        const Axis &a = axis[i];
        if (from == 0 && a.stride + low[i + 1] >= dim && high[i + 1] - a.stride <= -dim) return meet(i + 1, 0, apart);       // only 0 of them
        // below (dim - from - low) / stride and above (-dim - from - high) / stride: by division towards 0, one too many at either end
        const int64_t first = (-dim - from - high[i + 1]) / a.stride - 1, last = (dim - from - low[i + 1]) / a.stride + 1;
        for (int64_t m = first > a.low ? first : a.low; m <= a.high && m <= last; ++m)
            if (meet(i + 1, from + m * a.stride, apart || m != 0)) return true;
        return false;
    }

public:
    explicit Distances(const omni_rotary *r) : dim(r->dim) {}
    // Multiples of a stride from low to high; those of one stride in two results are one axis, of two axes of one result they are not.
    void add(uint64_t stride, int64_t from, int64_t to, bool join)
    {
        if (from == to) return;
        int i = 0;
        while (i < count && axis[i].stride > int64_t(stride)) ++i;
        if (!join || i == count || axis[i].stride != int64_t(stride)) {
            for (int j = count++; j > i; --j) axis[j] = axis[j - 1];
            axis[i] = {int64_t(stride), 0, 0};
        }
        axis[i].low += from;
        axis[i].high += to;
    }
    // What a result's indices add to a distance that begins (away) or ends (back) at one of its vectors.
    void add(const omni_rotary *r, const omni_attn_view *v, int heads, int away, int back, bool join)
    {
        const std::pair<int, uint64_t> all[3] = {{r->batch, v->batch}, {r->length, v->row}, {heads, v->head}};
        for (const auto &[extent, stride] : all) add(stride, -int64_t(extent - 1) * away, int64_t(extent - 1) * back, join);
    }
    // apart: the vectors are of two results, `from` apart at first.
    bool meet(int64_t from, bool apart)
    {
        low[count] = high[count] = 0;
        for (int i = count - 1; i >= 0; --i) {
            low[i] = low[i + 1] + axis[i].low * axis[i].stride;
            high[i] = high[i + 1] + axis[i].high * axis[i].stride;
        }
        return meet(0, from, apart);
    }
};
int check_written_once(const omni_rotary *r, const omni_attn_view *q, const omni_attn_view *k)
{
    if (uint64_t(r->batch) * uint64_t(r->length) == 0) return OMNI_OK;
    for (const auto &[v, heads] : {std::pair(q, r->heads), std::pair(k, r->kv_heads)}) {
        Distances own(r);
        own.add(r, v, heads, 1, 1, false);
        if (own.meet(0, false)) return OMNI_ERR_BAD_CONFIG;
    }
    Distances both(r);
    both.add(r, q, r->heads, 1, 0, true);
    both.add(r, k, r->kv_heads, 0, 1, true);
    const int64_t bytes = int64_t(reinterpret_cast<uintptr_t>(k->data) - reinterpret_cast<uintptr_t>(q->data));
    return both.meet(bytes / (r->dtype == OMNI_BF16 ? 2 : 4), true) ? OMNI_ERR_BAD_CONFIG : OMNI_OK;
}

View view_of(const omni_rotary *r, const omni_attn_view *v, int heads)
{
    return {v->data, r->batch > 1 ? v->batch : 0, r->length > 1 ? v->row : 0, heads > 1 ? v->head : 0};
}

// Whether every head vector of an operand begins on a boundary of `to` bytes.
bool on_boundaries(const omni_rotary *r, const View &v, size_t to)
{
    const size_t size = r->dtype == OMNI_BF16 ? 2 : 4;
    return aligned(v.data, to) && v.batch * size % to == 0 && v.row * size % to == 0 && v.head * size % to == 0;
}

// The bytes of an access: the most that every head vector, and every half of one, allows; 0: element by element, which floats never need.  Halves that begin on no group of
// eight run gathered where an access would be one element: forward, 5 x 2630, 32 heads on 8 of 64, float with 9 pairs turned 77 us gathered, 106 by 4
// bytes; bfloat16 with 9 53, element by element 163, but with 20 56, by 8 bytes 37, and 2 x 4096 of 128 with 62 51, by 4 bytes 37.
// Backward the float ones are 231 and 157, so there only odd halves of bfloat16 are left to it (107, element by element 225).
int grain_of(const omni_rotary *r, std::initializer_list<const View *> views, bool backward)
{
    const auto all_on = [&](size_t to) {
        for (const View *v : views)
            if (!on_boundaries(r, *v, to)) return false;
        return true;
    };
    const bool whole = r->dim % 16 == 0 && all_on(16);
    if (whole && (r->interleaved || r->pairs % 8 == 0)) return 16;
    for (int grain = 8; grain >= 4; grain /= 2) {
        const int each = grain / (r->dtype == OMNI_BF16 ? 2 : 4);
        if (whole && !backward && each == 1) return 16;
        if (r->dim % each == 0 && (r->interleaved || r->pairs % each == 0) && all_on(grain)) return grain;
    }
    return whole ? 16 : 0;
}

// The launch: lanes of a head vector, how rows and heads are dealt, blocks of either side.
struct Shape {
    int lanes, split;
    unsigned bundles, blocks[2];
};
int lanes_of(const omni_rotary *r, int grain)
{
    int units = r->dim / 2;
    if (grain) {
        const int each = grain / (r->dtype == OMNI_BF16 ? 2 : 4), rest = (r->dim - 2 * r->pairs) / each;
        units = grain == 16 || r->interleaved ? (r->dim + 15) / 16 : (r->pairs + (rest + 1) / 2 * each + 7) / 8;
    }
    int lanes = 1;
    while (lanes < units && lanes < 32) lanes *= 2;
    return lanes;
}

// Forward: a group has all heads of a row, so that every angle is made once; where there are few rows (decoding) groups share a row and
// make its angles each.
Shape forward_shape(const omni_rotary *r, int grain, int sms)
{
    Shape s = {lanes_of(r, grain), 1, 0, {0, 0}};
    const uint64_t rows = uint64_t(r->batch) * uint64_t(r->length);
    const int groups = kThreads / s.lanes, most = r->heads > r->kv_heads ? r->heads : r->kv_heads;
    while (s.split < groups && s.split < most && rows * s.split < uint64_t(sms) * groups * 2) s.split *= 2;
    const uint64_t of_block = groups / s.split;
    s.blocks[0] = s.blocks[1] = unsigned((rows + of_block - 1) / of_block);
    return s;
}

// Backward: as many blocks as are resident at once, shared between the sides by the work of a row, whose angles are about that of two
// heads; where there is less work a warp has one turn.
Shape backward_shape(const omni_rotary *r, int grain, int sms)
{
    Shape s = {lanes_of(r, grain), 1, 0, {0, 0}};
    const uint64_t rows = uint64_t(r->batch) * uint64_t(r->length), of_bundle = 32 / s.lanes;
    s.bundles = unsigned((rows + of_bundle - 1) / of_bundle);
    const uint64_t all = uint64_t(sms) * kResident, q = r->heads + 2, k = r->kv_heads + 2;
    uint64_t share = all * q / (q + k);
    share = share < 1 ? 1 : share > all - 1 ? all - 1 : share;
    const uint64_t q_most = (s.bundles * uint64_t(r->heads) + kWarps - 1) / kWarps, k_most = (s.bundles * uint64_t(r->kv_heads) + kWarps - 1) / kWarps;
    s.blocks[0] = unsigned(q_most < share ? q_most : share);
    s.blocks[1] = unsigned(k_most < all - share ? k_most : all - share);
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
    // division of what is below 2^31 by a number of up to 31 bits: ceil(2^(32 + shift) / length) - 2^32
    for (p->shift = 0; (1ull << p->shift) < p->length; ++p->shift) {}
    p->magic = unsigned(((1ull << 32) * ((1ull << p->shift) - p->length)) / p->length + 1);
    p->dim = r->dim;
    p->pairs = r->pairs;
    p->axes = r->axes;
    p->lanes = s.lanes;
    p->split = s.split;
    p->bundles = s.bundles;
    p->batch = r->batch;
    p->padded = r->lengths && r->batch <= kMostSequences;
    p->wide_positions = r->position_type == OMNI_I64;
    p->bf16_weight = r->weight_dtype == OMNI_BF16;
    p->interleaved = r->interleaved != 0;
    p->eps = r->eps;
    p->backwards = backwards;
    for (int i = 0; i < r->pairs; ++i) {
        const long double turns = (long double)r->frequency[i] * 0.159154943091895335768883763372514362L;     // 1 / (2 pi)
        const long double part = turns - floorl(turns);
        p->frequency[i] = part < 1.0L ? (unsigned long long)ldexpl(part, 64) : 0;
        p->axis[i] = r->axis ? (unsigned char)r->axis[i] : 0;
    }
    p->side[0].heads = r->heads;
    p->side[1].heads = r->kv_heads;
    p->side[0].weight = r->q_weight;
    p->side[1].weight = r->k_weight;
    for (int i = 0; i < 2; ++i) p->side[i].blocks = s.blocks[i];
}

constexpr int kMostShared = 112 * 1024;               // dynamic shared memory of a block: two fit an SM

int enqueue(omni_ctx *ctx, void (*kernel)(RotaryParams), const RotaryParams &p, size_t smem, cudaStream_t s)
{
    const int rc = smem > 32 * 1024 ? context_shared(ctx, reinterpret_cast<const void *>(kernel), kMostShared) : OMNI_OK;
    if (rc != OMNI_OK) return rc;
    kernel<<<p.side[0].blocks + p.side[1].blocks, kThreads, smem, s>>>(p);
    return context_launched(ctx, int(cudaGetLastError()));
}

template <typename T, bool NORM, int GRAIN> void (*forward_kernel(const RotaryParams &p))(RotaryParams)
{
    if (p.interleaved) return rotary_forward_wide_kernel<T, kNeighbours, NORM, GRAIN>;
    if constexpr (GRAIN == 16)
        if (p.pairs % 8) return rotary_forward_wide_kernel<T, kGathered, NORM, GRAIN>;
    return rotary_forward_wide_kernel<T, kHalves, NORM, GRAIN>;
}
template <typename T, bool NORM> int enqueue_forward(omni_ctx *ctx, const RotaryParams &p, int grain, cudaStream_t s)
{
    if constexpr (sizeof(T) == 2)
        if (!grain) return enqueue(ctx, rotary_forward_kernel<NORM>, p, 0, s);
    return enqueue(ctx, grain == 16 ? forward_kernel<T, NORM, 16>(p) : grain == 8 ? forward_kernel<T, NORM, 8>(p) : forward_kernel<T, NORM, 4>(p), p,
                   ForwardRing<T>::kBytes, s);
}

template <typename T, bool PADDED, int GRAIN> void (*backward_kernel(const RotaryParams &p))(RotaryParams)
{
    if (p.interleaved) return rotary_backward_wide_kernel<T, kNeighbours, PADDED, GRAIN>;
    if constexpr (GRAIN == 16 && sizeof(T) == 2)
        if (p.pairs % 8) return rotary_backward_wide_kernel<T, kGathered, PADDED, GRAIN>;
    return rotary_backward_wide_kernel<T, kHalves, PADDED, GRAIN>;
}
template <typename T, bool PADDED> int enqueue_backward(omni_ctx *ctx, const RotaryParams &p, int grain, cudaStream_t s)
{
    if constexpr (sizeof(T) == 2)
        if (!grain) return enqueue(ctx, rotary_backward_kernel<PADDED>, p, 0, s);
    return enqueue(ctx, grain == 16 ? backward_kernel<T, PADDED, 16>(p) : grain == 8 ? backward_kernel<T, PADDED, 8>(p) : backward_kernel<T, PADDED, 4>(p), p,
                   BackwardRing<T>::kBytes, s);
}
template <typename T> int enqueue_backward(omni_ctx *ctx, const RotaryParams &p, int grain, cudaStream_t s)
{
    return p.padded ? enqueue_backward<T, true>(ctx, p, grain, s) : enqueue_backward<T, false>(ctx, p, grain, s);
}

// One pass over both sides without sums: the forward call, and the gradient where there are no weights.
int rotate(omni_ctx *ctx, const omni_rotary *r, const omni_attn_view *const (&in)[2], const omni_attn_view *const (&out)[2], bool backwards,
           const ContextDevice &dev, void *stream)
{
    RotaryParams p;
    for (int i = 0; i < 2; ++i) {
        const int heads = i ? r->kv_heads : r->heads;
        p.side[i] = {view_of(r, in[i], heads), {}, view_of(r, out[i], heads), nullptr, nullptr, 0, 0};
    }
    const int grain = grain_of(r, {&p.side[0].x, &p.side[0].out, &p.side[1].x, &p.side[1].out}, false);
    fill(&p, r, forward_shape(r, grain, dev.sm_count), backwards);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool norm = r->q_weight && !backwards;
    if (r->dtype == OMNI_BF16)
        return norm ? enqueue_forward<__nv_bfloat16, true>(ctx, p, grain, s) : enqueue_forward<__nv_bfloat16, false>(ctx, p, grain, s);
    return norm ? enqueue_forward<float, true>(ctx, p, grain, s) : enqueue_forward<float, false>(ctx, p, grain, s);
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
    if (rc == OMNI_OK) rc = check_written_once(r, q_out, k_out);
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
    rc = check_written_once(r, dq, dk);
    if (rc != OMNI_OK) return rc;
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
        for (int i = 0; i < 2; ++i) {
            const int heads = i ? r->kv_heads : r->heads;
            p.side[i] = {view_of(r, x[i], heads), view_of(r, dy[i], heads), view_of(r, dx[i], heads), nullptr, nullptr, 0, 0};
        }
        const int grain = grain_of(r, {&p.side[0].x, &p.side[0].dy, &p.side[0].out, &p.side[1].x, &p.side[1].dy, &p.side[1].out}, true);
        const Shape shape = backward_shape(r, grain, dev.sm_count < kMostSms ? dev.sm_count : kMostSms);
        fill(&p, r, shape, false);
        p.overlap = dev.overlap;
        p.side[0].partial = static_cast<float *>(workspace);
        p.side[1].partial = p.side[0].partial + uint64_t(shape.blocks[0]) * r->dim;
        for (int i = 0; i < 2; ++i) {
            w.partial[i] = p.side[i].partial;
            w.blocks[i] = shape.blocks[i];
        }
        rc = r->dtype == OMNI_BF16 ? enqueue_backward<__nv_bfloat16>(ctx, p, grain, s) : enqueue_backward<float>(ctx, p, grain, s);
        if (rc != OMNI_OK) return rc;
    }
    Dependent launch(dev, dim3((r->dim + kJoin - 1) / kJoin, 2), 1024, 0, s);
    if (empty) launch.cfg.numAttrs = 0;
    return context_launched(ctx, int(cudaLaunchKernelEx(&launch.cfg, rotary_weight_kernel, w)));
}

}  // extern "C"
