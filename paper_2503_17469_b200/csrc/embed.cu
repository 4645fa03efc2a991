// Embedding lookup with scaling, and its dense gradient by sorted tokens.
//
// Lookup: out_i = s * W[t_i].  Pure gather: the floor is the n rows written plus the distinct rows
// read.  A group of lanes owns a row, 8 elements (16 or 32 bytes) per lane and access, two rows in flight.
// 65536 rows of 1024 bfloat16 from a table of 50257, Zipf: 33 us a call, 5.1 TB/s.  Rows that no 16-byte access fits go element
// by element: of 1023 88 us, of 1025 94 us.
//
// Gradient: dW_v = s * sum_{t_i = v} dy_i.  Scattered adds with atomics would leave the order of
// the sum to chance, so the tokens are sorted first and a row's sum is then written by one owner that adds its terms
// in order:
//   1. sort_tokens: a stable radix sort of (position, id) by nine bits a pass, by one cluster of up to eight CTAs.  A
//      CTA takes a consecutive stretch of the list, a warp a consecutive part of that; counts per (warp,
//      digit) in shared memory, joined over the cluster through distributed shared memory, give every token its place;
//      lanes of one digit rank by lane.  The other CTAs of the launch set the whole table to zero meanwhile: a row
//      with tokens is written twice, but the sort, which waits more than it moves, is hidden.
//   2. sum_runs: the sorted list is cut into blocks of 32, whatever the ids, so that a token that
//      fills a tenth of the batch is spread over as many owners as it needs.  A group of lanes adds a
//      block's rows in registers and writes a row where the id changes; runs that cross blocks are joined
//      in block order in shared memory, those that cross CTAs leave a float partial in the workspace.
//   3. join_runs: the CTA in which such a run starts adds its partials in order and writes the row.
// 32768 bfloat16 rows of 768 into 50257 float rows: 29.6 us sort and zeros (154 MB), 27.5 us sums, 5 us joins, 63.6 us a call
// against a floor of 31 (each input read, each output written once): the sort, 23 us by itself, waits on its barriers; the sums
// wait on their loads (22 % of DRAM, and at four CTAs an SM their rows in flight spill 108 bytes a thread) while the zeros leave L2.
// Added to the table 64 us; rows of 767 or 769, element by element, 118-120 us.  Small calls are bound by their three launches.
// Tried: every CTA counting its own ids among all tokens 30 us and as much skew as the tokens have; matches by
// __match_any_sync 31.6 against 28.5 us with nine ballots; one launch of one cluster for small batches 30.7 against 20.5 us.
#include "context.h"
#include "vector.cuh"

namespace omni {
namespace {

constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortPerCta = 1024;   // tokens that make another CTA worth its barriers
constexpr int kBlock = 32;          // sorted tokens per block
constexpr int kThreads = 256;
constexpr int kRunLanes = 32;       // of a block of sorted tokens, however narrow the rows: 32768 rows of 8 floats took 126 us with a lane a block
constexpr int kRunsPer = kThreads / kRunLanes;      // blocks per CTA
constexpr int kBatch = 4;           // accesses in flight per lane
constexpr int kJoinAhead = 8;       // partials in flight of a run that is joined

struct Entry { int pos, id; };      // a token's place in the batch, and its id

template <typename I>
__device__ __forceinline__ int token_id(const void *tokens, long long i, int vocab, long long padding)
{
    const long long t = load_index<I>(tokens, i);
    return t >= 0 && t < vocab && t != padding ? int(t) : -1;
}

// Eight elements of a row, or one: kept as loaded, so that more of them are in flight per register.
template <typename T, bool WIDE> struct RawRow;
template <> struct RawRow<__nv_bfloat16, true> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { u = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float *f) const { widen(u, f); }
    __device__ __forceinline__ void add(float *acc) const
    {
        float f[kGroup];
        widen(u, f);
#pragma unroll
        for (int e = 0; e < kGroup; ++e) acc[e] += f[e];
    }
};
template <> struct RawRow<float, true> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p)
    {
        float f[kGroup];
        load_group(p, f);
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ void get(float *f) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void add(float *acc) const
    {
        acc[0] += a.x; acc[1] += a.y; acc[2] += a.z; acc[3] += a.w;
        acc[4] += b.x; acc[5] += b.y; acc[6] += b.z; acc[7] += b.w;
    }
};
template <typename T> struct RawRow<T, false> {
    T x;
    __device__ __forceinline__ void load(const T *p) { x = *p; }
    __device__ __forceinline__ void get(float *f) const { f[0] = to_float(x); }
    __device__ __forceinline__ void add(float *acc) const { acc[0] += to_float(x); }
};

// ---- lookup -------------------------------------------------------------------------------------

// `lanes` lanes take `each` rows in turn, two at a time.  WIDE: groups of 8 elements (dim a multiple of 8, rows 16-byte
// aligned), else single elements.
template <typename I, typename T, typename O, bool WIDE>
__global__ void __launch_bounds__(kThreads) embed_lookup_kernel(const void *tokens, long long n, const T *table,
                                                                unsigned long long table_stride, int vocab, int dim, float scale,
                                                                O *out, unsigned long long out_stride, int lanes, int each)
{
    constexpr int E = WIDE ? kGroup : 1, kPair = 2;
    const int per = kThreads / lanes, lane = threadIdx.x % lanes;
    const long long first = ((long long)blockIdx.x * per + threadIdx.x / lanes) * each;
    const long long last = first + each < n ? first + each : n;
    const int units = dim / E;
    for (long long i = first; i < last; i += kPair) {
        long long t[kPair];
#pragma unroll
        for (int r = 0; r < kPair; ++r) {
            t[r] = i + r < last ? load_index<I>(tokens, i + r) : -1;
            if (t[r] >= vocab) t[r] = -1;
        }
        for (int u = lane; u < units; u += lanes * kBatch) {
            RawRow<T, WIDE> x[kPair][kBatch];
#pragma unroll
            for (int r = 0; r < kPair; ++r)
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (t[r] >= 0 && u + b * lanes < units) x[r][b].load(table + (unsigned long long)t[r] * table_stride + (u + b * lanes) * E);
#pragma unroll
            for (int r = 0; r < kPair; ++r)
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int w = u + b * lanes;
                    if (i + r >= last || w >= units) continue;
                    float f[E] = {};
                    if (t[r] >= 0) x[r][b].get(f);
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] = t[r] >= 0 ? f[e] * scale : 0.0f;
                    O *dst = out + (unsigned long long)(i + r) * out_stride + w * E;
                    if constexpr (WIDE) store_group(dst, f);
                    else *dst = from_float<O>(f[0]);
                }
        }
    }
}

// ---- sort ---------------------------------------------------------------------------------------

struct SortParams {
    const void *tokens;
    long long n, padding;
    int vocab, passes;
    Entry *sorted, *other;       // the last pass ends in `sorted`
    int *total;                  // tokens that count
    int ranks;                   // CTAs that sort: the first cluster
    char *table;                 // what the others set to zero: vocab rows of row_bytes, table_stride bytes apart; or null
    unsigned long long row_bytes, table_stride;
    bool overlap;                // the next kernel may begin early
};

// The table set to zero by the CTAs rank = 0..ranks-1.  16-byte stores where rows allow them.
__device__ __forceinline__ void zero_table(const SortParams &p, long long rank, long long ranks)
{
    const bool packed = p.row_bytes == p.table_stride;
    const unsigned long long rows = packed ? 1 : p.vocab, bytes = packed ? p.row_bytes * p.vocab : p.row_bytes;
    const bool wide = (reinterpret_cast<uintptr_t>(p.table) | (packed ? 0 : p.table_stride)) % 16 == 0;
    const unsigned long long at = (unsigned long long)rank * blockDim.x + threadIdx.x, step = (unsigned long long)ranks * blockDim.x;
    if (packed) {
        char *t = p.table;
        const unsigned long long whole = wide ? bytes / 16 : 0;
        for (unsigned long long i = at; i < whole; i += step) __stcs(reinterpret_cast<uint4 *>(t) + i, make_uint4(0, 0, 0, 0));
        for (unsigned long long i = whole * 16 + 2 * at; i < bytes; i += 2 * step) *reinterpret_cast<unsigned short *>(t + i) = 0;
        return;
    }
    const unsigned long long warps = step / 32;
    for (unsigned long long r = at / 32; r < rows; r += warps) {
        char *t = p.table + r * p.table_stride;
        const unsigned long long whole = wide ? bytes / 16 : 0;
        for (unsigned long long i = threadIdx.x % 32; i < whole; i += 32) __stcs(reinterpret_cast<uint4 *>(t) + i, make_uint4(0, 0, 0, 0));
        for (unsigned long long i = whole * 16 + 2 * (threadIdx.x % 32); i < bytes; i += 64) *reinterpret_cast<unsigned short *>(t + i) = 0;
    }
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int load_remote(const int *cell, unsigned rank)
{
    unsigned at;
    int x;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(unsigned(__cvta_generic_to_shared(cell))), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
    return x;
}

// The lanes of a warp that have this lane's digit (-1: none).
__device__ __forceinline__ unsigned lanes_of(int digit)
{
    unsigned peers = __ballot_sync(~0u, digit >= 0);
#pragma unroll
    for (int bit = 0; bit < kDigitBits; ++bit) {
        const bool set = digit >> bit & 1;
        const unsigned b = __ballot_sync(~0u, set);
        peers &= set ? b : ~b;
    }
    return peers;
}

template <typename I>
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const SortParams p)
{
    extern __shared__ int hist[];                   // [kSortWarps][kDigits]: a warp's tokens, then its first place in the CTA's
    __shared__ int mine[kDigits], place_of[kDigits], warp_sum[kDigits / 32];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, ranks = p.ranks, rank = blockIdx.x;
    let_next_begin(p.overlap);
    if (rank >= ranks) {
        zero_table(p, rank - ranks, gridDim.x - ranks);
        return;
    }
    int *own = hist + warp * kDigits;
    long long m = p.n;
    const Entry *from = nullptr;
    for (int pass = 0; pass < p.passes; ++pass) {
        Entry *to = (p.passes - pass) % 2 == 1 ? p.sorted : p.other;
        const int shift = pass * kDigitBits;
        // this warp's part [first, last) of the list
        const long long part = ((m + ranks * kSortWarps - 1) / (ranks * kSortWarps) + 31) / 32 * 32;
        const long long first = ((long long)rank * kSortWarps + warp) * part, last = first + part < m ? first + part : m;
        auto fetch = [&](long long base, Entry (&e)[kBatch], int (&digit)[kBatch]) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const long long i = base + b * 32 + lane;
                e[b] = {-1, -1};
                if (i < last) {
                    if (!from) {
                        e[b] = {int(i), token_id<I>(p.tokens, i, p.vocab, p.padding)};
                    } else {
                        const int2 x = __ldcg(reinterpret_cast<const int2 *>(from + i));
                        e[b] = {x.x, x.y};
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) digit[b] = e[b].id >= 0 ? e[b].id >> shift & (kDigits - 1) : -1;
        };
        Entry e[kBatch];
        int digit[kBatch];
        unsigned peers[kBatch];
        fetch(first, e, digit);
        for (int i = tid; i < kSortWarps * kDigits / 4; i += kSortThreads) reinterpret_cast<int4 *>(hist)[i] = make_int4(0, 0, 0, 0);
        __syncthreads();
        for (long long base = first; base < last; base += 32 * kBatch) {
            if (base > first) fetch(base, e, digit);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (base + b * 32 >= last) break;
                peers[b] = lanes_of(digit[b]);      // one add per digit: half of a batch may have the same
                if (digit[b] >= 0 && (peers[b] & ((1u << lane) - 1u)) == 0) own[digit[b]] += __popc(peers[b]);
                __syncwarp();
            }
        }
        __syncthreads();
        // over the warps of a digit, over the CTAs, over the digits
        int before = 0, all = 0;
        if (tid < kDigits) {
            int c[kSortWarps], sum = 0;
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) c[w] = hist[w * kDigits + tid];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                hist[w * kDigits + tid] = sum;
                sum += c[w];
            }
            mine[tid] = sum;
            all = sum;
        }
        if (ranks > 1) {
            cluster_sync();
            if (tid < kDigits) {
                all = 0;
                for (int k = 0; k < ranks; ++k) {
                    const int c = load_remote(mine + tid, k);
                    if (k < rank) before += c;
                    all += c;
                }
            }
        }
        int inc = all;
        for (int o = 1; o < 32; o *= 2) {
            const int y = __shfl_up_sync(~0u, inc, o);
            if (lane >= o) inc += y;
        }
        if (tid < kDigits && lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        int total = 0;
#pragma unroll
        for (int w = 0; w < kDigits / 32; ++w) {
            if (w < warp) before += warp_sum[w];
            total += warp_sum[w];
        }
        if (tid < kDigits) place_of[tid] = before + inc - all;
        __syncthreads();
        const bool once = part <= 32 * kBatch;      // the batch of the first walk is still there
        for (long long base = first; base < last; base += 32 * kBatch) {
            if (!once) fetch(base, e, digit);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (base + b * 32 >= last) break;
                if (!once) peers[b] = lanes_of(digit[b]);
                const int rank_in = __popc(peers[b] & ((1u << lane) - 1u));
                if (digit[b] >= 0) to[place_of[digit[b]] + own[digit[b]] + rank_in] = e[b];
                __syncwarp();
                if (digit[b] >= 0 && rank_in == 0) own[digit[b]] += __popc(peers[b]);
                __syncwarp();
            }
        }
        m = total;
        from = to;
        // the next pass reads what the others wrote, and nobody leaves while `mine` may be read
        if (ranks > 1) cluster_sync();
        else __syncthreads();
    }
    if (rank == 0 && tid == 0) *p.total = int(m);
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
    const int *total;
    float *partial;             // [2 * CTAs along the list][padded dim]: the run that enters, the run that leaves
    int dim, padded;            // padded: dim rounded up to 8
    int slices;                 // of the columns, kRunLanes * E elements each
    float scale;
    int accumulate;
    bool overlap;               // the next kernel may begin early
    unsigned long long src_stride, dst_stride;
};

// A CTA takes kThreads / lanes consecutive blocks of the sorted list and one slice of the columns.
template <typename T, typename G, bool WIDE>
__global__ void __launch_bounds__(kThreads, 4) sum_runs_kernel(const RunParams p, const T *src, G *dst)
{
    constexpr int E = WIDE ? kGroup : 1;
    constexpr int kRowsAhead = !WIDE ? 16 : sizeof(T) == 2 ? 8 : 4;
    let_next_begin(p.overlap);
    wait_for_previous();
    __shared__ float enters[kThreads * E], leaves[kThreads * E];    // [block of the CTA][column of the slice]
    __shared__ int4 runs[kRunsPer];                                 // per block: first id, last id, see below
    constexpr int per = kRunsPer, cols = kRunLanes * E;
    const int lane = threadIdx.x % kRunLanes, mine = threadIdx.x / kRunLanes;
    const int slice = blockIdx.x % p.slices;
    const long long cta = blockIdx.x / p.slices;
    const int col = slice * cols + lane * E;
    const int total = *p.total;
    const long long begin = (cta * per + mine) * kBlock;
    if (cta * per * kBlock >= total) return;
    constexpr int kEnters = 1, kLeaves = 2, kWhole = 4;             // the run crosses the block's start, its end, fills it
    int how = 0, cur = -1, first_id = -1;
    if (begin < total) {
        const int end = begin + kBlock < total ? int(begin) + kBlock : total;
        first_id = cur = p.sorted[begin].id;
        bool open = begin > 0 && p.sorted[begin - 1].id == cur;
        const int next = end < total ? p.sorted[end].id : -1;
        if (open) how |= kEnters;
        float acc[E] = {};
        const bool inside = col < p.dim;
        for (int i = int(begin); i < end; i += kRowsAhead) {
            Entry en[kRowsAhead];
            RawRow<T, WIDE> x[kRowsAhead];
#pragma unroll
            for (int b = 0; b < kRowsAhead; ++b) en[b] = i + b < end ? p.sorted[i + b] : Entry{-1, -1};
#pragma unroll
            for (int b = 0; b < kRowsAhead; ++b)
                if (en[b].id >= 0 && inside) x[b].load(src + (unsigned long long)en[b].pos * p.src_stride + col);
#pragma unroll
            for (int b = 0; b < kRowsAhead; ++b) {
                if (en[b].id < 0) continue;
                if (en[b].id != cur) {
                    if (open) {
#pragma unroll
                        for (int e = 0; e < E; ++e) enters[mine * cols + lane * E + e] = acc[e];
                    } else if (inside) {
                        put_row<G, WIDE>(dst + (unsigned long long)cur * p.dst_stride, col, acc, p.scale, p.accumulate);
                    }
                    open = false;
                    cur = en[b].id;
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
                }
                if (inside) x[b].add(acc);
            }
        }
        if (next == cur) how |= kLeaves;
        if (open) how |= kWhole;                                    // one run from start to end: its sum is in `enters`
        if (open || next == cur) {
            float *to = (open ? enters : leaves) + mine * cols + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e) to[e] = acc[e];
        } else if (inside) {
            put_row<G, WIDE>(dst + (unsigned long long)cur * p.dst_stride, col, acc, p.scale, p.accumulate);
        }
    }
    if (lane == 0) runs[mine] = make_int4(first_id, cur, how, 0);
    __syncthreads();
    // the runs that cross blocks, in block order, a thread per group of E columns
    if (threadIdx.x >= kRunLanes || col >= p.dim) return;             // the first group's lanes: their columns are the CTA's
    float acc[E] = {};
    bool before = (runs[0].z & kEnters) != 0;                       // the run at hand began before the CTA
    for (int k = 0; k < per && (cta * per + k) * kBlock < total; ++k) {
        const int4 r = runs[k];
        if (r.z & kEnters) {
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += enters[k * cols + lane * E + e];
            if ((r.z & kWhole) && (r.z & kLeaves)) continue;
            if (before) {
#pragma unroll
                for (int e = 0; e < E; ++e) p.partial[2 * cta * p.padded + col + e] = acc[e];
            } else {
                put_row<G, WIDE>(dst + (unsigned long long)r.x * p.dst_stride, col, acc, p.scale, p.accumulate);
            }
            before = false;
        }
        if (r.z & kLeaves) {
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = leaves[k * cols + lane * E + e];
        }
    }
    const long long after = (cta + 1) * per * kBlock;
    if (after < total && (runs[per - 1].z & kLeaves)) {             // into the next CTA, as one that entered or one that leaves
#pragma unroll
        for (int e = 0; e < E; ++e) p.partial[(2 * cta + (before ? 0 : 1)) * p.padded + col + e] = acc[e];
    }
}

// A group per (CTA of sum_runs, slice): if a run starts there and goes on in the next, its partials are added.
template <typename G, bool WIDE>
__global__ void __launch_bounds__(kThreads) join_runs_kernel(const RunParams p, G *dst, long long ctas)
{
    constexpr int E = WIDE ? kGroup : 1;
    constexpr int per = kRunsPer, span = per * kBlock;
    const int lane = threadIdx.x % kRunLanes;
    const long long g = (long long)blockIdx.x * per + threadIdx.x / kRunLanes, cta = g / p.slices;
    const int col = (int(g % p.slices) * kRunLanes + lane) * E;
    wait_for_previous();
    const int total = *p.total;
    const long long edge = (cta + 1) * span;
    if (cta >= ctas || edge >= total || col >= p.dim) return;
    const int id = p.sorted[edge].id;
    if (p.sorted[edge - 1].id != id || (cta > 0 && p.sorted[cta * span - 1].id == id)) return;   // not crossed, or begun earlier
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = p.partial[(2 * cta + 1) * p.padded + col + e];
    for (long long b = cta + 1;; b += kJoinAhead) {
        bool goes_on[kJoinAhead];
        float x[kJoinAhead][E];
#pragma unroll
        for (int k = 0; k < kJoinAhead; ++k) {
            const long long at = (b + k) * span;                 // the run reaches CTA b + k if it has its first token
            goes_on[k] = at < total;
            if (goes_on[k]) {                                    // fetched before it is known to belong: one wait instead of two
                goes_on[k] = p.sorted[at].id == id;
#pragma unroll
                for (int e = 0; e < E; ++e) x[k][e] = p.partial[2 * (b + k) * p.padded + col + e];
            }
        }
        bool more = true;
#pragma unroll
        for (int k = 0; k < kJoinAhead; ++k) {
            more = more && goes_on[k];
            if (more) {
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += x[k][e];
            }
        }
        if (!more) break;
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

struct EmbedWorkspace { unsigned long long other, total, partial, bytes; };

EmbedWorkspace plan_workspace(uint64_t n, int32_t dim)
{
    EmbedWorkspace w;                 // the sorted list comes first
    w.other = round_up(n * sizeof(Entry), 256);
    w.total = 2 * w.other;
    w.partial = w.total + 256;
    const uint64_t ctas = (n + kRunsPer * kBlock - 1) / (kRunsPer * kBlock);      // of sum_runs along the list
    w.bytes = w.partial + 2 * ctas * round_up(dim, kGroup) * sizeof(float);
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
    // Several rows per group once every SM has enough, so that blocks come and go less often: 65536 rows of 1024 bfloat16 take
    // 33.1 us with four (34.8 with two, 34.4 with eight, 39.1 with sixteen; 47 with one row a group and one in flight).  One / two /
    // four from a cold L2, in the timer's steps of 2 us: 1000 x 1024 8 / 8 / 10, 6000 x 256 10 / 8 / 8, 20000 x 1024 20 / 16 / 18,
    // 40000 x 256 27 / 18 / 16, 131072 x 1024 94 / 68 / 61.
    const int each = n > uint64_t(dev.sm_count) * 16 * per ? 4 : n > uint64_t(dev.sm_count) * 4 * per ? 2 : 1;
    const unsigned grid = unsigned((n + uint64_t(per) * each - 1) / (uint64_t(per) * each));
    return with_index(index_type, [&](auto *ip) {
        return with_type(table_dtype, [&](auto *tp) {
            return with_type(out_dtype, [&](auto *op) {
                return with_flag(wide, [&](auto w) {
                    using I = std::remove_pointer_t<decltype(ip)>;
                    using T = std::remove_pointer_t<decltype(tp)>;
                    using O = std::remove_pointer_t<decltype(op)>;
                    embed_lookup_kernel<I, T, O, decltype(w)::value><<<grid, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
                        tokens, (long long)n, static_cast<const T *>(table), table_stride, vocab, dim, scale,
                        static_cast<O *>(out), out_stride, lanes, each);
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
    *bytes = plan_workspace(n, dim).bytes;
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
    const EmbedWorkspace w = plan_workspace(n, dim);
    if (workspace_bytes < w.bytes) return OMNI_ERR_TOO_LARGE;
    ContextDevice dev;
    rc = context_bind(ctx, &dev);
    if (rc != OMNI_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    SortParams o;
    o.tokens = tokens;
    o.n = (long long)n;
    o.padding = padding;
    o.vocab = vocab;
    o.passes = 1;
    while (o.passes < 4 && (uint64_t(vocab) - 1) >> (o.passes * kDigitBits) != 0) ++o.passes;
    o.sorted = reinterpret_cast<Entry *>(ws);
    o.other = reinterpret_cast<Entry *>(ws + w.other);
    o.total = reinterpret_cast<int *>(ws + w.total);
    o.ranks = 1;
    while (o.ranks < 8 && n > uint64_t(o.ranks) * kSortPerCta) o.ranks *= 2;
    o.table = static_cast<char *>(grad);
    o.row_bytes = uint64_t(dim) * element_size(grad_dtype);
    o.table_stride = vocab == 1 ? o.row_bytes : grad_stride * element_size(grad_dtype);
    // beside the sort: CTAs for the zeros, as many as find 64 KB each to write, two per SM at most
    int zero_ctas = 0;
    o.overlap = dev.overlap && n > 0;
    if (!accumulate) {
        const uint64_t want = o.row_bytes * vocab / 65536 + 1, most = 2ull * dev.sm_count;
        zero_ctas = int(round_up(want < most ? want : most, o.ranks));
        // Blocks of the sums that wait beside the sort and the zeros are there at once when those end, but take their place on the
        // SMs meanwhile: worth it while both are short.  Without / with an early start, us a call: 8192 tokens into 331 x 99 floats
        // 19.7 / 18.4, into 8192 x 128 29.2 / 28.6; 32768 tokens into 2048 x 128 36.7 / 38.4, into 8192 x 512 44.3 / 48.4; into 50257 x 768
        // 1500 tokens 44.8 / 51.6, 32768 62.9 / 70.3.  (Adding to the table, with nothing to set to zero: even at every size.)
        o.overlap = o.overlap && n <= 8 * kSortPerCta && o.row_bytes * vocab < (16u << 20);
    }
    rc = with_index(index_type, [&](auto *ip) {
        using I = std::remove_pointer_t<decltype(ip)>;
        const void *kernel = reinterpret_cast<const void *>(sort_tokens_kernel<I>);
        const int smem = kSortWarps * kDigits * int(sizeof(int));
        const int r = context_shared(ctx, kernel, smem);
        if (r != OMNI_OK) return r;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(o.ranks + zero_ctas);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = o.ranks;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        void *args[] = {&o};
        return context_launched(ctx, int(cudaLaunchKernelExC(&cfg, kernel, args)));
    });
    if (rc != OMNI_OK) return rc;
    const bool wide = dim % kGroup == 0 && wide_rows(grad_out, grad_out_dtype, grad_out_stride) &&
                      wide_rows(grad, grad_dtype, grad_stride);
    RunParams p;
    p.sorted = o.sorted;
    p.total = o.total;
    p.partial = reinterpret_cast<float *>(ws + w.partial);
    p.dim = dim;
    p.padded = int(round_up(dim, kGroup));
    const int cols = kRunLanes * (wide ? kGroup : 1);
    p.slices = (dim + cols - 1) / cols;
    p.scale = scale;
    p.accumulate = accumulate != 0;
    p.src_stride = grad_out_stride;
    p.dst_stride = grad_stride;
    constexpr int per = kRunsPer;
    const long long ctas = ((long long)n + per * kBlock - 1) / (per * kBlock);
    if (ctas == 0) return OMNI_OK;
    p.overlap = dev.overlap && ctas > 1;
    return with_type(grad_out_dtype, [&](auto *tp) {
        return with_type(grad_dtype, [&](auto *gp) {
            return with_flag(wide, [&](auto wd) {
                using T = std::remove_pointer_t<decltype(tp)>;
                using G = std::remove_pointer_t<decltype(gp)>;
                constexpr bool W = decltype(wd)::value;
                const T *src = static_cast<const T *>(grad_out);
                G *dst = static_cast<G *>(grad);
                Dependent sum(dev, dim3(unsigned(ctas * p.slices)), kThreads, 0, s);
                const int r = context_launched(ctx, int(cudaLaunchKernelEx(&sum.cfg, sum_runs_kernel<T, G, W>, p, src, dst)));
                if (r != OMNI_OK || ctas == 1) return r;
                Dependent join(dev, dim3(unsigned((ctas * p.slices + per - 1) / per)), kThreads, 0, s);
                return context_launched(ctx, int(cudaLaunchKernelEx(&join.cfg, join_runs_kernel<G, W>, p, dst, ctas)));
            });
        });
    });
}

}  // extern "C"
