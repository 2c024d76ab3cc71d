// Rows of a table, scaled, and their gradient by sorted ids: ne_embed_lookup, ne_embed_grad.
//
// Lookup: out[i] = scale * table[ids[i]].  A gather: bound by memory, 4 bytes of id and a row read and written
// per position.  A lane group takes four rows at a time, so that a wavefront has four wide loads in flight.
//
// Gradient: T[r] = sum over i with ids[i] = r of scale * grad[i].  Positions are sorted by id (stable radix sort, so
// the order of a row's terms is fixed by the ids alone), then every row of T is written by one lane group that adds
// its run of positions in registers: no atomics, no clearing pass, each gradient row read once and each table row
// written once.  A run of thousands of positions (ids are skewed: the most frequent of a text or a graph takes
// percents of all positions) would leave one lane group with all of it, so whole chunks of 16 sorted positions that
// name one row are summed first, by a launch of their own over all positions, and 256 at a time where a run is that
// long; a row's lane group then adds at most 60 single terms and sums, and one sum per 256 positions.
#include "ne_internal.h"
#include "ne_ops.h"

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16;          // sorted positions that are summed together where they name one row
constexpr int kSuper = 256;         // the same, one size up
constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 4;
constexpr int kSortRound = kSortThreads * kSortItems;
constexpr int kMostTiles = 128;     // workgroups of a sorting pass; each reads the counts of all
constexpr int kMostDigits = 1024;
constexpr int kSmallSort = 4096;    // ids that one workgroup sorts in LDS, in one launch
constexpr int kSmallBits = 8;
constexpr int kRowsPerGroup = 64;   // table rows of a workgroup of the rows launch

// ---------------------------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------------------------
struct LookupArgs {
    const void* table;
    const int32_t* ids;
    void* out;
    int64_t table_stride, out_stride, n;
    uint32_t num_rows;
    int32_t dim, chunks, lanes_log2;
    float scale;
};

// Chunk c of a row is V elements from min(c V, dim - V) on: the last one of a dim that V does not divide overlaps the
// one before it, and both write the same values there.
template <class TI, class TO, int V>
__global__ void __launch_bounds__(kThreads) lookup_kernel(LookupArgs a)
{
    constexpr int R = 4;
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), groups = kThreads >> a.lanes_log2;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * (R * groups) + (threadIdx.x >> a.lanes_log2);
    uint32_t id[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t i = first + r * groups;
        id[r] = i < a.n ? static_cast<uint32_t>(a.ids[i]) : 0xFFFFFFFFu;
    }
    for (int c = lane; c < a.chunks; c += lanes) {
        const int at = min(c * V, a.dim - V);
        float x[R][V];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (id[r] < a.num_rows) {
                load_vec<TI, V>(static_cast<const TI*>(a.table) + static_cast<int64_t>(id[r]) * a.table_stride + at, x[r]);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) x[r][e] = 0.0f;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t i = first + r * groups;
            if (i >= a.n) continue;
            // (zeros of ids that name no row stay zeros, whatever the scale's sign)
            if (id[r] < a.num_rows)
#pragma unroll
                for (int e = 0; e < V; ++e) x[r][e] *= a.scale;
            store_vec<TO, V>(static_cast<TO*>(a.out) + i * a.out_stride + at, x[r]);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// sorting: entries {key, position} by key, stable; key = id, or num_rows for ids that name no row
// ---------------------------------------------------------------------------------------------
struct SortArgs {
    const int32_t* ids;        // first pass
    const uint2* in;           // later passes
    uint2* out;
    uint32_t* hist;            // [passes][tiles][digits]
    uint32_t n, num_rows, tile_len, tiles;
    int32_t pass, passes, bits, shift;
};

__device__ __forceinline__ uint32_t key_of(int32_t id, uint32_t num_rows) { return min(static_cast<uint32_t>(id), num_rows); }

// Rank of each of this lane's items among the items of the same digit that its wavefront has seen, counts in
// count[digit]; items of a wavefront are taken in the order j, lane.
template <int ITEMS>
__device__ __forceinline__ void wave_ranks(const uint32_t (&digit)[ITEMS], const bool (&valid)[ITEMS], int bits, uint32_t* count,
                                           uint32_t (&rank)[ITEMS])
{
    const uint64_t below = (1ull << (threadIdx.x & 63)) - 1;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        uint64_t same = __ballot(valid[j]);
        for (int b = 0; b < bits; ++b) {
            const uint64_t ones = __ballot((digit[j] >> b) & 1);
            same &= (digit[j] >> b) & 1 ? ones : ~ones;
        }
        if (!valid[j]) same = 1ull << (threadIdx.x & 63);
        const int leader = __ffsll(static_cast<unsigned long long>(same)) - 1;
        uint32_t before = 0;
        if (valid[j] && leader == static_cast<int>(threadIdx.x & 63)) before = atomicAdd(&count[digit[j]], static_cast<uint32_t>(__popcll(same)));
        rank[j] = __shfl(before, leader, 64) + static_cast<uint32_t>(__popcll(same & below));
    }
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(SortArgs a)
{
    __shared__ uint32_t count[kMostDigits];
    const uint32_t digits = 1u << a.bits, mask = digits - 1;
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) {
        count[d] = 0;
        for (int p = 1; p < a.passes; ++p) a.hist[(static_cast<size_t>(p) * a.tiles + blockIdx.x) * digits + d] = 0;
    }
    __syncthreads();
    const uint32_t lo = blockIdx.x * a.tile_len, hi = min(lo + a.tile_len, a.n);
    for (uint32_t i = lo + threadIdx.x; i < hi; i += kSortThreads) atomicAdd(&count[key_of(a.ids[i], a.num_rows) & mask], 1u);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.hist[static_cast<size_t>(blockIdx.x) * digits + d] = count[d];
}

// Sum of all earlier threads' values (and of none of the later ones'); total over the workgroup in *total.
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t* wave_sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(s, o, 64);
        if (lane >= o) s += u;
    }
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += wave_sums[w];
    return before + s - v;
}

// One pass: where a tile's entries of a digit begin follows from the counts of all tiles, which each workgroup adds up
// by itself (at most 128 x 1024 words, in L2); the next pass's counts are made with integer additions, whose order
// changes nothing.
__global__ void __launch_bounds__(kSortThreads) sort_pass_kernel(SortArgs a)
{
    __shared__ uint32_t base[kMostDigits];
    __shared__ uint32_t count[kSortWaves][kMostDigits];
    __shared__ uint32_t wave_sums[kSortWaves];
    const uint32_t digits = 1u << a.bits, mask = digits - 1;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t* hist = a.hist + static_cast<size_t>(a.pass) * a.tiles * digits;
    // thread t has digits 2t and 2t + 1
    uint32_t total[2] = {0, 0}, mine[2] = {0, 0};
    for (int q = 0; q < 2; ++q) {
        const uint32_t d = 2 * threadIdx.x + q;
        if (d >= digits) break;
        for (uint32_t t = 0; t < a.tiles; ++t) {
            const uint32_t c = hist[static_cast<size_t>(t) * digits + d];
            if (t < blockIdx.x) mine[q] += c;
            total[q] += c;
        }
    }
    const uint32_t before = block_prefix(total[0] + total[1], wave_sums);
    if (2 * threadIdx.x < digits) {
        base[2 * threadIdx.x] = before + mine[0];
        if (2 * threadIdx.x + 1 < digits) base[2 * threadIdx.x + 1] = before + total[0] + mine[1];
    }
    uint32_t* next = a.hist + static_cast<size_t>(a.pass + 1) * a.tiles * digits;
    const uint32_t lo = blockIdx.x * a.tile_len, hi = min(lo + a.tile_len, a.n);
    for (uint32_t r0 = lo; r0 < hi; r0 += kSortRound) {
        for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) count[w][d] = 0;
        uint2 e[kSortItems];
        uint32_t digit[kSortItems], rank[kSortItems];
        bool valid[kSortItems];
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            const uint32_t i = r0 + wave * (64 * kSortItems) + j * 64 + lane;
            valid[j] = i < hi;
            e[j] = make_uint2(0, 0);
            if (valid[j]) e[j] = a.pass == 0 ? make_uint2(key_of(a.ids[i], a.num_rows), i) : a.in[i];
            digit[j] = (e[j].x >> a.shift) & mask;
        }
        __syncthreads();
        wave_ranks<kSortItems>(digit, valid, a.bits, count[wave], rank);
        __syncthreads();
        for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) {
            uint32_t at = base[d];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = count[w][d];
                count[w][d] = at;
                at += c;
            }
            base[d] = at;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSortItems; ++j)
            if (valid[j]) {
                const uint32_t to = count[wave][digit[j]] + rank[j];
                a.out[to] = e[j];
                if (a.pass + 1 < a.passes) atomicAdd(&next[static_cast<size_t>(to / a.tile_len) * digits + ((e[j].x >> (a.shift + a.bits)) & mask)], 1u);
            }
        __syncthreads();
    }
}

// All passes of up to kSmallSort ids by one workgroup.
__global__ void __launch_bounds__(kSortThreads) sort_small_kernel(SortArgs a)
{
    __shared__ uint2 buf[2][kSmallSort];
    __shared__ uint32_t count[kSortWaves][1 << kSmallBits];
    __shared__ uint32_t wave_sums[kSortWaves];
    constexpr int ITEMS = kSmallSort / kSortThreads;
    const uint32_t digits = 1u << a.bits, mask = digits - 1;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t per = (a.n + kSortThreads - 1) / kSortThreads;      // items of a lane; a wavefront's lie side by side
    for (uint32_t i = threadIdx.x; i < a.n; i += kSortThreads) buf[0][i] = make_uint2(key_of(a.ids[i], a.num_rows), i);
    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * a.bits;
        for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) count[w][d] = 0;
        __syncthreads();
        uint2 e[ITEMS];
        uint32_t digit[ITEMS], rank[ITEMS];
        bool valid[ITEMS];
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            const uint32_t i = (static_cast<uint32_t>(wave) * per + j) * 64 + lane;
            valid[j] = static_cast<uint32_t>(j) < per && i < a.n;
            e[j] = valid[j] ? buf[p & 1][i] : make_uint2(0, 0);
            digit[j] = (e[j].x >> shift) & mask;
        }
        wave_ranks<ITEMS>(digit, valid, a.bits, count[wave], rank);
        __syncthreads();
        uint32_t sum = 0;
        if (threadIdx.x < digits)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) sum += count[w][threadIdx.x];
        uint32_t at = block_prefix(sum, wave_sums);
        if (threadIdx.x < digits)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = count[w][threadIdx.x];
                count[w][threadIdx.x] = at;
                at += c;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (valid[j]) {
                const uint32_t to = count[wave][digit[j]] + rank[j];
                if (p + 1 < a.passes) buf[(p + 1) & 1][to] = e[j];
                else a.out[to] = e[j];
            }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------
// sums of runs
// ---------------------------------------------------------------------------------------------
struct GradArgs {
    const uint2* sorted;
    const void* grad;
    float* partial;            // [n / kChunk][dim]  sums of chunks that name one row; of 256 positions in the place of their first chunk
    void* table;
    int64_t grad_stride, table_stride;
    uint32_t n, num_rows;
    int32_t dim, chunks, lanes_log2;
    float scale;
};

// Terms of a run [s, e) of sorted positions: single positions up to a multiple of 16, sums of 16 up to a multiple of
// 256, sums of 256, sums of 16, single positions.
struct Run {
    uint32_t s, c0, u0, u1, c1, e;      // where each of the five parts ends or begins
    uint32_t terms;
};

__device__ __forceinline__ Run run_of(uint32_t s, uint32_t e)
{
    Run r;
    r.s = s; r.e = e;
    r.c0 = min((s + kChunk - 1) / kChunk * kChunk, e);
    r.c1 = max(e / kChunk * kChunk, r.c0);
    r.u0 = min((r.c0 + kSuper - 1) / kSuper * kSuper, r.c1);
    r.u1 = max(r.c1 / kSuper * kSuper, r.u0);
    r.terms = (r.c0 - r.s) + (r.u0 - r.c0) / kChunk + (r.u1 - r.u0) / kSuper + (r.c1 - r.u1) / kChunk + (r.e - r.c1);
    return r;
}

// Adds term t of the run to acc.
template <class TG, int V>
__device__ __forceinline__ void load_term(const GradArgs& a, const Run& r, uint32_t t, int at, float (&x)[V])
{
    uint32_t single = 0xFFFFFFFFu, chunk = 0;
    uint32_t k = r.c0 - r.s;
    if (t < k) {
        single = r.s + t;
    } else {
        t -= k;
        k = (r.u0 - r.c0) / kChunk;
        if (t < k) {
            chunk = r.c0 / kChunk + t;
        } else {
            t -= k;
            k = (r.u1 - r.u0) / kSuper;
            if (t < k) {
                chunk = r.u0 / kChunk + t * (kSuper / kChunk);
            } else {
                t -= k;
                k = (r.c1 - r.u1) / kChunk;
                if (t < k) chunk = r.u1 / kChunk + t;
                else single = r.c1 + (t - k);
            }
        }
    }
    if (single != 0xFFFFFFFFu)
        load_vec<TG, V>(static_cast<const TG*>(a.grad) + static_cast<int64_t>(a.sorted[single].y) * a.grad_stride + at, x);
    else
        load_vec<float, V>(a.partial + static_cast<int64_t>(chunk) * a.dim + at, x);
}

// Every `step`-th term of a run from `t` on, four in flight.
template <class TG, int V>
__device__ __forceinline__ void sum_terms(const GradArgs& a, const Run& r, uint32_t t, uint32_t step, int at, float (&acc)[V])
{
    for (; t + 3 * step < r.terms; t += 4 * step) {
        float x[4][V];
#pragma unroll
        for (int q = 0; q < 4; ++q) load_term<TG, V>(a, r, t + q * step, at, x[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += x[q][e];
    }
    for (; t < r.terms; t += step) {
        float x[V];
        load_term<TG, V>(a, r, t, at, x);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += x[e];
    }
}

// Writes scale * acc to chunk c of a row, added to what is there where it accumulates.  (The last chunk of a dim that V
// does not divide overlaps the one before: an addition must not be made twice.)
template <class TT, int V, bool ADD>
__device__ __forceinline__ void write_chunk(const GradArgs& a, uint32_t row, int c, int at, const float (&acc)[V])
{
    TT* to = static_cast<TT*>(a.table) + static_cast<int64_t>(row) * a.table_stride + at;
    float x[V];
    if (ADD && at != c * V) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (at + e >= c * V) {
                load_vec<TT, 1>(to + e, *reinterpret_cast<float(*)[1]>(&x[e]));
                x[e] = fmaf(a.scale, acc[e], x[e]);
                store_vec<TT, 1>(to + e, *reinterpret_cast<const float(*)[1]>(&x[e]));
            }
        return;
    }
    if (ADD) load_vec<TT, V>(to, x);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = ADD ? fmaf(a.scale, acc[e], x[e]) : a.scale * acc[e];
    store_vec<TT, V>(to, x);
}

// Sum over the lane groups of a workgroup, in the groups' order, for group 0.
template <int V>
__device__ __forceinline__ void join_groups(float (*lds)[V], int lanes_log2, float (&acc)[V])
{
    const int lanes = 1 << lanes_log2, groups = kThreads >> lanes_log2;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) lds[threadIdx.x][e] = acc[e];
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < lanes)
        for (int g = 1; g < groups; ++g)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += lds[threadIdx.x + g * lanes][e];
}

// Sums of 16 and of 256 sorted positions that name one row; a workgroup has 256 positions.
template <class TG, int V>
__global__ void __launch_bounds__(kThreads) chunk_sums_kernel(GradArgs a)
{
    __shared__ float lds[kThreads][V];
    const uint32_t k0 = blockIdx.x * kSuper, end = min(k0 + kSuper, a.n);
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log2, groups = kThreads >> a.lanes_log2;
    const uint32_t key = a.sorted[k0].x;
    if (key >= a.num_rows) return;
    if (end == k0 + kSuper && a.sorted[end - 1].x == key) {
        Run all;
        all.s = k0; all.c0 = all.u0 = all.u1 = all.c1 = all.e = end; all.terms = kSuper;
        for (int c0 = 0; c0 < a.chunks; c0 += lanes) {
            const int c = c0 + lane, at = min(min(c, a.chunks - 1) * V, a.dim - V);
            float acc[V] = {};
            sum_terms<TG, V>(a, all, group, groups, at, acc);
            join_groups<V>(lds, a.lanes_log2, acc);
            if (group == 0 && c < a.chunks) store_vec<float, V>(a.partial + static_cast<int64_t>(k0 / kChunk) * a.dim + at, acc);
        }
        return;
    }
    for (uint32_t k = k0 + group * kChunk; k + kChunk <= end; k += groups * kChunk) {
        const uint32_t row = a.sorted[k].x;
        if (row >= a.num_rows || a.sorted[k + kChunk - 1].x != row) continue;
        Run all;
        all.s = k; all.c0 = all.u0 = all.u1 = all.c1 = all.e = k + kChunk; all.terms = kChunk;
        for (int c = lane; c < a.chunks; c += lanes) {
            const int at = min(c * V, a.dim - V);
            float acc[V] = {};
            sum_terms<TG, V>(a, all, 0, 1, at, acc);
            store_vec<float, V>(a.partial + static_cast<int64_t>(k / kChunk) * a.dim + at, acc);
        }
    }
}

// First sorted position whose key is at least `key`.
__device__ __forceinline__ uint32_t lower_bound(const uint2* sorted, uint32_t n, uint32_t key)
{
    uint32_t lo = 0, len = n;
    while (len) {
        const uint32_t half = len >> 1;
        if (sorted[lo + half].x < key) { lo += half + 1; len -= half + 1; }
        else len = half;
    }
    return lo;
}

constexpr uint32_t kLongRun = 64;   // terms from which on a run is summed by the whole workgroup

// The rows launch.  ADD: a workgroup has 64 sorted positions and writes the rows whose runs begin there; otherwise it has
// 64 rows and writes them all.
template <class TG, class TT, int V, bool ADD>
__global__ void __launch_bounds__(kThreads) rows_kernel(GradArgs a)
{
    __shared__ float lds[kThreads][V];
    __shared__ uint32_t start[kRowsPerGroup + 1], key[kRowsPerGroup];
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log2, groups = kThreads >> a.lanes_log2;
    const uint32_t first = blockIdx.x * kRowsPerGroup;
    uint32_t rows;
    if (ADD) {
        // the runs that begin in [first, first + 64), side by side; the last one's end is looked for
        const uint32_t k = first + threadIdx.x;
        const int in = threadIdx.x < kRowsPerGroup && k < a.n;
        const uint32_t mine = in ? a.sorted[k].x : 0xFFFFFFFFu;
        const bool begins = in && mine < a.num_rows && (k == 0 || a.sorted[k - 1].x != mine);
        const uint64_t all = __ballot(begins);
        if (threadIdx.x < 64) {
            const int at = __popcll(all & ((1ull << threadIdx.x) - 1));
            if (begins) { start[at] = k; key[at] = mine; }
            if (threadIdx.x == 0) start[kRowsPerGroup] = __popcll(all);
        }
        __syncthreads();
        rows = start[kRowsPerGroup];
        __syncthreads();
        if (rows == 0) return;
        if (threadIdx.x == 0) start[rows] = lower_bound(a.sorted, a.n, key[rows - 1] + 1);
    } else {
        rows = min(static_cast<uint32_t>(kRowsPerGroup), a.num_rows - first);
        if (threadIdx.x <= rows) start[threadIdx.x] = lower_bound(a.sorted, a.n, first + threadIdx.x);
    }
    __syncthreads();
    for (uint32_t r = group; r < rows; r += groups) {
        const Run run = run_of(start[r], start[r + 1]);
        if (run.terms >= kLongRun) continue;
        const uint32_t row = ADD ? key[r] : first + r;
        for (int c = lane; c < a.chunks; c += lanes) {
            const int at = min(c * V, a.dim - V);
            float acc[V] = {};
            sum_terms<TG, V>(a, run, 0, 1, at, acc);
            write_chunk<TT, V, ADD>(a, row, c, at, acc);
        }
    }
    for (uint32_t r = 0; r < rows; ++r) {
        const Run run = run_of(start[r], start[r + 1]);
        if (run.terms < kLongRun) continue;
        const uint32_t row = ADD ? key[r] : first + r;
        for (int c0 = 0; c0 < a.chunks; c0 += lanes) {
            const int c = c0 + lane, at = min(min(c, a.chunks - 1) * V, a.dim - V);
            float acc[V] = {};
            sum_terms<TG, V>(a, run, group, groups, at, acc);
            join_groups<V>(lds, a.lanes_log2, acc);
            if (group == 0 && c < a.chunks) write_chunk<TT, V, ADD>(a, row, c, at, acc);
        }
    }
}

// Writes zeros: the gradient of no positions.
template <class TT>
__global__ void __launch_bounds__(kThreads) zero_rows_kernel(TT* table, int64_t stride, int64_t rows, int32_t dim)
{
    const int64_t total = rows * dim;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * kThreads)
        table[i / dim * stride + i % dim] = from_float<TT>(0.0f);
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct EmbedWs {
    uint2* entries[2];
    uint32_t* hist;
    float* partial;
    uint32_t tiles, tile_len;
    int32_t passes, bits;
    size_t total;
};

bool sizes_ok(int64_t num_rows, int32_t dim, int64_t n)
{
    return num_rows > 0 && num_rows < (1ll << 31) && dim >= 1 && dim <= NE_OP_MAX_DIM && n >= 0 && n <= NE_EMBED_MAX_IDS;
}

EmbedWs embed_layout(int64_t num_rows, int32_t dim, int64_t n, char* base)
{
    EmbedWs w{};
    int key_bits = 1;
    while ((num_rows >> key_bits) != 0) key_bits += 1;      // keys are 0 .. num_rows
    const int most = n <= kSmallSort ? kSmallBits : 10;
    w.passes = (key_bits + most - 1) / most;
    w.bits = (key_bits + w.passes - 1) / w.passes;
    int64_t len = (n + kMostTiles - 1) / kMostTiles;
    len = std::max<int64_t>((len + kSortRound - 1) / kSortRound * kSortRound, kSortRound);
    w.tile_len = static_cast<uint32_t>(len);
    w.tiles = static_cast<uint32_t>((n + len - 1) / len);
    Carver take{base};
    w.entries[0] = take.get<uint2>(static_cast<size_t>(n));
    w.entries[1] = take.get<uint2>(n > kSmallSort ? static_cast<size_t>(n) : 0);
    w.hist = take.get<uint32_t>(n > kSmallSort ? (static_cast<size_t>(w.passes) * w.tiles) << w.bits : 0);
    w.partial = take.get<float>(static_cast<size_t>((n + kChunk - 1) / kChunk) * dim);
    w.total = take.total();
    return w;
}

int lanes_log2_for(int chunks)
{
    int l = 0;
    while (l < 6 && (1 << l) < chunks) l += 1;
    return l;
}

template <class TG, class TT, int V>
hipError_t launch_grad(const GradArgs& a, bool add, hipStream_t st)
{
    if (a.n >= kChunk) {
        hipLaunchKernelGGL((chunk_sums_kernel<TG, V>), dim3((a.n + kSuper - 1) / kSuper), dim3(kThreads), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (add)
        hipLaunchKernelGGL((rows_kernel<TG, TT, V, true>), dim3((a.n + kRowsPerGroup - 1) / kRowsPerGroup), dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((rows_kernel<TG, TT, V, false>), dim3((a.num_rows + kRowsPerGroup - 1) / kRowsPerGroup), dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

template <class TG, class TT>
hipError_t launch_grad_dim(GradArgs a, bool add, hipStream_t st)
{
    constexpr int V = vec_of<TG, TT>();
    const bool wide = a.dim >= V;
    a.chunks = wide ? (a.dim + V - 1) / V : a.dim;
    a.lanes_log2 = lanes_log2_for(a.chunks);
    return wide ? launch_grad<TG, TT, V>(a, add, st) : launch_grad<TG, TT, 1>(a, add, st);
}

template <class TI, class TO>
hipError_t launch_lookup(LookupArgs a, hipStream_t st)
{
    constexpr int V = vec_of<TI, TO>();
    const bool wide = a.dim >= V;
    a.chunks = wide ? (a.dim + V - 1) / V : a.dim;
    a.lanes_log2 = lanes_log2_for(a.chunks);
    const int64_t rows = 4 * (kThreads >> a.lanes_log2);
    const dim3 grid(static_cast<unsigned>((a.n + rows - 1) / rows));
    if (wide) hipLaunchKernelGGL((lookup_kernel<TI, TO, V>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((lookup_kernel<TI, TO, 1>), grid, dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_sort(const EmbedWs& w, const int32_t* ids, int64_t n, int64_t num_rows, const uint2** sorted, hipStream_t st)
{
    SortArgs s{};
    s.ids = ids; s.hist = w.hist; s.n = static_cast<uint32_t>(n); s.num_rows = static_cast<uint32_t>(num_rows);
    s.tile_len = w.tile_len; s.tiles = w.tiles; s.passes = w.passes; s.bits = w.bits;
    if (n <= kSmallSort) {
        s.out = w.entries[0];
        *sorted = w.entries[0];
        hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(kSortThreads), 0, st, s);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(sort_count_kernel, dim3(w.tiles), dim3(kSortThreads), 0, st, s);
    hipError_t e = hipGetLastError();
    for (int p = 0; p < w.passes && e == hipSuccess; ++p) {
        s.pass = p; s.shift = p * w.bits;
        s.in = w.entries[(p + 1) & 1];
        s.out = w.entries[p & 1];
        *sorted = s.out;
        hipLaunchKernelGGL(sort_pass_kernel, dim3(w.tiles), dim3(kSortThreads), 0, st, s);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

extern "C" {

size_t ne_embed_workspace_bytes(int64_t num_rows, int32_t dim, int64_t n)
{
    if (!sizes_ok(num_rows, dim, n) || n == 0) return 0;
    return embed_layout(num_rows, dim, n, nullptr).total;
}

ne_status ne_embed_lookup(const void* table_dev, int32_t table_type, int64_t table_stride, int64_t num_rows, int32_t dim,
                          const int32_t* ids_dev, int64_t n, float scale, void* out_dev, int32_t out_type,
                          int64_t out_stride, void* hip_stream)
{
    if (!sizes_ok(num_rows, dim, n)) return fail(NE_ERR_ARG, "ne_embed_lookup: num_rows, dim or n out of range");
    if (!type_ok(table_type) || !type_ok(out_type)) return fail(NE_ERR_ARG, "ne_embed_lookup: a type is neither NE_F32 nor NE_BF16");
    if (table_stride < dim || out_stride < dim) return fail(NE_ERR_ARG, "ne_embed_lookup: a row stride is smaller than dim");
    if (!std::isfinite(scale)) return fail(NE_ERR_ARG, "ne_embed_lookup: scale is not finite");
    if (n == 0) return NE_OK;
    if (!table_dev || !aligned(table_dev, type_bytes(table_type))) return fail(NE_ERR_ARG, "ne_embed_lookup: table_dev is NULL or misaligned");
    if (!out_dev || !aligned(out_dev, type_bytes(out_type))) return fail(NE_ERR_ARG, "ne_embed_lookup: out_dev is NULL or misaligned");
    if (!ids_dev || !aligned(ids_dev, 4)) return fail(NE_ERR_ARG, "ne_embed_lookup: ids_dev is NULL or not 4-byte aligned");
    LookupArgs a{};
    a.table = table_dev; a.ids = ids_dev; a.out = out_dev; a.table_stride = table_stride; a.out_stride = out_stride;
    a.n = n; a.num_rows = static_cast<uint32_t>(num_rows); a.dim = dim; a.scale = scale;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = table_type == NE_F32 ? (out_type == NE_F32 ? launch_lookup<float, float>(a, st) : launch_lookup<float, bf16_t>(a, st))
                                              : (out_type == NE_F32 ? launch_lookup<bf16_t, float>(a, st) : launch_lookup<bf16_t, bf16_t>(a, st));
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("lookup launch: ") + hipGetErrorString(e));
    return NE_OK;
}

ne_status ne_embed_grad(const int32_t* ids_dev, int64_t n, const void* grad_dev, int32_t grad_type, int64_t grad_stride,
                        float scale, int64_t num_rows, int32_t dim, void* table_grad_dev, int32_t table_grad_type,
                        int64_t table_grad_stride, int32_t accumulate, void* workspace_dev, size_t workspace_bytes,
                        void* hip_stream)
{
    if (!sizes_ok(num_rows, dim, n)) return fail(NE_ERR_ARG, "ne_embed_grad: num_rows, dim or n out of range");
    if (!type_ok(grad_type) || !type_ok(table_grad_type)) return fail(NE_ERR_ARG, "ne_embed_grad: a type is neither NE_F32 nor NE_BF16");
    if (table_grad_stride < dim || (grad_stride < dim && grad_stride != 0))
        return fail(NE_ERR_ARG, "ne_embed_grad: a row stride is smaller than dim (and the gradient's not 0)");
    if (!std::isfinite(scale)) return fail(NE_ERR_ARG, "ne_embed_grad: scale is not finite");
    if (!table_grad_dev || !aligned(table_grad_dev, type_bytes(table_grad_type)))
        return fail(NE_ERR_ARG, "ne_embed_grad: table_grad_dev is NULL or misaligned");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (n == 0) {
        if (accumulate) return NE_OK;
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>((num_rows * dim + kThreads - 1) / kThreads, 4096)));
        if (table_grad_type == NE_F32)
            hipLaunchKernelGGL(zero_rows_kernel<float>, grid, dim3(kThreads), 0, st, static_cast<float*>(table_grad_dev), table_grad_stride, num_rows, dim);
        else
            hipLaunchKernelGGL(zero_rows_kernel<bf16_t>, grid, dim3(kThreads), 0, st, static_cast<bf16_t*>(table_grad_dev), table_grad_stride, num_rows, dim);
        NE_HIP_CHECK(hipGetLastError());
        return NE_OK;
    }
    if (!ids_dev || !aligned(ids_dev, 4)) return fail(NE_ERR_ARG, "ne_embed_grad: ids_dev is NULL or not 4-byte aligned");
    if (!grad_dev || !aligned(grad_dev, type_bytes(grad_type))) return fail(NE_ERR_ARG, "ne_embed_grad: grad_dev is NULL or misaligned");
    const EmbedWs w = embed_layout(num_rows, dim, n, static_cast<char*>(workspace_dev));
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < w.total)
        return fail(NE_ERR_ARG, "ne_embed_grad: workspace_dev is NULL, not 256-byte aligned, or smaller than ne_embed_workspace_bytes()");
    GradArgs a{};
    hipError_t e = launch_sort(w, ids_dev, n, num_rows, &a.sorted, st);
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("sort launch: ") + hipGetErrorString(e));
    a.grad = grad_dev; a.partial = w.partial; a.table = table_grad_dev; a.grad_stride = grad_stride; a.table_stride = table_grad_stride;
    a.n = static_cast<uint32_t>(n); a.num_rows = static_cast<uint32_t>(num_rows); a.dim = dim; a.scale = scale;
    const bool add = accumulate != 0;
    e = grad_type == NE_F32 ? (table_grad_type == NE_F32 ? launch_grad_dim<float, float>(a, add, st) : launch_grad_dim<float, bf16_t>(a, add, st))
                            : (table_grad_type == NE_F32 ? launch_grad_dim<bf16_t, float>(a, add, st) : launch_grad_dim<bf16_t, bf16_t>(a, add, st));
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("embedding gradient launch: ") + hipGetErrorString(e));
    return NE_OK;
}

}  // extern "C"
