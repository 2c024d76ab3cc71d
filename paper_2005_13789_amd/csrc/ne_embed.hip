// Rows of a table, scaled, and their gradient by sorted ids: ne_embed_lookup, ne_embed_grad.
//
// Lookup: out[i] = scale * table[ids[i]].  A gather: bound by memory, 4 bytes of id and a row read and written
// per position.  A lane group takes four rows at a time, so that a wavefront has four wide loads in flight
// (262 144 of a million rows of 256 bf16: 52 us, 5.1 TB/s, where a copy of as much makes 4.75; one row: 6.6 us, what a launch takes).
//
// Gradient: T[r] = sum over i with ids[i] = r of scale * grad[i], bound by memory: the gradient's rows read, the
// table's written.  Positions are sorted by id (stable radix sort, so the order of a row's terms is fixed by the ids
// alone), then a lane group adds the runs of some neighbouring rows in registers and rounds each sum once: no atomics
// on values.  While the ids are sorted, which leaves most of the machine idle, further workgroups of the same launches
// clear the table; the rows launch then writes the named rows only.  A run of thousands of positions (ids are
// skewed: the most frequent of a text or a graph takes percents of all positions) would leave one lane group with all
// of it, so whole chunks of 16 sorted positions that name one row are summed first, by a launch of their own over all
// positions, and 256 at a time where there are many positions; a long run is then at most 60 single terms and sums,
// and one sum per 256 positions, which a whole workgroup adds.
// Measured, 65 536 positions into 200 003 rows of 512 bf16 (272 MB, 57 us at a copy's rate): 100 us, of which the four
// sorting launches with the clearing 43 (clearing alone: 30), sums of 16 positions 9, rows 34.
// Up to 16 384 ids take one launch instead (few_ids_kernel): 4096 into 10 000 rows of 128 fp32 8.5 us, where the
// launches of the other way take 5 us each.
#include "ne_internal.h"
#include "ne_ops.h"

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16;          // sorted positions that are summed together where they name one row
constexpr int kSuper = 256;         // the same, one size up
constexpr int kSuperFrom = 131072;  // positions from which on that is done (a launch of 6 us); below, the longest runs have 8192 sums of 16
constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortFew = 65536;     // positions up to which a thread has two at a time, otherwise four (16 385 ids 25.9 us, 27.8
                                    // with four; 65 536 the same; 114 438: 48.9 and 46.8)
constexpr int kMostTiles = 128;     // workgroups of a sorting pass; each reads the counts of all
constexpr int kMostDigits = 1024;
constexpr int kRowsPerGroup = 64;   // table rows of a workgroup of the rows launch
constexpr int kFewIds = 16384;      // up to so many ids every workgroup looks through all of them
constexpr int kScan = 16;           // ids of a thread and round there
constexpr int kMostSlots = 256;     // rows of a workgroup there
constexpr int kFewWide = 6800;      // up to so many their slots are kept in LDS, too (4096: 7.2 us, 8.3 if ids are read again)
constexpr int kFewLds = 43000;      // bytes for what is found with which three workgroups have place on a CU, twice as many ids two
constexpr int kAddIds = 32;         // accumulate: positions of a workgroup there, at most ...
constexpr int kAddPlaces = 128;     // ... places of the hash table that finds their rows
constexpr int kAddFilter = 1024;    // ... and words of the filter before it: a bit for each hash of 15 bits

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
    uint32_t* hist;            // [tiles][digits]
    uint32_t n, num_rows, tile_len, tiles;
    int32_t pass, bits, shift;
    // the table's rows [clear_from, clear_to) are cleared by the launch's further workgroups, so many bytes of every clear_stride
    unsigned char* table;
    int64_t clear_stride, clear_bytes;
    uint32_t clear_from, clear_to;
};

// Share `part` of `parts` of the rows that a sorting launch clears.  (A sorting pass occupies an eighth of the machine for 5 to 8 us, most
// of which it waits.  65 536 positions, 200 003 rows of 512 bf16: 111 us with rows cleared by the rows launch, 100 so.)
__device__ __forceinline__ void clear_rows(const SortArgs& a, uint32_t part, uint32_t parts)
{
    const uint32_t rows = a.clear_to - a.clear_from;
    const uint32_t r0 = a.clear_from + static_cast<uint32_t>(static_cast<uint64_t>(rows) * part / parts);
    const uint32_t r1 = a.clear_from + static_cast<uint32_t>(static_cast<uint64_t>(rows) * (part + 1) / parts);
    const bool flat = a.clear_stride == a.clear_bytes;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (uint32_t r = r0; r < r1; r = flat ? r1 : r + 1) {
        unsigned char* to = a.table + r * a.clear_stride;
        const int64_t bytes = flat ? (r1 - r0) * a.clear_bytes : a.clear_bytes;
#pragma unroll 4
        for (int64_t i = threadIdx.x * 16; i + 16 <= bytes; i += kSortThreads * 16) __builtin_memcpy(to + i, &zero, 16);
        for (int64_t i = bytes / 16 * 16 + threadIdx.x * 2; i < bytes; i += kSortThreads * 2) __builtin_memcpy(to + i, &zero, 2);
    }
}

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
    if (blockIdx.x >= a.tiles) {
        clear_rows(a, blockIdx.x - a.tiles, gridDim.x - a.tiles);
        return;
    }
    const uint32_t digits = 1u << a.bits, mask = digits - 1;
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
    __syncthreads();
    const uint32_t lo = blockIdx.x * a.tile_len, hi = min(lo + a.tile_len, a.n);
#pragma unroll 4
    for (uint32_t i = lo + threadIdx.x; i < hi; i += kSortThreads)
        atomicAdd(&count[((a.pass == 0 ? key_of(a.ids[i], a.num_rows) : a.in[i].x) >> a.shift) & mask], 1u);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.hist[static_cast<size_t>(blockIdx.x) * digits + d] = count[d];
}

// Sum of all earlier threads' values (and of none of the later ones'), THREADS of them.
template <int THREADS>
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t* wave_sums, uint32_t* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(s, o, 64);
        if (lane >= o) s += u;
    }
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint32_t u = wave_sums[w];
        before += w < wave ? u : 0;
        all += u;
    }
    *total = all;
    return before + s - v;
}

// One pass: where a tile's entries of a digit begin follows from the counts of all tiles, which each workgroup adds up
// by itself (at most 128 x 1024 words, in L2: a launch less than with sums made in between).
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads) sort_pass_kernel(SortArgs a)
{
    __shared__ uint32_t base[kMostDigits];
    __shared__ uint32_t count[kSortWaves][kMostDigits];
    __shared__ uint32_t wave_sums[kSortWaves];
    if (blockIdx.x >= a.tiles) {
        clear_rows(a, blockIdx.x - a.tiles, gridDim.x - a.tiles);
        return;
    }
    const uint32_t digits = 1u << a.bits, mask = digits - 1;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // thread t has digits 2t and 2t + 1
    uint32_t total[2] = {0, 0}, mine[2] = {0, 0};
    if (2 * threadIdx.x < digits) {
        const uint2* hist = reinterpret_cast<const uint2*>(a.hist) + threadIdx.x;
        for (uint32_t t0 = 0; t0 < a.tiles; t0 += 16) {
            uint2 c[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) c[q] = t0 + q < a.tiles ? hist[static_cast<size_t>(t0 + q) * (digits / 2)] : make_uint2(0, 0);
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                total[0] += c[q].x;
                total[1] += c[q].y;
                if (t0 + q < blockIdx.x) {
                    mine[0] += c[q].x;
                    mine[1] += c[q].y;
                }
            }
        }
    }
    uint32_t all;
    const uint32_t before = block_prefix<kSortThreads>(total[0] + total[1], wave_sums, &all);
    if (2 * threadIdx.x < digits) {
        base[2 * threadIdx.x] = before + mine[0];
        base[2 * threadIdx.x + 1] = before + total[0] + mine[1];
    }
    const uint32_t lo = blockIdx.x * a.tile_len, hi = min(lo + a.tile_len, a.n);
    for (uint32_t r0 = lo; r0 < hi; r0 += kSortThreads * ITEMS) {
        uint2 e[ITEMS];
        uint32_t digit[ITEMS], rank[ITEMS];
        bool valid[ITEMS];
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            const uint32_t i = r0 + wave * (64 * ITEMS) + j * 64 + lane;
            valid[j] = i < hi;
            e[j] = make_uint2(0, 0);
            if (valid[j]) e[j] = a.pass == 0 ? make_uint2(key_of(a.ids[i], a.num_rows), i) : a.in[i];
            digit[j] = (e[j].x >> a.shift) & mask;
        }
        for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) count[w][d] = 0;
        __syncthreads();
        wave_ranks<ITEMS>(digit, valid, a.bits, count[wave], rank);
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
        for (int j = 0; j < ITEMS; ++j)
            if (valid[j]) a.out[count[wave][digit[j]] + rank[j]] = e[j];
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------
// sums of runs
// ---------------------------------------------------------------------------------------------
struct GradArgs {
    const uint2* sorted;
    const void* grad;
    float* partial;            // [n / kChunk][dim]  sums of chunks that name one row
    float* super;              // the same array's other half: sums of 256 positions, in the place of their first chunk
    void* table;
    int64_t grad_stride, table_stride;
    uint32_t n, num_rows;
    int32_t dim, chunks, lanes_log2;
    float scale;
    int32_t clear_all;         // rows are cleared before the named ones are written
};

// Terms of a run [s, e) of sorted positions: single positions up to a multiple of 16, sums of 16 up to a multiple of
// 256, sums of 256, sums of 16, single positions.
struct Run {
    uint32_t s, c0, u0, u1, c1, e;      // where each of the five parts ends or begins
    uint32_t terms;
};

__device__ __forceinline__ Run run_of(uint32_t s, uint32_t e, bool supers)
{
    Run r;
    r.s = s; r.e = e;
    r.c0 = min((s + kChunk - 1) / kChunk * kChunk, e);
    r.c1 = max(e / kChunk * kChunk, r.c0);
    r.u0 = supers ? min((r.c0 + kSuper - 1) / kSuper * kSuper, r.c1) : r.c1;
    r.u1 = max(r.c1 / kSuper * kSuper, r.u0);
    r.terms = (r.c0 - r.s) + (r.u0 - r.c0) / kChunk + (r.u1 - r.u0) / kSuper + (r.c1 - r.u1) / kChunk + (r.e - r.c1);
    return r;
}

// Term t of the run.
template <class TG, int V, class Position>
__device__ __forceinline__ void load_term(const GradArgs& a, const Run& r, uint32_t t, int at, float (&x)[V], Position position)
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
        load_vec<TG, V>(static_cast<const TG*>(a.grad) + static_cast<int64_t>(position(single)) * a.grad_stride + at, x);
    else
        load_vec<float, V>((r.u1 > r.u0 && chunk * kChunk >= r.u0 && chunk * kChunk < r.u1 ? a.super : a.partial) + static_cast<int64_t>(chunk) * a.dim + at, x);
}

// Every `step`-th of `terms` terms from t on, added up, U in flight; term(t, x) gives one.
template <int U, int V, class Term>
__device__ __forceinline__ void sum_terms(uint32_t t, uint32_t terms, uint32_t step, float (&acc)[V], Term term)
{
    for (; t + (U - 1) * step < terms; t += U * step) {
        float x[U][V];
#pragma unroll
        for (int q = 0; q < U; ++q) term(t + q * step, x[q]);
#pragma unroll
        for (int q = 0; q < U; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += x[q][e];
    }
    if (t < terms) {        // the last of them together, too
        float x[U - 1][V];
#pragma unroll
        for (int q = 0; q < U - 1; ++q) {
#pragma unroll
            for (int e = 0; e < V; ++e) x[q][e] = 0.0f;
            if (t + q * step < terms) term(t + q * step, x[q]);
        }
#pragma unroll
        for (int q = 0; q < U - 1; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += x[q][e];
    }
}

// What a row holds where a chunk of it will be added to.
template <class TT, int V>
__device__ __forceinline__ void load_old(const GradArgs& a, uint32_t row, int at, float (&x)[V])
{
    load_vec<TT, V>(static_cast<const TT*>(a.table) + static_cast<int64_t>(row) * a.table_stride + at, x);
}

// Writes scale * acc to chunk c of a row, ADD: added to what was there.  (The last chunk of a dim that V does not divide
// overlaps the one before: an addition must not be made twice.)
template <class TT, int V, bool ADD>
__device__ __forceinline__ void write_chunk(const GradArgs& a, uint32_t row, int c, int at, const float (&acc)[V], const float (&old)[V])
{
    TT* to = static_cast<TT*>(a.table) + static_cast<int64_t>(row) * a.table_stride + at;
    float x[V];
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = ADD ? fmaf(a.scale, acc[e], old[e]) : a.scale * acc[e];
    if (ADD && at != c * V) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (at + e >= c * V) to[e] = from_float<TT>(x[e]);
    } else {
        store_vec<TT, V>(to, x);
    }
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

// The rows [0, rows) of a workgroup, whose positions lie side by side: row r has those from start[r] to start[r + 1].  A lane
// group has some neighbouring rows and goes through their positions eight at a time, whichever rows they are of (most rows have
// none or one, and a fetch takes a microsecond: rows one after the other, four terms of each in flight, took 97 us where this
// takes 66, 65 536 positions, 200 003 rows of 512 bf16).  Rows of kLongRun positions or more are summed by the
// whole workgroup afterwards, from the terms of their run.
//   none(r): leave row r alone;  single(k, at, x): position k's values;  term(r, t, at, x): term t of a long row, which has terms(r).
constexpr uint32_t kLongRun = 32;

struct RowLists {
    uint16_t live[kMostSlots], hot[kMostSlots];     // rows of fewer than kLongRun positions (but some), and of more
    uint32_t wave_sums[kThreads / 64];
};

template <class TT, int V, bool ADD, class None, class Single, class Terms, class Term, class Row>
__device__ __forceinline__ void sum_rows(const GradArgs& a, uint32_t rows, const uint32_t* start, float (*lds)[V], RowLists& lists, None none, Single single,
                                         Terms terms, Term term, Row row_of)
{
    constexpr int U = 8, OLD = ADD ? 4 : 1;
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log2, groups = kThreads >> a.lanes_log2;
    const uint32_t mine = threadIdx.x < rows && !none(threadIdx.x) ? start[threadIdx.x + 1] - start[threadIdx.x] : 0;
    const uint32_t is_live = mine > 0 && mine < kLongRun, is_hot = mine >= kLongRun;
    uint32_t total;
    const uint32_t at_list = block_prefix<kThreads>(is_live | is_hot << 16, lists.wave_sums, &total);
    if (is_live) lists.live[at_list & 0xFFFF] = static_cast<uint16_t>(threadIdx.x);
    if (is_hot) lists.hot[at_list >> 16] = static_cast<uint16_t>(threadIdx.x);
    const uint32_t lives = total & 0xFFFF, hots = total >> 16;
    if (!ADD) {
        float zero[V];
#pragma unroll
        for (int e = 0; e < V; ++e) zero[e] = 0.0f;
        if (a.clear_all) {      // rows side by side, few of them named: all are cleared as one range (named ones are written after the barrier)
            TT* to = static_cast<TT*>(a.table) + static_cast<int64_t>(row_of(0)) * a.dim;
            const uint32_t count = rows * static_cast<uint32_t>(a.dim);
#pragma unroll 4
            for (uint32_t i = threadIdx.x * V; i + V <= count; i += kThreads * V) store_vec<TT, V>(to + i, zero);
            for (uint32_t i = count / V * V + threadIdx.x; i < count; i += kThreads) to[i] = from_float<TT>(0.0f);
        }
#pragma unroll 4
        for (uint32_t r = a.clear_all ? rows : group; r < rows; r += groups)
            if (start[r] == start[r + 1])
                for (int c = lane; c < a.chunks; c += lanes)
                    store_vec<TT, V>(static_cast<TT*>(a.table) + static_cast<int64_t>(row_of(r)) * a.table_stride + min(c * V, a.dim - V), zero);
    }
    __syncthreads();
    const uint32_t share = (lives + groups - 1) / groups, begin = min(group * share, lives), end = min(begin + share, lives);
    for (int c = lane; c < a.chunks; c += lanes) {
        const int at = min(c * V, a.dim - V);
        uint32_t i = begin;
        while (i < end) {
            // rows whose positions follow one another (no long row's are between them)
            uint32_t last = i + 1, stop = start[lists.live[i] + 1];
            while (last < end && (!ADD || last < i + OLD) && start[lists.live[last]] == stop) stop = start[lists.live[last++] + 1];
            uint32_t r = lists.live[i], k = start[r], next = start[r + 1];
            float acc[V] = {}, old[OLD][V] = {};        // (old: of the rows still to be written, the next one first)
            if (ADD)
#pragma unroll
                for (int q = 0; q < OLD; ++q)
                    if (i + q < last) load_old<TT, V>(a, row_of(lists.live[i + q]), at, old[q]);
            auto finish_row = [&]() {
                write_chunk<TT, V, ADD>(a, row_of(r), c, at, acc, old[0]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    acc[e] = 0.0f;
#pragma unroll
                    for (int q = 0; q + 1 < OLD; ++q) old[q][e] = old[q + 1][e];
                }
                if (++i < last) {
                    r = lists.live[i];
                    next = start[r + 1];
                }
            };
            for (; k < stop; k += U) {
                float x[U][V];
#pragma unroll
                for (int q = 0; q < U; ++q)
                    if (k + q < stop) single(k + q, at, x[q]);
#pragma unroll
                for (int q = 0; q < U; ++q)
                    if (k + q < stop) {
                        if (k + q == next) finish_row();
#pragma unroll
                        for (int e = 0; e < V; ++e) acc[e] += x[q][e];
                    }
            }
            finish_row();
        }
    }
    for (uint32_t h = 0; h < hots; ++h) {
        const uint32_t r = lists.hot[h];
        for (int c0 = 0; c0 < a.chunks; c0 += lanes) {
            const int c = c0 + lane, at = min(min(c, a.chunks - 1) * V, a.dim - V);
            float acc[V] = {};
            sum_terms<U, V>(group, terms(r), groups, acc, [&](uint32_t t, float (&x)[V]) { term(r, t, at, x); });
            join_groups<V>(lds, a.lanes_log2, acc);
            if (group == 0 && c < a.chunks) {
                float old[V] = {};
                if (ADD) load_old<TT, V>(a, row_of(r), at, old);
                write_chunk<TT, V, ADD>(a, row_of(r), c, at, acc, old);
            }
        }
    }
}

// Sums of 16 sorted positions that name one row; a lane group has 16 positions, all of whose rows are in flight at once.
template <class TG, int V>
__global__ void __launch_bounds__(kThreads) chunk_sums_kernel(GradArgs a)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const uint32_t chunk = blockIdx.x * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    if (chunk >= a.n / kChunk) return;
    const uint32_t k = chunk * kChunk, row = a.sorted[k].x;
    if (row >= a.num_rows || a.sorted[k + kChunk - 1].x != row) return;
    for (int c = lane; c < a.chunks; c += lanes) {
        const int at = min(c * V, a.dim - V);
        float acc[V] = {};
        sum_terms<kChunk, V>(0, kChunk, 1, acc, [&](uint32_t t, float (&x)[V]) {
            load_vec<TG, V>(static_cast<const TG*>(a.grad) + static_cast<int64_t>(a.sorted[k + t].y) * a.grad_stride + at, x);
        });
        store_vec<float, V>(a.partial + static_cast<int64_t>(chunk) * a.dim + at, acc);
    }
}

// The same for 16 such sums, of 256 positions that name one row.
template <int V>
__global__ void __launch_bounds__(kThreads) super_sums_kernel(GradArgs a)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const uint32_t group = blockIdx.x * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    if (group >= a.n / kSuper) return;
    const uint32_t k = group * kSuper, row = a.sorted[k].x;
    if (row >= a.num_rows || a.sorted[k + kSuper - 1].x != row) return;
    for (int c = lane; c < a.chunks; c += lanes) {
        const int at = min(c * V, a.dim - V);
        float acc[V] = {};
        sum_terms<kSuper / kChunk, V>(0, kSuper / kChunk, 1, acc, [&](uint32_t t, float (&x)[V]) {
            load_vec<float, V>(a.partial + static_cast<int64_t>(k / kChunk + t) * a.dim + at, x);
        });
        store_vec<float, V>(a.super + static_cast<int64_t>(k / kChunk) * a.dim + at, acc);
    }
}

// First sorted position whose key is at least `key`, by a whole wavefront: 64 probes at a time, three rounds of them for 2^18
// positions (each waits for memory, as the positions come from the launch before).
__device__ __forceinline__ uint32_t wave_lower_bound(const uint2* sorted, uint32_t n, uint32_t key)
{
    uint32_t lo = 0, len = n;
    while (len) {
        const uint32_t step = (len + 63) / 64, at = lo + (threadIdx.x & 63) * step + step - 1;
        const uint32_t below = __popcll(__ballot(at < lo + len && sorted[at].x < key));
        const uint32_t next = lo + below * step;
        len = min(step - 1, lo + len - next);
        lo = next;
    }
    return lo;
}

// The rows launch: a workgroup has 64 sorted positions and writes the rows whose runs begin there (the others were cleared while the
// positions were sorted; ADD: they keep what they hold).
template <class TG, class TT, int V, bool ADD>
__global__ void __launch_bounds__(kThreads) rows_kernel(GradArgs a)
{
    __shared__ float lds[kThreads][V];
    __shared__ RowLists lists;
    __shared__ uint32_t start[kRowsPerGroup + 1], key[kRowsPerGroup], place[2 * kRowsPerGroup], found;
    const uint32_t first = blockIdx.x * kRowsPerGroup;
    // the runs that begin here, side by side; the last one's end is looked for
    if (threadIdx.x < 2 * kRowsPerGroup) {
        const uint32_t k = first + threadIdx.x;
        const uint2 e = k < a.n ? a.sorted[k] : make_uint2(0xFFFFFFFFu, 0);
        place[threadIdx.x] = e.y;
        if (threadIdx.x < kRowsPerGroup) {
            const bool begins = e.x < a.num_rows && (k == 0 || a.sorted[k - 1].x != e.x);
            const uint64_t all = __ballot(begins);
            const int at = __popcll(all & ((1ull << threadIdx.x) - 1));
            if (begins) { start[at] = k; key[at] = e.x; }
            if (threadIdx.x == 0) found = __popcll(all);
        }
    }
    __syncthreads();
    const uint32_t rows = found;
    if (rows == 0) return;
    if (threadIdx.x < 64) {
        const uint32_t end = wave_lower_bound(a.sorted, a.n, key[rows - 1] + 1);
        if (threadIdx.x == 0) start[rows] = end;
    }
    __syncthreads();
    const TG* grad = static_cast<const TG*>(a.grad);
    auto position = [&](uint32_t k) { return k - first < 2 * kRowsPerGroup ? place[k - first] : a.sorted[k].y; };
    sum_rows<TT, V, ADD>(
        a, rows, start, lds, lists, [](uint32_t) { return false; },
        [&](uint32_t k, int at, float (&x)[V]) { load_vec<TG, V>(grad + static_cast<int64_t>(position(k)) * a.grad_stride + at, x); },
        [&](uint32_t r) { return run_of(start[r], start[r + 1], a.super != nullptr).terms; },
        [&](uint32_t r, uint32_t t, int at, float (&x)[V]) { load_term<TG, V>(a, run_of(start[r], start[r + 1], a.super != nullptr), t, at, x, position); },
        [&](uint32_t r) { return key[r]; });
}

// ---------------------------------------------------------------------------------------------
// few ids: one launch, no sorting of all of them
// ---------------------------------------------------------------------------------------------
// Every workgroup looks through all ids (they are in L2 after the first) for those that name one of its rows: its range of
// rows, or with ADD the rows that 32 positions are the first to name.  What it finds lies in LDS in the order of the positions and is
// sorted there by row (stably), so the order of a row's terms is that of the sorting path.
// Bound by the chain of a launch, the ids, the found rows' gradients and the store, each of which waits for memory once (4096 ids, 10 000
// rows of 128 fp32: 8.5 us), and with more ids by the looking (10 007 ids, ADD: 14 us; one bit for each hash is looked up first, since most
// ids of most workgroups are then done with).  LDS for as many found positions as there are ids bounds the workgroups of a CU, so it is
// kept small (16 384 ids, ADD: 17 us, 29 with 6 bytes for each; without ADD into 10 000 rows 13 and 20).
struct FewArgs {
    GradArgs g;
    const int32_t* ids;
    uint32_t slots;            // rows of a workgroup, ADD: positions; a power of two
    int32_t slot_bits;
    int32_t wide;              // what is found is kept with its slot; otherwise (less LDS) its id is read and looked up again
};

// Words of what is found, at most all n positions.
__host__ __device__ __forceinline__ uint32_t few_found(uint32_t n, bool wide) { return wide ? n : (n + 1) / 2; }

template <class TG, class TT, int V, bool ADD>
__global__ void __launch_bounds__(kThreads) few_ids_kernel(FewArgs f)
{
    extern __shared__ uint32_t found[];        // [n]  slot << 16 | position, or positions of 16 bits; behind them [n] positions by slot (16 bits)
    __shared__ union {
        uint32_t count[kThreads / 64][kMostSlots];      // while sorting
        float sums[kThreads][V];                        // afterwards
    } lds;
    __shared__ RowLists lists;
    __shared__ uint32_t wave_sums[kThreads / 64];
    __shared__ uint32_t start[kMostSlots + 1];
    // ADD: the ids of the places and the slots that they have, the slots' ids, and whether an earlier workgroup has them
    __shared__ uint32_t place_id[ADD ? kAddPlaces : 1], owner[ADD ? kAddIds : 1], taken[ADD ? kAddIds : 1], slots_used;
    __shared__ uint8_t place_slot[ADD ? kAddPlaces : 1];
    __shared__ uint32_t filter[ADD ? kAddFilter : 1];
    const GradArgs& a = f.g;
    uint16_t* found16 = reinterpret_cast<uint16_t*>(found);
    uint16_t* sorted = found16 + few_found(a.n, f.wide) * 2;
    const uint32_t first = blockIdx.x * f.slots;
    const int wave = threadIdx.x >> 6, lane64 = threadIdx.x & 63;
    if (ADD) {
        for (uint32_t i = threadIdx.x; i < kAddPlaces; i += kThreads) place_id[i] = 0xFFFFFFFFu;
        for (uint32_t i = threadIdx.x; i < kAddFilter; i += kThreads) filter[i] = 0;
        if (threadIdx.x < kAddIds) taken[threadIdx.x] = 0;
        if (threadIdx.x == 0) slots_used = 0;
        __syncthreads();
        if (threadIdx.x < f.slots && first + threadIdx.x < a.n) {
            const uint32_t id = static_cast<uint32_t>(f.ids[first + threadIdx.x]);
            if (id < a.num_rows)
                for (uint32_t at = hash_position(id, kAddPlaces - 1);; at = (at + 1) & (kAddPlaces - 1)) {
                    const uint32_t was = atomicCAS(&place_id[at], 0xFFFFFFFFu, id);
                    if (was == 0xFFFFFFFFu) {       // (which slot an id gets changes nothing)
                        const uint32_t slot = atomicAdd(&slots_used, 1u);
                        place_slot[at] = static_cast<uint8_t>(slot);
                        owner[slot] = id;
                        const uint32_t bit = hash_position(id, 32 * kAddFilter - 1);
                        atomicOr(&filter[bit >> 5], 1u << (bit & 31));
                    }
                    if (was == 0xFFFFFFFFu || was == id) break;
                }
        }
        __syncthreads();
    }
    uint32_t have = 0;
    uint32_t ahead[kScan];      // the next round's ids travel during a round
    auto fetch_ids = [&](uint32_t at) {
        if (at + kScan <= a.n) {
#pragma unroll
            for (int q = 0; q < kScan; q += 4) __builtin_memcpy(&ahead[q], f.ids + at + q, 16);
        } else {
#pragma unroll
            for (int q = 0; q < kScan; ++q) ahead[q] = at + q < a.n ? static_cast<uint32_t>(f.ids[at + q]) : 0xFFFFFFFFu;
        }
    };
    fetch_ids(threadIdx.x * kScan);
    for (uint32_t r0 = 0; r0 < a.n; r0 += kThreads * kScan) {
        uint32_t id[kScan];
        const uint32_t at = r0 + threadIdx.x * kScan;
#pragma unroll
        for (int q = 0; q < kScan; ++q) id[q] = ahead[q];
        if (r0 + kThreads * kScan < a.n) fetch_ids(at + kThreads * kScan);
        uint32_t wanted = 0, word[kScan];
        if (ADD)
#pragma unroll
            for (int q = 0; q < kScan; ++q) word[q] = filter[hash_position(id[q], 32 * kAddFilter - 1) >> 5];
#pragma unroll
        for (int q = 0; q < kScan; ++q) {
            const bool in = id[q] < a.num_rows && (ADD ? word[q] >> (hash_position(id[q], 32 * kAddFilter - 1) & 31) & 1 : id[q] - first < f.slots);
            wanted |= static_cast<uint32_t>(in) << q;
        }
        uint32_t total;
        uint32_t to = have + block_prefix<kThreads>(__popc(wanted), wave_sums, &total);
#pragma unroll
        for (int q = 0; q < kScan; ++q)
            if (wanted >> q & 1) {
                if (f.wide) found[to++] = (ADD ? 0 : (id[q] - first) << 16) | (at + q);
                else found16[to++] = static_cast<uint16_t>(at + q);
            }
        have += total;
        __syncthreads();
    }
    // ADD: what passed the filter is looked up; slot kAddIds takes what has no row here, or stands before all of this workgroup's
    auto look_up = [&](uint32_t k) -> uint32_t {
        const uint32_t id = static_cast<uint32_t>(f.ids[k]);
        if (!ADD) return id - first;
        for (uint32_t at = hash_position(id, kAddPlaces - 1);; at = (at + 1) & (kAddPlaces - 1)) {
            const uint32_t o = place_id[at];
            if (o == 0xFFFFFFFFu) return kAddIds;
            if (o != id) continue;
            const uint32_t slot = place_slot[at];
            if (k >= first) return slot;
            taken[slot] = 1;
            return kAddIds;
        }
    };
    if (ADD && f.wide) {
        for (uint32_t i = threadIdx.x; i < have; i += kThreads) found[i] |= look_up(found[i]) << 16;
        __syncthreads();
    }
    auto entry = [&](uint32_t i) -> uint32_t { return f.wide ? found[i] : look_up(found16[i]) << 16 | found16[i]; };
    // stable sort by slot: counts of every wavefront's share, then places
    const uint32_t share = (have + kThreads - 1) / kThreads * 64;      // entries of a wavefront, side by side
    for (uint32_t i = threadIdx.x; i < kMostSlots; i += kThreads)
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) lds.count[w][i] = 0;
    __syncthreads();
    uint32_t first_entry = 0;
    for (uint32_t i0 = wave * share; i0 < min((wave + 1) * share, have); i0 += 64) {
        if (i0 + lane64 >= min((wave + 1) * share, have)) continue;
        const uint32_t e = entry(i0 + lane64);
        if (i0 == wave * share) first_entry = e;
        atomicAdd(&lds.count[wave][e >> 16], 1u);
    }
    __syncthreads();
    {
        const bool has_slot = threadIdx.x < kMostSlots;
        uint32_t sum = 0, total;
        if (has_slot)
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) sum += lds.count[w][threadIdx.x];
        uint32_t at = block_prefix<kThreads>(sum, wave_sums, &total);
        if (threadIdx.x == 0) start[kMostSlots] = total;
        if (has_slot) {
            start[threadIdx.x] = at;
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) {
                const uint32_t c = lds.count[w][threadIdx.x];
                lds.count[w][threadIdx.x] = at;
                at += c;
            }
        }
    }
    __syncthreads();
    for (uint32_t i0 = wave * share; i0 < min((wave + 1) * share, have); i0 += 64) {
        const bool valid[1] = {i0 + lane64 < min((wave + 1) * share, have)};
        const uint32_t e = !valid[0] ? 0 : i0 == wave * share ? first_entry : entry(i0 + lane64);
        const uint32_t digit[1] = {e >> 16};
        uint32_t rank[1];
        wave_ranks<1>(digit, valid, f.slot_bits, lds.count[wave], rank);
        if (valid[0]) sorted[rank[0]] = static_cast<uint16_t>(e);
    }
    __syncthreads();
    auto single = [&](uint32_t k, int at, float (&x)[V]) {
        load_vec<TG, V>(static_cast<const TG*>(a.grad) + static_cast<int64_t>(sorted[k]) * a.grad_stride + at, x);
    };
    sum_rows<TT, V, ADD>(
        a, ADD ? slots_used : min(f.slots, a.num_rows - first), start, lds.sums, lists, [&](uint32_t r) { return ADD && taken[r]; }, single,
        [&](uint32_t r) { return start[r + 1] - start[r]; },
        [&](uint32_t r, uint32_t t, int at, float (&x)[V]) { single(start[r] + t, at, x); }, [&](uint32_t r) { return ADD ? owner[r] : first + r; });
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
    float *partial, *super;
    uint32_t tiles, tile_len;
    int32_t passes, bits;
    size_t total;
};

// Whether every workgroup looks through all ids: few of them, and no fewer rows than share them among enough workgroups.  (16 384 ids and, sorted,
// 16 385, skewed as words are, us: written into 200 003 rows of 128 fp32 30 and 45, of 1024 178 and 249, into 10 000 rows of 128 20 and 29, of 1024 77
// and 83; added to 200 003 rows of 128 21 and 32, of 1024 62 and 91.  The rule knows neither widths nor repeated ids: added to 10 000 rows of 128
// 33 and 29, of 1024 108 and 87, and 16 384 ids that all name one row, which one workgroup sums, 191 and 45 at 128 columns, 1060 and 213 at 1024.)
bool few_ids(int64_t num_rows, int64_t n) { return n <= kFewIds && n <= 16 * num_rows; }

bool sizes_ok(int64_t num_rows, int32_t dim, int64_t n)
{
    return num_rows > 0 && num_rows < (1ll << 31) && dim >= 1 && dim <= NE_OP_MAX_DIM && n >= 0 && n <= NE_EMBED_MAX_IDS;
}

EmbedWs embed_layout(int64_t num_rows, int32_t dim, int64_t n, char* base)
{
    EmbedWs w{};
    int key_bits = 1;
    while ((num_rows >> key_bits) != 0) key_bits += 1;      // keys are 0 .. num_rows
    w.passes = (key_bits + 9) / 10;
    w.bits = (key_bits + w.passes - 1) / w.passes;
    int64_t len = (n + kMostTiles - 1) / kMostTiles;
    const int64_t round = kSortThreads * (n <= kSortFew ? 2 : 4);
    len = std::max<int64_t>((len + round - 1) / round * round, round);
    w.tile_len = static_cast<uint32_t>(len);
    w.tiles = static_cast<uint32_t>((n + len - 1) / len);
    Carver take{base};
    if (!few_ids(num_rows, n)) {
        w.entries[0] = take.get<uint2>(static_cast<size_t>(n));
        w.entries[1] = take.get<uint2>(static_cast<size_t>(n));
        // (for as many tiles as shorter ones would be: no less for larger n)
        w.hist = take.get<uint32_t>(static_cast<size_t>(std::min<int64_t>(kMostTiles, (n + 2 * kSortThreads - 1) / (2 * kSortThreads))) << w.bits);
        w.partial = take.get<float>(static_cast<size_t>(n / kChunk) * dim);
        if (n > kSuperFrom) w.super = take.get<float>(static_cast<size_t>(n / kChunk) * dim);
    }
    w.total = std::max<size_t>(take.total(), 256);
    return w;
}

int lanes_log2_for(int chunks)
{
    int l = 0;
    while (l < 6 && (1 << l) < chunks) l += 1;
    return l;
}

template <class TG, class TT, int V>
hipError_t launch_few(const GradArgs& a, const int32_t* ids, bool add, hipStream_t st)
{
    FewArgs f{a, ids, 0, 0, a.n <= kFewWide};
    const size_t lds = few_found(a.n, f.wide) * size_t{4} + static_cast<size_t>(a.n) * 2;
    if (add) {      // 16 positions for each workgroup where all then run at once (8192: 11.0 us, 12.1 with 32)
        const uint32_t at_once = 256 * (lds <= kFewLds ? 3 : 2);
        f.slots = (a.n + 15) / 16 <= at_once ? 16 : kAddIds;
    } else {        // 512 workgroups, and up to 4096 where looking through all ids costs each of them little
        const uint32_t most = std::min(std::max(4u << 20, 512 * a.n) / a.n, 4096u);
        f.slots = 32;
        while (f.slots < kMostSlots && a.num_rows / f.slots > most) f.slots *= 2;
    }
    while ((1u << f.slot_bits) < (add ? kAddIds + 1 : f.slots)) f.slot_bits += 1;
    const uint32_t blocks = ((add ? a.n : a.num_rows) + f.slots - 1) / f.slots;
    if (add) hipLaunchKernelGGL((few_ids_kernel<TG, TT, V, true>), dim3(blocks), dim3(kThreads), lds, st, f);
    else hipLaunchKernelGGL((few_ids_kernel<TG, TT, V, false>), dim3(blocks), dim3(kThreads), lds, st, f);
    return hipGetLastError();
}

template <class TG, class TT, int V>
hipError_t launch_grad(const GradArgs& a, const int32_t* ids, bool add, hipStream_t st)
{
    if (few_ids(a.num_rows, a.n)) return launch_few<TG, TT, V>(a, ids, add, st);
    const uint32_t groups = kThreads >> a.lanes_log2;
    hipLaunchKernelGGL((chunk_sums_kernel<TG, V>), dim3((a.n / kChunk + groups - 1) / groups), dim3(kThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.super) {
        hipLaunchKernelGGL((super_sums_kernel<V>), dim3((a.n / kSuper + groups - 1) / groups), dim3(kThreads), 0, st, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid((a.n + kRowsPerGroup - 1) / kRowsPerGroup);
    if (add) hipLaunchKernelGGL((rows_kernel<TG, TT, V, true>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((rows_kernel<TG, TT, V, false>), grid, dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

template <class TG, class TT>
hipError_t launch_grad_dim(GradArgs a, const int32_t* ids, bool add, hipStream_t st)
{
    constexpr int V = vec_of<TG, TT>();
    const bool wide = a.dim >= V;
    a.chunks = wide ? (a.dim + V - 1) / V : a.dim;
    a.lanes_log2 = lanes_log2_for(a.chunks);
    return wide ? launch_grad<TG, TT, V>(a, ids, add, st) : launch_grad<TG, TT, 1>(a, ids, add, st);
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

// table: NULL, or the rows that the sorting launches clear meanwhile, an equal share each.
hipError_t launch_sort(const EmbedWs& w, const int32_t* ids, int64_t n, int64_t num_rows, void* table, int64_t row_bytes, int64_t row_stride,
                       const uint2** sorted, hipStream_t st)
{
    SortArgs s{};
    s.ids = ids; s.hist = w.hist; s.n = static_cast<uint32_t>(n); s.num_rows = static_cast<uint32_t>(num_rows);
    s.tile_len = w.tile_len; s.tiles = w.tiles; s.bits = w.bits;
    s.table = static_cast<unsigned char*>(table); s.clear_bytes = row_bytes; s.clear_stride = row_stride;
    const int launches = 2 * w.passes;
    int done = 0;
    auto share = [&]() -> uint32_t {        // the next share, and the workgroups for it: 64 KB or more each
        if (!table) return 0;
        s.clear_from = static_cast<uint32_t>(num_rows * done / launches);
        s.clear_to = static_cast<uint32_t>(num_rows * (done + 1) / launches);
        done += 1;
        return static_cast<uint32_t>(std::min<int64_t>(((s.clear_to - s.clear_from) * row_bytes + 65535) / 65536, 1024));
    };
    hipError_t e = hipSuccess;
    for (int p = 0; p < w.passes && e == hipSuccess; ++p) {
        s.pass = p; s.shift = p * w.bits;
        s.in = w.entries[(p + 1) & 1];
        s.out = w.entries[p & 1];
        *sorted = s.out;
        uint32_t more = share();
        hipLaunchKernelGGL(sort_count_kernel, dim3(w.tiles + more), dim3(kSortThreads), 0, st, s);
        e = hipGetLastError();
        if (e != hipSuccess) break;
        more = share();
        if (n <= kSortFew) hipLaunchKernelGGL(sort_pass_kernel<2>, dim3(w.tiles + more), dim3(kSortThreads), 0, st, s);
        else hipLaunchKernelGGL(sort_pass_kernel<4>, dim3(w.tiles + more), dim3(kSortThreads), 0, st, s);
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
    const bool few = few_ids(num_rows, n);
    const int64_t element = static_cast<int64_t>(type_bytes(table_grad_type));
    hipError_t e = few ? hipSuccess
                       : launch_sort(w, ids_dev, n, num_rows, accumulate ? nullptr : table_grad_dev, dim * element, table_grad_stride * element, &a.sorted, st);
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("sort launch: ") + hipGetErrorString(e));
    a.grad = grad_dev; a.partial = w.partial; a.super = w.super; a.table = table_grad_dev; a.grad_stride = grad_stride; a.table_stride = table_grad_stride;
    a.n = static_cast<uint32_t>(n); a.num_rows = static_cast<uint32_t>(num_rows); a.dim = dim; a.scale = scale;
    a.clear_all = few && table_grad_stride == dim && n * 4 <= num_rows;      // (a row written twice costs less than rows cleared one by one)
    const bool add = accumulate != 0;
    e = grad_type == NE_F32 ? (table_grad_type == NE_F32 ? launch_grad_dim<float, float>(a, ids_dev, add, st) : launch_grad_dim<float, bf16_t>(a, ids_dev, add, st))
                            : (table_grad_type == NE_F32 ? launch_grad_dim<bf16_t, float>(a, ids_dev, add, st) : launch_grad_dim<bf16_t, bf16_t>(a, ids_dev, add, st));
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("embedding gradient launch: ") + hipGetErrorString(e));
    return NE_OK;
}

}  // extern "C"
