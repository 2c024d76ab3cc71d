// Answers from a whole table: log probabilities of given ids, entropies, and the best ids of every row (ne_logprob).
//
//     S = H . W^T [n x V],   lse_i = log sum_v exp S_iv,   logp_i = S_i,id - lse_i
//     entropy_i = - sum_v p_iv log p_iv = log sum_v e^x_iv - sum_v p_iv x_iv,   x_iv = S_iv - max S_i  (nothing large is subtracted)
//     top: the k ids of largest S_iv in falling order, of equal scores the lowest id first
//
// Scores are never kept.  One pass over them leaves, beside the maximum and the two sums of every row's softmax, one record of 8 bytes for every
// chunk of table rows (64, or 16) and row of H: the chunk's best score with its place in the low bits, and
// its second best.  A score is off by at most `off_by` from what 64 bits would give.  So, with t the k-th largest of the chunks' best, the answers are among
// the chunks' best of at least t - 2 off_by and, where a chunk's second best reaches that, too (4 chunks in 100 rows at k = 16 of 200 003), its
// other rows.  A wavefront or more for every row of H finds these in the records, takes their scores again with sums in 64 bits, and orders them:
// what it answers does not depend on how the table was cut into tiles, and equal rows tie exactly.
#include "ne_tiles.h"

namespace {

// Chunks of table rows.  kWide: 64.  kNarrow: 16, what a lane has of 32 rows of a tile.  kStreamed: 16, a tile of few rows' kernel.
enum Chunks { kNone, kWide, kNarrow, kStreamed };
constexpr int chunk_log2(int chunks) { return chunks == kWide ? 6 : 4; }
constexpr int64_t kLateGroups = 512;
constexpr int64_t kUngrouped = 1024;                   // chunks that a wavefront looks through
constexpr int64_t kChunksOfFour = 4096;                 // chunks that four wavefronts look through
constexpr int64_t kTeamsOfMany = 512;                  // rows of H up to which several wavefronts look for the answers of each
constexpr float kNoScore = -1e30f;                     // below all scores: they are bounded by kMostScore
constexpr float kMostScore = 1e29f;
// Scores, in powers of two, from which on a softmax's maximum is taken from the sums as they are and subtracted before anything is multiplied: a
// maximum with a place in its low bits is 2^-17 of itself too small or too large, up to 1 here, and a product's rounding is no exponent's any more.
constexpr float kLargeScore = 0x1p17f;

// A row's softmax so far: maximum and, relative to it, the sums of e^x and x e^x (all in powers of two).
struct Softmax {
    float top, sum, moment, unused;
};

// How far a maximum is below a new one, as far as that counts: 2^-1000 is 0, and a sum times more would be infinite where scores are very large.
__device__ __forceinline__ float below(float top, float now) { return fmaxf(top - now, -1000.0f); }

__device__ __forceinline__ void join(Softmax& a, float top, float sum, float moment)
{
    const float now = fmaxf(a.top, top), da = below(a.top, now), db = below(top, now), ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
    a.moment = fmaf(a.sum, da, a.moment) * ea + fmaf(sum, db, moment) * eb;
    a.sum = a.sum * ea + sum * eb;
    a.top = now;
}

__device__ __forceinline__ void join_lanes(Softmax& a, int other)
{
    join(a, __shfl_xor(a.top, other, 64), __shfl_xor(a.sum, other, 64), __shfl_xor(a.moment, other, 64));
}

// The best and the second best of what a lane has seen.
struct Best {
    float first = kNoScore, second = kNoScore;
    // `place` in the low bits of the score, which moves it by 2^-17 of itself at most
    __device__ __forceinline__ void see(float score, uint32_t place, uint32_t mask)
    {
        const float x = __uint_as_float((__float_as_uint(score) & mask) | place);
        second = __builtin_amdgcn_fmed3f(first, second, x);
        first = __builtin_amdgcn_fmed3f(first, x, INFINITY);      // (the larger; a plain maximum would be preceded by another instruction)
    }
    __device__ __forceinline__ void join_lanes(int other)
    {
        const float f = __shfl_xor(first, other, 64), s = __shfl_xor(second, other, 64);
        second = fmaxf(fminf(first, f), fmaxf(second, s));
        first = fmaxf(first, f);
    }
    // As it is left behind: both scores times a power of two, which must not touch the place (of a score of 0 it is all there is).
    __device__ __forceinline__ float2 record(float factor, uint32_t mask) const
    {
        return make_float2(__uint_as_float((__float_as_uint(first * factor) & mask) | (__float_as_uint(first) & ~mask)), second * factor);
    }
};

// ---------------------------------------------------------------------------------------------
// norms
// ---------------------------------------------------------------------------------------------
// A bound of the largest norm of a row of W, squared (its pieces of eight elements take their maxima over rows apart, so that rows need no sums of
// their own), and the largest magnitudes that halves are scaled by.  Read as bits, values that are not finite are largest.
struct NormArgs {
    const void *w, *h;
    int64_t w_stride, h_stride, n, num_rows;
    const int32_t* ids;
    int32_t dim;
    uint32_t* norms;        // [workgroups]
    float* amax;            // NULL, or [2][kAmaxBlocks]  of W, of H's rows that count
};

__device__ __forceinline__ uint32_t block_max_bits(uint32_t v, uint32_t* lds)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o, 64)));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    for (uint32_t w = 0; w < blockDim.x / 64; ++w) v = max(v, lds[w]);
    return v;
}

// Bits of eight elements without their signs: 0 where all are.
template <class T>
__device__ __forceinline__ uint32_t magnitude_bits(const T (&x)[8])
{
    uint32_t words[2 * sizeof(T)], bits = 0;
    __builtin_memcpy(words, x, sizeof(words));
#pragma unroll
    for (uint32_t q = 0; q < 2 * sizeof(T); ++q) bits |= words[q];
    return bits & (sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu);
}

// A lane's share of the norms: pieces of a row from column e on, all rows' pieces of one column after the other.
struct NormShare {
    float total = 0.0f;
    uint32_t most = 0;
    int at = 0;
    template <class T>
    __device__ __forceinline__ void see(int e, const T (&x)[8])
    {
        if (e != at) {
            total += __uint_as_float(most);
            most = 0;
            at = e;
        }
        float squares = 0.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) squares = fmaf(static_cast<float>(x[q]), static_cast<float>(x[q]), squares);
        if (magnitude_bits(x) && squares < 0x1p-126f) squares = 0x1p-126f;      // (squares of small values may be 0)
        most = max(most, __float_as_uint(squares) & 0x7FFFFFFFu);
    }
    // of `width` columns, by all of a workgroup
    __device__ __forceinline__ void leave(int width, uint32_t* norm, uint32_t* lds)
    {
        total += __uint_as_float(most);
        int lanes = 1;
        while (lanes < 64 && 8 * lanes < width) lanes *= 2;
        for (int o = 1; o < lanes; o <<= 1) total += __shfl_xor(total, o, 64);
        const uint32_t all = block_max_bits(__float_as_uint(total) & 0x7FFFFFFFu, lds);
        if (threadIdx.x == 0) *norm = all;
    }
};

template <class T>
__device__ __forceinline__ void norms_of(const NormArgs& a, uint32_t block, uint32_t blocks, uint32_t* lds)
{
    NormShare share;
    float largest = 0.0f;
    for_eights(static_cast<const T*>(a.w), a.w_stride, a.num_rows, a.dim, a.dim, block, blocks, [&](int64_t, int e, const T (&x)[8]) {
        share.see(e, x);
        if (sizeof(T) == 4)
#pragma unroll
            for (int q = 0; q < 8; ++q) largest = fmaxf(largest, finite_abs(static_cast<float>(x[q])));
    });
    share.leave(a.dim, a.norms + block, lds);
    if (sizeof(T) == 2 || !a.amax) return;
    float h = 0.0f;
    for_eights(static_cast<const T*>(a.h), a.h_stride, a.n, a.dim, a.dim, block, blocks, [&](int64_t i, int, const T (&x)[8]) {
        if (a.ids && static_cast<uint32_t>(a.ids[i]) >= static_cast<uint32_t>(a.num_rows)) return;
#pragma unroll
        for (int q = 0; q < 8; ++q) h = fmaxf(h, finite_abs(static_cast<float>(x[q])));
    });
    const uint32_t w_top = block_max_bits(__float_as_uint(largest), lds), h_top = block_max_bits(__float_as_uint(h), lds);
    if (threadIdx.x == 0) {
        a.amax[block] = __uint_as_float(w_top);
        a.amax[kAmaxBlocks + block] = __uint_as_float(h_top);
    }
}

// (10 007 rows against 10 000, 100 columns fp32, 8 MB: 7 us, mostly a launch's.)
__global__ void __launch_bounds__(kThreads) norms_kernel(NormArgs a)
{
    __shared__ uint32_t lds[kThreads / 64];
    norms_of<float>(a, blockIdx.x, gridDim.x, lds);
}

// bf16: rows of H into stages and the table's norms in one launch, and the table's rows where they cannot be used as they lie.
// (Bound by memory: 200 003 x 512 as it lies, 205 MB: 60 us with 8192 rows of H; 199 879 x 438 packed with its norms: 96, 172 as two passes.)
template <bool DIRECT>
__global__ void __launch_bounds__(kThreads) prepare_kernel(PackJobs jobs, NormArgs a)
{
    __shared__ uint32_t lds[kThreads / 64];
    if (blockIdx.y == 1) {
        pack_rows<1, kThreads>(jobs.job[0], blockIdx.x, gridDim.x, reinterpret_cast<float*>(lds));
    } else if constexpr (DIRECT) {
        norms_of<bf16_t>(a, blockIdx.x, gridDim.x, lds);
    } else {
        NormShare share;
        pack_rows<1, kThreads>(jobs.job[1], blockIdx.x, gridDim.x, reinterpret_cast<float*>(lds), [&](int e, const auto& x) { share.see(e, x); });
        share.leave(jobs.job[1].padded, a.norms + blockIdx.x, lds);
    }
}

// ---------------------------------------------------------------------------------------------
// scores of tiles
// ---------------------------------------------------------------------------------------------
struct TileArgs {
    Operand w, h;                  // both by rows
    const int32_t* shift;          // fp32 only: powers of two of W and H
    int64_t n;
    uint32_t num_rows, row_tiles, splits, tokens;   // tokens: padded n
    int32_t steps;                 // stages of a tile
    Softmax* stat;                 // [n][splits]
    float2* best;                  // [n][chunks]
    int64_t chunks;
    float* group;                  // NULL, or [n][groups]: the best of group_tiles tiles' halves one after the other
    int64_t groups;
    uint32_t group_tiles;          // a power of two
    const uint32_t* norms;         // [norm_count]
    uint32_t norm_count;
    uint32_t* norm;
    uint32_t* late;                // NULL, or a number that becomes 0
};

// Tiles, stages and operands are the cross entropy's; a workgroup keeps a tile of H's rows and goes through its split of the table.  What is added to
// a score there, for the moment one multiply-add, for records two instructions, runs on the vector units beside the matrix cores, and is why these wait:
// 8192 rows against 200 003 x 512 bf16, k = 16: 1890 to 2070 us, 0.81 to 0.89 PFLOP/s (k = 0: 1690 to 1790); 10 007 against 10 000 x 100 fp32: 121 (the loss 100).
// Chunks of 64 rows take an exchange between lanes a chunk; those of 16 are a lane's own, four times as many records (80 MB of 8 bytes there).
template <int P, int W, int KS, int CHUNKS>
__global__ void __launch_bounds__(64 * W, 2) answer_tiles_kernel(TileArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * stage_bytes<W>()];
    constexpr int R = rows_of<W>(), MT = W / 2;
    const int lane = threadIdx.x & 63, m0 = first_row<W>(), n0 = first_col<W>();
    uint32_t token_tile, split;
    pair_of(by_xcd(blockIdx.x, gridDim.x), (a.tokens + R - 1) / R, a.splits, token_tile, split);
    const uint32_t per = (a.row_tiles + a.splits - 1) / a.splits, tile0 = split * per;
    if (blockIdx.x == 0) {          // the table's norm, from shares
        uint32_t all = 0;
        for (uint32_t i = threadIdx.x; i < a.norm_count; i += 64 * W) all = max(all, a.norms[i]);
        all = block_max_bits(all, reinterpret_cast<uint32_t*>(lds));
        if (threadIdx.x == 0) {
            *a.norm = all;
            if (a.late) *a.late = 0;
        }
        __syncthreads();
    }
    const float factor = score_factor<P>(a.shift), to_log2 = kLog2e * factor;
    Softmax s[2] = {{kNoScore, 0.0f, 0.0f, 0.0f}, {kNoScore, 0.0f, 0.0f, 0.0f}};
    uint32_t seen = 0;
    float of_group[2] = {-INFINITY, -INFINITY};
    const uint32_t tile1 = min(tile0 + per, a.row_tiles);
    const float low = fmaxf(-3e38f, kNoScore / factor);          // (in units of the sums; below all of them)
    all_scores<P, W, KS>(a.w, a.h, token_tile, 0, tile0, tile1, a.steps, lds, [&](uint32_t tile_row0, f32x16 (&acc)[MT][2]) {
        const uint32_t row0 = tile_row0 + m0;
        ++seen;
        const bool group_ends = CHUNKS != kNone && a.group && ((seen & (a.group_tiles - 1)) == 0 || tile0 + seen == tile1);
        const bool ends = row0 + 32 * MT > a.num_rows;
        const int left = static_cast<int>(a.num_rows - (row0 + lane_row()));     // (the difference is small where both are not)
        if (ends) {
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * im + sum_row(i) >= left) acc[im][0][i] = acc[im][1][i] = low;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float t = low;
            const int64_t token = static_cast<int64_t>(token_tile) * R + n0 + 32 * j + (lane & 31);
            float2* best = a.best + token * a.chunks;
            if constexpr (CHUNKS == kWide) {
#pragma unroll
                for (int c = 0; c < MT / 2; ++c) {
                    Best b{low, low};
#pragma unroll
                    for (int im = 0; im < 2; ++im)
#pragma unroll
                        for (int i = 0; i < 16; ++i) b.see(acc[2 * c + im][j][i], 32 * im + sum_row(i), ~63u);
                    t = fmaxf(t, b.first);
                    b.first = __uint_as_float(__float_as_uint(b.first) | lane_row());
                    b.join_lanes(32);
                    const uint32_t chunk = (row0 >> 6) + c;
                    if (lane < 32 && token < a.n && chunk < a.chunks) best[chunk] = b.record(factor, ~63u);
                }
            } else if constexpr (CHUNKS == kNarrow) {
#pragma unroll
                for (int im = 0; im < MT; ++im) {
                    Best b{low, low};
#pragma unroll
                    for (int i = 0; i < 16; ++i) b.see(acc[im][j][i], i, ~15u);
                    t = fmaxf(t, b.first);
                    const uint32_t chunk = 2 * ((row0 >> 5) + im) + (lane >> 5);
                    if (token < a.n && chunk < a.chunks) best[chunk] = b.record(factor, ~15u);
                }
            } else {
#pragma unroll
                for (int im = 0; im < MT; ++im)
#pragma unroll
                    for (int i = 0; i < 16; ++i) t = fmaxf(t, acc[im][j][i]);
            }
            if constexpr (CHUNKS != kNone) {
                of_group[j] = fmaxf(of_group[j], t);
                if (group_ends) {
                    const float both = fmaxf(of_group[j], __shfl_xor(of_group[j], 32, 64));
                    const uint32_t group = 2 * (split * ((per + a.group_tiles - 1) / a.group_tiles) + (seen - 1) / a.group_tiles) + (m0 ? 1 : 0);
                    if (lane < 32 && token < a.n) a.group[token * a.groups + group] = both * factor;
                    of_group[j] = -INFINITY;
                }
            }
            // (rows behind the last count for nothing, however little `low` is once it is scaled; every row of H goes by its own scores, whichever are beside it)
            const bool large = fabsf(t) * to_log2 > kLargeScore, apart = ends || __any(large);
            if (apart) {
                float top = low;
#pragma unroll
                for (int im = 0; im < MT; ++im)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, acc[im][j][i]);
                t = large ? top : t;
            }
            const float here = t * to_log2, now = fmaxf(s[j].top, here), d = below(s[j].top, now), e = __builtin_amdgcn_exp2f(d);
            const float rest = here < now ? here - now : 0.0f;      // (here - now alone would become one multiply-add, without here's rounding)
            float sum = 0.0f, moment = 0.0f;
            auto add = [&](float x) {
                const float p = __builtin_amdgcn_exp2f(x);
                sum += p;
                moment = fmaf(p, x, moment);
            };
#pragma unroll
            for (int im = 0; im < MT && !apart; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i) add(fmaf(acc[im][j][i], to_log2, -now));
#pragma unroll
            for (int im = 0; im < MT && apart; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i) add(ends && 32 * im + sum_row(i) >= left ? -1000.0f : large ? fmaf(acc[im][j][i] - t, to_log2, rest) : fmaf(acc[im][j][i], to_log2, -now));
            s[j].moment = fmaf(fmaf(s[j].sum, d, s[j].moment), e, moment);
            s[j].sum = fmaf(s[j].sum, e, sum);
            s[j].top = now;
        }
    });
    if (CHUNKS != kNone && a.group) {      // a split that ends early has no more groups
        const uint32_t of_split = (per + a.group_tiles - 1) / a.group_tiles;
        for (uint32_t g = (seen + a.group_tiles - 1) / a.group_tiles; g < of_split; ++g)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t token = static_cast<int64_t>(token_tile) * R + n0 + 32 * j + (lane & 31);
                if (lane < 32 && token < a.n) a.group[token * a.groups + 2 * (split * of_split + g) + (m0 ? 1 : 0)] = -INFINITY;
            }
    }
    // lanes l and l + 32 and the two wavefronts of a column have the same rows of H
    Softmax* shared = reinterpret_cast<Softmax*>(lds);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        join_lanes(s[j], 32);
        if (lane < 32) shared[(m0 ? R : 0) + n0 + 32 * j + lane] = s[j];
    }
    __syncthreads();
    const uint32_t row = token_tile * R + threadIdx.x;
    if (threadIdx.x < R && row < a.n) {
        Softmax p = shared[threadIdx.x];
        const Softmax q = shared[R + threadIdx.x];
        join(p, q.top, q.sum, q.moment);
        a.stat[static_cast<int64_t>(row) * a.splits + split] = p;
    }
}

// ---------------------------------------------------------------------------------------------
// few rows of H: the table streams through registers once, straight from memory
// ---------------------------------------------------------------------------------------------
// As for the cross entropy's loss: a wavefront has 16 table rows at a time, as the matrix cores' first operand; H lies in LDS as second operands, in
// blocks of 16 rows; fp32 operands are split into three bf16 parts.  Bound by reading the table: 200 003 x 256 bf16 for one row 21 us, 4.9 TB/s; fp32 for 16 rows
// 40 to 52 us, 3.9 to 5.1 TB/s.
struct FewAnswerArgs {
    const void *h, *w;
    int64_t h_stride, w_stride;
    const int32_t* ids;            // NULL, or whose rows outside the table do not count
    uint32_t n, num_rows;
    int32_t dim, steps;            // steps of 32 elements
    Softmax* stat;                 // [n][workgroups]
    float2* best;                  // NULL, or [n][chunks]
    int64_t chunks;
    uint32_t* norms;               // [workgroups]
};

template <class T, int BLOCKS, int THREADS>
__global__ void __launch_bounds__(THREADS) answer_few_kernel(FewAnswerArgs a)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, AHEAD = sizeof(T) == 4 ? 4 : 8, CHAINS = BLOCKS == 1 ? 4 : BLOCKS == 2 ? 2 : 1;
    constexpr bool APART = PARTS > 1 && BLOCKS < 4;
    extern __shared__ __align__(16) unsigned char few_lds[];       // [blocks][steps][parts][64 lanes] 16 bytes
    bf16x8* hs = reinterpret_cast<bf16x8*>(few_lds);
    __shared__ Softmax shared[THREADS / 64][BLOCKS * 16];
    __shared__ uint32_t norms[THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    for (int i = wave; i < BLOCKS * a.steps; i += THREADS / 64) {
        const int block = i / a.steps, step = i % a.steps;
        const uint32_t t = block * 16 + col;
        T x[8];
        if (t < a.n && (!a.ids || static_cast<uint32_t>(a.ids[t]) < a.num_rows)) {
            load_eight(static_cast<const T*>(a.h) + t * a.h_stride, step * 32 + quarter * 8, a.dim, x);
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = from_float<T>(0.0f);
        }
        bf16x8 parts[PARTS];
        split_bf16<PARTS>(x, parts);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) hs[(i * PARTS + p) * 64 + lane] = parts[p];
    }
    Softmax s[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) s[b] = Softmax{kNoScore, 0.0f, 0.0f, 0.0f};
    uint32_t most = 0;
    __syncthreads();
    const uint32_t tiles = (a.num_rows + 15) / 16, stride = gridDim.x * (THREADS / 64);
    for (uint32_t tile = blockIdx.x * (THREADS / 64) + wave; tile < tiles; tile += stride) {
        const T* row = static_cast<const T*>(a.w) + static_cast<int64_t>(min(tile * 16 + col, a.num_rows - 1)) * a.w_stride;
        f32x4 sums[BLOCKS][CHAINS], small[BLOCKS];
        float squares = 0.0f;
        uint32_t some = 0;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            small[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < CHAINS; ++c) sums[b][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        for (int s0 = 0; s0 < a.steps; s0 += AHEAD) {
            T x[AHEAD][8];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (s0 + k < a.steps) load_eight(row, (s0 + k) * 32 + quarter * 8, a.dim, x[k]);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (s0 + k >= a.steps) break;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float y = static_cast<float>(x[k][q]);
                    squares = fmaf(y, y, squares);
                }
                some |= magnitude_bits(x[k]);
                bf16x8 w[PARTS];
                split_bf16<PARTS>(x[k], w);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    bf16x8 h[PARTS];
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) h[p] = hs[((b * a.steps + s0 + k) * PARTS + p) * 64 + lane];
                    // (the smallest products first)
#pragma unroll
                    for (int sum_of_parts = PARTS - 1; sum_of_parts >= 0; --sum_of_parts) {
                        f32x4& to = APART && sum_of_parts > 0 ? small[b] : sums[b][k % CHAINS];
#pragma unroll
                        for (int p = 0; p <= sum_of_parts; ++p) to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[p], h[sum_of_parts - p], to, 0, 0, 0);
                    }
                }
            }
        }
        if (some && squares < 0x1p-126f) squares = 0x1p-126f;      // (squares of small values may be 0)
        most = max(most, __float_as_uint(squares) & 0x7FFFFFFFu);
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            f32x4& acc = sums[b][0];
#pragma unroll
            for (int c = 1; c < CHAINS; ++c) acc += sums[b][c];
            if (APART) acc += small[b];
            Best best;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (tile * 16 + quarter * 4 + i >= a.num_rows) acc[i] = kNoScore;
                best.see(acc[i], i, ~15u);
            }
            float t = best.first;
            const bool large = fabsf(t) * kLog2e > kLargeScore;
            if (large) t = fmaxf(fmaxf(acc[0], acc[1]), fmaxf(acc[2], acc[3]));
            const float here = t * kLog2e, now = fmaxf(s[b].top, here), d = below(s[b].top, now), e = __builtin_amdgcn_exp2f(d);
            const float rest = here < now ? here - now : 0.0f;      // (here - now alone would become one multiply-add, without here's rounding)
            float sum = 0.0f, moment = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = large ? fmaf(acc[i] - t, kLog2e, rest) : fmaf(acc[i], kLog2e, -now), p = __builtin_amdgcn_exp2f(x);
                sum += p;
                moment = fmaf(p, x, moment);
            }
            s[b].moment = fmaf(fmaf(s[b].sum, d, s[b].moment), e, moment);
            s[b].sum = fmaf(s[b].sum, e, sum);
            s[b].top = now;
            if (a.best) {
                best.first = __uint_as_float(__float_as_uint(best.first) | (quarter * 4));
                best.join_lanes(16);
                best.join_lanes(32);
                const uint32_t t = b * 16 + col;
                if (lane < 16 && t < a.n) a.best[t * a.chunks + tile] = make_float2(best.first, best.second);
            }
        }
    }
    // (a bound for all of the wavefront's rows: of each quarter the largest share)
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), o, 64)));
    float norm = __uint_as_float(most);
    norm += __shfl_xor(norm, 16, 64);
    norm += __shfl_xor(norm, 32, 64);
    const uint32_t all = block_max_bits(__float_as_uint(norm) & 0x7FFFFFFFu, norms);
    if (threadIdx.x == 0) a.norms[blockIdx.x] = all;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        join_lanes(s[b], 16);
        join_lanes(s[b], 32);
        if (lane < 16) shared[wave][b * 16 + lane] = s[b];
    }
    __syncthreads();
    if (threadIdx.x < a.n) {
        Softmax p = shared[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) join(p, shared[w][threadIdx.x].top, shared[w][threadIdx.x].sum, shared[w][threadIdx.x].moment);
        a.stat[static_cast<int64_t>(threadIdx.x) * gridDim.x + blockIdx.x] = p;
    }
}

// ---------------------------------------------------------------------------------------------
// answers
// ---------------------------------------------------------------------------------------------
struct FinishArgs {
    const void *h, *w;
    int64_t h_stride, w_stride;
    const int32_t* ids;
    int64_t n;
    uint32_t num_rows, splits, norm_count, k;
    int32_t dim, kind;             // kind of chunks
    const Softmax* stat;           // [n][splits]
    const uint32_t* norms;
    const int32_t* shift;          // NULL, or powers of two of W and H
    const float2* best;            // [n][chunks]
    int64_t chunks;
    const float* group;            // NULL, or [n][groups]
    uint32_t groups, group_tiles, per_split, row_tiles, tile_rows;
    uint32_t* late;                // NULL, or number of rows that sixteen wavefronts take over, and the rows
    float *logp, *lse, *entropy;   // logp, entropy: NULL where not wanted
    int32_t* top_ids;
    float* top_logp;
};

// A row of H is a team's: a wavefront where there are many rows (four teams a workgroup, which never wait for one another); otherwise four, or sixteen
// where there are many chunks (one row, 12 501 chunks: 15 us with sixteen; 48 rows, 625 chunks: 10.5 with four, 14.5 with sixteen).  Where there are
// many rows and many chunks, the wavefront does not look through all records: tiles also leave the best of every group of them behind, the threshold
// follows from these, and only the records of groups that reach it are read.  Rows of many candidates are left to sixteen wavefronts, as the launch would
// wait for them (8192 rows of 200 003 x 512, k = 16: 170 us with neither, 52 and 58 with both).
// Bound by chains of dependent loads (records, rows of the table) and by instructions, not by memory.
template <int WAVES> constexpr int threads_of() { return WAVES == 1 ? kThreads : 64 * WAVES; }
template <int WAVES> constexpr int most_found() { return WAVES == 1 ? 192 : WAVES == 4 ? 1024 : 2048; }       // candidates that a team looks at together
constexpr uint32_t kMostGroups = 2048, kMostHits = 256;         // groups of a row; those that a wavefront notes

template <int WAVES>
__device__ __forceinline__ void team_sync()
{
    if (WAVES == 1) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    else __syncthreads();
}

template <int WAVES>
struct Team {
    uint32_t ids[64 + most_found<WAVES>() + 1];        // the best so far, candidates, the given id
    double scores[64 + most_found<WAVES>() + 1];
    uint32_t next_ids[64];
    double next_scores[64];
    Softmax stats[WAVES];
    float norms[WAVES];
    float maxima[WAVES == 1 ? 1 : 64 * WAVES];
    uint16_t hits[WAVES == 1 ? kMostHits : 1];         // groups that reach the threshold
    uint32_t count, bits[WAVES];
    float threshold;
};

// Scores of table rows, LANES lanes each, with products and sums in 64 bits, in an order that depends on dim alone.  A row's last piece ends with the row:
// what it has in common with the piece before it is multiplied with zeros.  FLIGHT rows of a group of lanes are in flight; of their sums a lane passes
// on half in each exchange, until it has the row that its last bits name.
template <class T, int FLIGHT, int LANES>
__device__ __forceinline__ void exact_scores_by(const FinishArgs& a, const T* h, const uint32_t* ids, double* scores, uint32_t count, uint32_t thread, uint32_t threads)
{
    constexpr int BITS = FLIGHT == 8 ? 3 : FLIGHT == 4 ? 2 : 1;
    static_assert(1 << BITS == FLIGHT);
    const int lane = thread % LANES;
    for (uint32_t c = thread / LANES * FLIGHT; c < count; c += threads / LANES * FLIGHT) {
        const T* row[FLIGHT];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) row[f] = static_cast<const T*>(a.w) + static_cast<int64_t>(ids[min(c + f, count - 1)]) * a.w_stride;
        double sum[FLIGHT] = {};
        for (int e = lane * 8; e < a.dim; e += 8 * LANES) {
            const int at = min(e, a.dim - 8);
            T x[FLIGHT][8], y[8];
            __builtin_memcpy(y, h + at, 8 * sizeof(T));
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) __builtin_memcpy(x[f], row[f] + at, 8 * sizeof(T));
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const double z = at + q >= e ? static_cast<double>(static_cast<float>(y[q])) : 0.0;
#pragma unroll
                for (int f = 0; f < FLIGHT; ++f) sum[f] = fma(static_cast<double>(static_cast<float>(x[f][q])), z, sum[f]);
            }
        }
        uint32_t which = 0;
#pragma unroll
        for (int bit = 0; bit < BITS; ++bit) {
            const bool upper = lane >> bit & 1;
            const int half = FLIGHT >> (bit + 1);
            if (upper) which += half;
#pragma unroll
            for (int f = 0; f < half; ++f) {
                const double mine = upper ? sum[f + half] : sum[f], theirs = upper ? sum[f] : sum[f + half];
                sum[f] = mine + __shfl_xor(theirs, 1 << bit, 64);
            }
        }
#pragma unroll
        for (int o = FLIGHT; o < LANES; o <<= 1) sum[0] += __shfl_xor(sum[0], o, 64);
        if (lane < FLIGHT && c + which < count) scores[c + which] = sum[0];
    }
}

template <class T, int WAVES>
__device__ __forceinline__ void exact_scores(const FinishArgs& a, const T* h, const uint32_t* ids, double* scores, uint32_t count, uint32_t thread)
{
    constexpr int FLIGHT = WAVES == 1 ? 4 : 2;
    if (a.dim > 256) {
        exact_scores_by<T, FLIGHT, 64>(a, h, ids, scores, count, thread, 64 * WAVES);
    } else if (a.dim >= 8) {
        exact_scores_by<T, FLIGHT, 16>(a, h, ids, scores, count, thread, 64 * WAVES);
    } else {
        for (uint32_t c = thread; c < count; c += 64 * WAVES) {
            const T* row = static_cast<const T*>(a.w) + static_cast<int64_t>(ids[c]) * a.w_stride;
            double sum = 0.0;
            for (int e = 0; e < a.dim; ++e) sum = fma(static_cast<double>(static_cast<float>(row[e])), static_cast<double>(static_cast<float>(h[e])), sum);
            scores[c] = sum;
        }
    }
}

// Floats as numbers of the same order.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }

// A bound that k of a wavefront's values reach, within 2^-9 below the k-th largest: bit after bit, counted by ballots.
template <int VALUES>
__device__ __forceinline__ float reached_by(const float (&x)[VALUES], uint32_t k)
{
    uint32_t key[VALUES], t = 0;
#pragma unroll
    for (int v = 0; v < VALUES; ++v) key[v] = ordered(x[v]);
    for (uint32_t bit = 0x80000000u; bit >= 1u << 14; bit >>= 1) {
        uint32_t count = 0;
#pragma unroll
        for (int v = 0; v < VALUES; ++v) count += __popcll(__ballot(key[v] >= (t | bit)));
        if (count >= k) t |= bit;
    }
    return from_ordered(t);
}

// A thread's records c0 + thread, + threads .. below c1, all loads in flight.  A team of sixteen wavefronts keeps them in registers where these are all
// (fewer wavefronts would lose more to the registers than a second read from L2 costs).
template <int WAVES> constexpr int at_once() { return WAVES == 16 ? 16 : 8; }

template <int THREADS, int COUNT>
__device__ __forceinline__ void load_records(const float2* best, int64_t c0, int64_t c1, uint32_t thread, float2 (&b)[COUNT])
{
#pragma unroll
    for (int f = 0; f < COUNT; ++f) {
        const int64_t c = c0 + thread + f * THREADS;
        b[f] = make_float2(-INFINITY, -INFINITY);
        if (c < c1) b[f] = best[c];
    }
}

// A softmax's logarithm of its sum, in powers of two (of a mantissa, whose logarithm is below 1 and as much more exact).
__device__ __forceinline__ double log2_of(float top, float sum)
{
    int e;
    const float m = frexpf(sum, &e);
    return static_cast<double>(top) + e + static_cast<double>(log2f(m));
}

// The answers of row i, by a team.
template <class T, int WAVES>
__device__ __forceinline__ void answer_row(const FinishArgs& a, Team<WAVES>& team, int64_t i)
{
    constexpr uint32_t MOST = most_found<WAVES>(), THREADS = 64 * WAVES;
    const uint32_t thread = threadIdx.x % THREADS, lane = thread & 63, wave = thread >> 6;
    // (what is loaded first does not wait for the id)
    const T* h = static_cast<const T*>(a.h) + i * a.h_stride;
    const uint32_t id = a.ids ? static_cast<uint32_t>(a.ids[i]) : 0xFFFFFFFFu, k = a.k;
    Softmax s{kNoScore, 0.0f, 0.0f, 0.0f};
    uint32_t largest = 0;
    if (thread < a.splits) s = a.stat[i * a.splits + thread];
    if (thread < a.norm_count) largest = a.norms[thread];
    constexpr int HELD = at_once<WAVES>();
    float2 record[HELD];
    const float2* best = a.best + i * a.chunks;
    const bool held = WAVES == 16 && a.chunks <= HELD * THREADS;
    if (k && held) load_records<THREADS>(best, 0, a.chunks, thread, record);
    int32_t* top_ids = a.top_ids + i * k;
    float* top_logp = a.top_logp + i * k;
    if (a.ids && id >= a.num_rows) {
        if (thread == 0) {
            a.lse[i] = 0.0f;
            if (a.logp) a.logp[i] = 0.0f;
            if (a.entropy) a.entropy[i] = 0.0f;
        }
        if (thread < k) {
            top_ids[thread] = -1;
            top_logp[thread] = -INFINITY;
        }
        return;
    }
    // the row's norm and softmax, and the table's largest norm
    float squares = 0.0f;
    for (int e = thread * 8; e < a.dim; e += 8 * THREADS) {
        T x[8];
        load_eight(h, e, a.dim, x);
#pragma unroll
        for (int q = 0; q < 8; ++q) squares = fmaf(static_cast<float>(x[q]), static_cast<float>(x[q]), squares);
        if (magnitude_bits(x) && squares < 0x1p-126f) squares = 0x1p-126f;      // (squares of small values may be 0)
    }
    for (uint32_t p = thread + THREADS; p < a.splits; p += THREADS) {
        const Softmax q = a.stat[i * a.splits + p];
        join(s, q.top, q.sum, q.moment);
    }
    for (uint32_t p = thread + THREADS; p < a.norm_count; p += THREADS) largest = max(largest, a.norms[p]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        join_lanes(s, o);
        squares += __shfl_xor(squares, o, 64);
        largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), o, 64)));
    }
    if constexpr (WAVES > 1) {
        if (lane == 0) {
            team.stats[wave] = s;
            team.norms[wave] = squares;
            team.bits[wave] = largest;
        }
        __syncthreads();
        s = team.stats[lane % WAVES];
        squares = team.norms[lane % WAVES];
        largest = team.bits[lane % WAVES];
#pragma unroll
        for (int o = 1; o < WAVES; o <<= 1) {
            join_lanes(s, o);
            squares += __shfl_xor(squares, o, 64);
            largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), o, 64)));
        }
    }
    // (joined in another order a sum is rounded otherwise: what every thread goes on with is the first lane's, the same in all wavefronts)
    auto first_lane = [](float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); };
    s = Softmax{first_lane(s.top), first_lane(s.sum), first_lane(s.moment), 0.0f};
    // Bounds of both norms: squares and roots are rounded, and those of small values left something out.
    const float left_out = 0x1p-62f * sqrtf(static_cast<float>(a.dim));
    const float h_norm = squares == 0.0f ? 0.0f : 1.001f * sqrtf(squares) + left_out;
    const float w_norm = largest == 0 ? 0.0f : 1.001f * sqrtf(__uint_as_float(largest)) + left_out;
    const float product = h_norm * w_norm;
    const double lse = log2_of(s.top, s.sum) * 0.693147180559945309;
    const bool bad = !(product < kMostScore), zero = h_norm == 0.0f || w_norm == 0.0f;       // bad: a value that is not finite, or scores that fp32 may not hold
    if (thread == 0) {
        a.lse[i] = bad ? NAN : static_cast<float>(lse);
        if (a.entropy) a.entropy[i] = bad ? NAN : (log2f(s.sum) - s.moment / s.sum) * kLn2;
        if (bad && a.logp) a.logp[i] = NAN;
    }
    if (bad || k == 0 || zero) {
        // (all scores are 0 where a norm is: the lowest ids)
        if (thread < k) {
            const bool is = !bad && thread < a.num_rows;
            top_ids[thread] = is ? static_cast<int32_t>(thread) : -1;
            top_logp[thread] = bad ? NAN : is ? static_cast<float>(-lse) : -INFINITY;
        }
        if (bad || !a.logp) return;
        if (thread == 0) team.ids[0] = id;
        team_sync<WAVES>();
        exact_scores<T, WAVES>(a, h, team.ids, team.scores, 1, thread);
        if (thread == 0) a.logp[i] = static_cast<float>(team.scores[0] - lse);
        return;
    }
    // How far a score of the pass may be off: rounded products and sums (a chain of dim / 16 of them), and what halves of the rows leave out.
    float off_by = static_cast<float>(a.dim / 16 + 8) * 0x1p-23f * product;
    if (sizeof(T) == 4) off_by += 0x1p-20f * product;
    if (a.shift) off_by += 0x1p-36f * sqrtf(static_cast<float>(a.dim)) * w_norm * (h_norm + ldexpf(1.0f, 14 - a.shift[1]));
    off_by = 2.0f * off_by + 1e-36f * a.dim;
    // t: what k of the chunks' best reach: of each lane's best two, or of each thread's best
    float mine[2] = {-INFINITY, -INFINITY};
    auto see = [&](const float2 (&b)[HELD]) {
#pragma unroll
        for (int f = 0; f < HELD; ++f) {
            if (WAVES == 1) mine[1] = __builtin_amdgcn_fmed3f(mine[0], mine[1], b[f].x);
            mine[0] = fmaxf(mine[0], b[f].x);
        }
    };
    bool grouped = WAVES == 1 && a.group;
    const float* group = a.group + i * a.groups;
    if (grouped) {
        for (uint32_t g0 = 0; g0 < a.groups; g0 += HELD * THREADS) {
#pragma unroll
            for (int f = 0; f < HELD; ++f) {
                const uint32_t g = g0 + thread + f * THREADS;
                record[f] = make_float2(g < a.groups ? group[g] : -INFINITY, 0.0f);
            }
            see(record);
        }
    } else if (held) {
        see(record);
    } else {
        for (int64_t c = 0; c < a.chunks; c += HELD * THREADS) {
            load_records<THREADS>(best, c, a.chunks, thread, record);
            see(record);
        }
    }
    float t = -INFINITY;
    if ((grouped ? a.groups : a.chunks) >= k) {
        if constexpr (WAVES == 1) {
            t = reached_by(mine, k);
        } else {
            team.maxima[thread] = mine[0];
            __syncthreads();
            if (wave == 0) {
                float all[WAVES];
#pragma unroll
                for (int w = 0; w < WAVES; ++w) all[w] = team.maxima[w * 64 + lane];
                t = reached_by(all, k);
                if (lane == 0) team.threshold = t;
            }
            __syncthreads();
            t = team.threshold;
        }
        t -= 2.0f * off_by + fabsf(t) * 0x1p-15f;
    }
    // The records to look at: of all chunks, or of the chunks of groups that reach t, one group after the other.
    const int log2_rows = chunk_log2(a.kind);
    const uint32_t per_tile = a.tile_rows >> (log2_rows + 1), per_group = per_tile * a.group_tiles;
    int64_t records = a.chunks;
    if constexpr (WAVES == 1) {
        if (grouped) {
            uint32_t hits = 0;
            for (uint32_t g0 = 0; g0 < a.groups; g0 += 64) {
                const uint32_t g = g0 + lane;
                const bool hit = g < a.groups && group[g] >= t;
                const uint64_t mask = __ballot(hit);
                const uint32_t to = hits + __popcll(mask & ((1ull << lane) - 1));
                if (hit && to < kMostHits) team.hits[to] = static_cast<uint16_t>(g);
                hits += __popcll(mask);
            }
            if (hits <= kMostHits) records = static_cast<int64_t>(hits) * per_group;
            else grouped = false;
            team_sync<WAVES>();
        }
    }
    // (of a group: 2 (its split, its place there) + its half of the tiles)
    const uint32_t groups_of_split = grouped ? (a.per_split + a.group_tiles - 1) / a.group_tiles : 1;
    auto chunk_of = [&](int64_t r) -> int64_t {
        if (!grouped) return r;
        const uint32_t at = static_cast<uint32_t>(r), group_id = team.hits[at / per_group], in = at % per_group;
        const uint32_t split = (group_id >> 1) / groups_of_split, tile = split * a.per_split + (group_id >> 1) % groups_of_split * a.group_tiles + in / per_tile;
        const bool there = tile < min((split + 1) * a.per_split, a.row_tiles);
        const int64_t first = (static_cast<int64_t>(tile) * a.tile_rows + (group_id & 1) * (a.tile_rows / 2)) >> log2_rows;
        return there ? first + in % per_tile : a.chunks;
    };
    // Candidates of records r0 .. r1 - 1 go to team.ids[64 ..]: a chunk's best, or all of its rows.  Returns their number, of which those beyond MOST
    // are not written.
    auto collect = [&](int64_t r0, int64_t r1) {
        uint32_t count = 0;
        if (WAVES > 1) {
            if (thread == 0) team.count = 0;
            __syncthreads();
        }
        auto place_for = [&](uint32_t some) {
            uint32_t to = count;
            if constexpr (WAVES == 1) {
                count += some;
            } else {
                if (lane == 0) to = atomicAdd(&team.count, some);
                to = __builtin_amdgcn_readfirstlane(to);
            }
            return to;
        };
        auto write = [&](bool is, uint32_t row) {
            const uint64_t mask = __ballot(is);
            if (!mask) return;
            const uint32_t to = place_for(__popcll(mask)) + __popcll(mask & ((1ull << lane) - 1));
            if (is && to < MOST) team.ids[64 + to] = row;
        };
        auto row_of = [&](uint32_t chunk, uint32_t place) {
            return a.kind == kNarrow ? (chunk >> 1) * 32 + 8 * (place >> 2) + 4 * (chunk & 1) + (place & 3) : (chunk << log2_rows) + place;
        };
        for (int64_t r = held ? 0 : r0; r < r1; r += HELD * THREADS) {
            uint32_t chunk[HELD];
#pragma unroll
            for (int f = 0; f < HELD; ++f) {
                const int64_t mine = r + thread + f * THREADS, c = mine >= r0 && mine < r1 ? chunk_of(mine) : a.chunks;
                chunk[f] = static_cast<uint32_t>(c);
                if (held) {
                    if (c >= a.chunks) chunk[f] = 0xFFFFFFFFu;
                } else {
                    record[f] = make_float2(-INFINITY, -INFINITY);
                    if (c < a.chunks) record[f] = best[c];
                    else chunk[f] = 0xFFFFFFFFu;
                }
            }
#pragma unroll
            for (int f = 0; f < HELD; ++f) {
                const bool reaches = chunk[f] != 0xFFFFFFFFu && record[f].x >= t;
                if (!__any(reaches)) continue;
                const bool whole = reaches && record[f].y >= t;
                const uint32_t one = row_of(chunk[f], __float_as_uint(record[f].x) & ((1u << log2_rows) - 1));
                write(reaches && !whole && one < a.num_rows, one);       // (narrow chunks behind the last row hold nothing)
                for (uint64_t wholes = __ballot(whole); wholes; wholes &= wholes - 1) {
                    const uint32_t all = __builtin_amdgcn_readlane(chunk[f], __builtin_ctzll(wholes)), row = row_of(all, lane);
                    write(lane < 1u << log2_rows && row < a.num_rows, row);
                }
            }
        }
        if (WAVES > 1) {
            __syncthreads();
            count = team.count;
            __syncthreads();        // (the next call begins by clearing it, at once where there was no room: all have read it by then)
        }
        return count;
    };
    const int64_t part = MOST >> log2_rows;         // chunks whose rows all fit
    int64_t at = 0, to = 0, span = records;         // so many records at a time that there is room for their candidates
    auto next_candidates = [&]() {
        at = to;
        while (true) {
            to = min(at + span, records);
            const uint32_t count = collect(at, to);
            if (count <= MOST) return count;
            span = max(span / 2, part);
        }
    };
    uint32_t count = next_candidates(), have = 0;
    // A row of many candidates would take one wavefront several times as long as the others: sixteen take it over.
    if (WAVES == 1 && a.late && count + (records - to) > a.k + (a.kind == kWide ? 40u : 112u)) {
        if (lane == 0) a.late[1 + atomicAdd(a.late, 1u)] = static_cast<uint32_t>(i);
        return;
    }
    bool given = a.logp != nullptr;
    while (true) {
        if (given && thread == 0) team.ids[64 + count] = id;
        team_sync<WAVES>();
        exact_scores<T, WAVES>(a, h, team.ids + 64, team.scores + 64, count + given, thread);
        team_sync<WAVES>();
        if (given && thread == 0) a.logp[i] = static_cast<float>(team.scores[64 + count] - lse);
        given = false;
        // the best so far lie in front of the candidates
        const uint32_t all = have + count, base = 64 - have;
        const bool last = to >= records;
        for (uint32_t c = thread; c < all; c += THREADS) {
            const uint32_t my_id = team.ids[base + c];
            const double my_score = team.scores[base + c];
            uint32_t rank = 0, o = 0;
            auto beats = [&](double other, uint32_t other_id) { return other > my_score || (other == my_score && other_id < my_id); };
            for (; o + 8 <= all; o += 8) {
                double other[8];
                uint32_t other_id[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    other[q] = team.scores[base + o + q];
                    other_id[q] = team.ids[base + o + q];
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) rank += beats(other[q], other_id[q]);
            }
            for (; o < all; ++o) rank += beats(team.scores[base + o], team.ids[base + o]);
            if (rank >= k) continue;
            if (last) {
                top_ids[rank] = static_cast<int32_t>(my_id);
                top_logp[rank] = static_cast<float>(my_score - lse);
            } else {
                team.next_ids[rank] = my_id;
                team.next_scores[rank] = my_score;
            }
        }
        have = min(all, k);
        if (last) break;
        team_sync<WAVES>();
        if (thread < have) {
            team.ids[64 - have + thread] = team.next_ids[thread];
            team.scores[64 - have + thread] = team.next_scores[thread];
        }
        team_sync<WAVES>();
        if (have == k) {
            const float least = static_cast<float>(team.scores[63]);
            t = fmaxf(t, least - off_by - fabsf(least) * 0x1p-15f);
        }
        count = next_candidates();
    }
    if (thread >= have && thread < k) {
        top_ids[thread] = -1;
        top_logp[thread] = -INFINITY;
    }
}

template <class T, int WAVES>
__global__ void __launch_bounds__(threads_of<WAVES>()) answers_kernel(FinishArgs a)
{
    constexpr int TEAMS = threads_of<WAVES>() / 64 / WAVES;
    __shared__ Team<WAVES> teams[TEAMS];
    const uint32_t which = threadIdx.x / (64 * WAVES);
    const int64_t i = static_cast<int64_t>(blockIdx.x) * TEAMS + which;
    if (i < a.n) answer_row<T, WAVES>(a, teams[which], i);
}

// Rows that wavefronts left, sixteen for each: a workgroup's LDS leaves room for one on a CU, and 512 workgroups share all rows.  (8192 rows of 200 003 x 512: 58 us;
// with no row left, 4.)
template <class T>
__global__ void __launch_bounds__(1024) late_answers_kernel(FinishArgs a)
{
    __shared__ Team<16> team;
    const uint32_t count = a.late[0];
    for (uint32_t r = blockIdx.x; r < count; r += gridDim.x) {
        answer_row<T, 16>(a, team, a.late[1 + r]);
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct AnswerWs : Packs {
    uint32_t row_tiles, splits;
    int32_t few_blocks, kind;
    int64_t chunks;
    uint32_t groups, group_tiles, per_split;
    float* group;
    uint32_t *norms, *norm, *late;
    Softmax* stat;
    float2* best;
    size_t total;
};

// Wide chunks where hardly any has two of the best k: the rows of those that have are looked at again, k^2 64^2 / (2 num_rows) of them about.
int chunks_of(int64_t num_rows, int32_t k) { return k == 0 ? kNone : static_cast<int64_t>(k) * k * 320 > num_rows ? kNarrow : kWide; }

int64_t chunk_count(int64_t num_rows, int kind) { return kind == kNone ? 0 : kind == kNarrow ? 2 * ceil_div(num_rows, 32) : ceil_div(num_rows, int64_t{1} << chunk_log2(kind)); }

AnswerWs answer_layout(int64_t n, int64_t num_rows, int32_t dim, int32_t type, int32_t k, char* base)
{
    AnswerWs w{};
    w.parts = type == NE_F32 ? 2 : 1;
    const int64_t step = w.parts == 1 ? step_of<1>() : step_of<2>();
    w.padded = static_cast<int32_t>(round_up(dim, step));
    w.tokens = round_up(n, step);
    w.large_scores = large_scores(n, num_rows, dim, w.parts);
    const int64_t side = w.large_scores ? 256 : 128, token_tiles = ceil_div(w.tokens, side);
    w.row_tiles = static_cast<uint32_t>(ceil_div(num_rows, side));
    w.few_blocks = few_blocks_of(n, num_rows, dim, w.parts);
    w.kind = w.few_blocks && k ? kStreamed : chunks_of(num_rows, k);
    w.chunks = chunk_count(num_rows, w.kind);
    Carver take{base};
    w.norms = take.get<uint32_t>(kMostPack);
    w.norm = take.get<uint32_t>(1);
    if (w.few_blocks) {
        const bool alone = few_bytes_of(w.few_blocks, dim, w.parts) > kFewBytes;
        w.splits = static_cast<uint32_t>(std::min<int64_t>(ceil_div(num_rows, alone ? 128 : 64), alone ? 256 : kFewGroups));
    } else {
        w.splits = splits_of(w.row_tiles, token_tiles, w.large_scores);
        w.amax = take.get<float>(2 * kAmaxBlocks);
        w.shift = take.get<int32_t>(3);
        for (int p = 0; p < w.parts; ++p) {
            w.h[p] = take.get<uint16_t>(static_cast<size_t>(w.tokens) * w.padded);
            w.w[p] = take.get<uint16_t>(static_cast<size_t>(num_rows) * w.padded);
        }
    }
    w.stat = take.get<Softmax>(static_cast<size_t>(w.splits) * n);
    w.best = k ? take.get<float2>(static_cast<size_t>(w.chunks) * n) : nullptr;
    w.late = k && !w.few_blocks && n > kTeamsOfMany ? take.get<uint32_t>(static_cast<size_t>(n) + 1) : nullptr;
    w.per_split = static_cast<uint32_t>(ceil_div(w.row_tiles, w.splits));
    if (!w.few_blocks && n > kTeamsOfMany && w.chunks > kUngrouped) {
        // as large as leaves several times k of them, and at most kMostGroups
        auto groups = [&](uint32_t tiles) { return static_cast<uint32_t>(2 * w.splits * ceil_div(w.per_split, tiles)); };
        w.group_tiles = 1;
        while (w.group_tiles < w.per_split && (groups(w.group_tiles) > kMostGroups || groups(2 * w.group_tiles) >= std::max<uint32_t>(256, 6 * k))) w.group_tiles *= 2;
        w.groups = groups(w.group_tiles);
        w.group = take.get<float>(static_cast<size_t>(w.groups) * n);
    }
    w.total = take.total();
    return w;
}

// Bytes of a workspace for up to n rows: bounds of what answer_layout takes, each growing with n.
size_t answer_bytes(int64_t n, int64_t num_rows, int32_t dim, int32_t type, int32_t k)
{
    const int parts = type == NE_F32 ? 2 : 1;
    const int64_t step = parts == 1 ? step_of<1>() : step_of<2>(), tokens = round_up(n, step), padded = round_up(dim, step), few = std::min<int64_t>(n, 192);
    int64_t bytes = 32 << 10;
    // shares of few rows; of tiles: as many workgroups as run in four rounds, or one for every tile
    bytes += (std::min<int64_t>(ceil_div(num_rows, 64), kFewGroups) * few + tokens + std::min<int64_t>(ceil_div(num_rows, 128) * tokens, 4 * 512 * 128)) * 16;
    bytes += std::max(chunk_count(num_rows, k ? kStreamed : kNone) * few, chunk_count(num_rows, chunks_of(num_rows, k)) * n) * 8;
    if (k && n > kTeamsOfMany) bytes += (kMostGroups + 1) * 4 * n;
    if (!few_blocks_of(n, num_rows, dim, parts)) bytes += parts * 2 * padded * (tokens + num_rows);
    return static_cast<size_t>(bytes);
}

// The workspace of up to n rows, and the number that a call of n rows carves out of it, whichever is larger.
size_t answer_need(int64_t n, int64_t num_rows, int32_t dim, int32_t type, int32_t k)
{
    return std::max(answer_bytes(n, num_rows, dim, type, k), answer_layout(n, num_rows, dim, type, k, nullptr).total);
}

template <class T>
hipError_t few_answers(const SoftmaxCall& x, const AnswerWs& w, hipStream_t st)
{
    FewAnswerArgs a{};
    a.w = x.w; a.h_stride = x.h_stride; a.w_stride = x.w_stride; a.num_rows = static_cast<uint32_t>(x.num_rows); a.dim = x.dim;
    a.steps = static_cast<int32_t>(ceil_div(x.dim, 32)); a.chunks = w.chunks; a.norms = w.norms;
    const size_t lds = static_cast<size_t>(few_bytes_of(w.few_blocks, x.dim, w.parts));
    auto launch = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(w.splits), dim3(threads), lds, st, a); };
    for (int64_t base = 0; base < x.n; base += 16 * w.few_blocks) {
        a.h = static_cast<const T*>(x.h) + base * x.h_stride; a.ids = x.targets ? x.targets + base : nullptr;
        a.n = static_cast<uint32_t>(std::min<int64_t>(x.n - base, 16 * w.few_blocks));
        a.stat = w.stat + base * w.splits; a.best = w.best ? w.best + base * w.chunks : nullptr;
        if (lds > kFewBytes) {
            if (w.few_blocks == 1) launch(answer_few_kernel<T, 1, 512>, 512);
            else if (w.few_blocks == 2) launch(answer_few_kernel<T, 2, 512>, 512);
            else launch(answer_few_kernel<T, 4, 512>, 512);
        } else {
            if (w.few_blocks == 1) launch(answer_few_kernel<T, 1, 256>, 256);
            else if (w.few_blocks == 2) launch(answer_few_kernel<T, 2, 256>, 256);
            else launch(answer_few_kernel<T, 4, 256>, 256);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int P, int CHUNKS>
hipError_t tile_answers(const SoftmaxCall& x, const AnswerWs& w, hipStream_t st)
{
    PackJobs jobs{};
    const bool direct = P == 1 && usable_as_it_lies(x);
    auto job = [&](PackArgs& a, const void* in, int64_t stride, int64_t rows, int64_t padded_rows, const int32_t* ids, uint16_t* const* out, int which) {
        a.in = in; a.in_stride = stride; a.rows = rows; a.padded_rows = padded_rows; a.targets = ids;
        a.num_targets = static_cast<uint32_t>(x.num_rows); a.dim = x.dim; a.padded = w.padded;
        a.out[0] = out[0]; a.out[1] = out[1]; a.shift = w.shift + which;
        if (P == 2) { a.amax = w.amax + which * kAmaxBlocks; a.maxima = kAmaxBlocks; }
    };
    job(jobs.job[0], x.h, x.h_stride, x.n, w.tokens, x.targets, w.h, 1);
    job(jobs.job[1], x.w, x.w_stride, x.num_rows, x.num_rows, nullptr, w.w, 0);
    const NormArgs norms{x.w, x.h, x.w_stride, x.h_stride, x.n, x.num_rows, x.targets, x.dim, w.norms, P == 2 ? w.amax : nullptr};
    const uint32_t blocks = pack_blocks(w, std::max(w.tokens, x.num_rows), kThreads, kMostPack);
    if (P == 2) {
        hipLaunchKernelGGL(norms_kernel, dim3(kAmaxBlocks), dim3(kThreads), 0, st, norms);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(pack_kernel<2>, dim3(blocks, 2), dim3(kThreads), 0, st, jobs);
    } else {
        if (direct) hipLaunchKernelGGL(prepare_kernel<true>, dim3(blocks, 2), dim3(kThreads), 0, st, jobs, norms);
        else hipLaunchKernelGGL(prepare_kernel<false>, dim3(blocks, 2), dim3(kThreads), 0, st, jobs, norms);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    TileArgs a{};
    a.w = packed_operand(w.w, x.num_rows, w.padded);
    if (direct) a.w = Operand{{static_cast<const uint16_t*>(x.w), nullptr}, x.w_stride, static_cast<uint32_t>(x.num_rows - 1), static_cast<uint32_t>(x.dim)};
    a.h = packed_operand(w.h, w.tokens, w.padded);
    a.shift = w.shift; a.n = x.n; a.num_rows = static_cast<uint32_t>(x.num_rows); a.row_tiles = w.row_tiles; a.splits = w.splits;
    a.tokens = static_cast<uint32_t>(w.tokens); a.steps = w.padded / step_of<P>(); a.stat = w.stat; a.best = w.best; a.chunks = w.chunks;
    a.group = w.group; a.groups = w.groups; a.group_tiles = w.group_tiles; a.late = w.late; a.norms = w.norms; a.norm_count = P == 2 ? kAmaxBlocks : blocks; a.norm = w.norm;
    const dim3 grid(static_cast<unsigned>(ceil_div(w.tokens, w.large_scores ? 256 : 128) * w.splits));
    const int held = held_stages(w, w.row_tiles, w.splits, a.steps);
    if (P == 1 && w.large_scores) hipLaunchKernelGGL((answer_tiles_kernel<1, 8, 0, CHUNKS>), grid, dim3(512), 0, st, a);
    else if (held == 0) hipLaunchKernelGGL((answer_tiles_kernel<P, 4, 0, CHUNKS>), grid, dim3(256), 0, st, a);
    else if (held == 2) hipLaunchKernelGGL((answer_tiles_kernel<P, 4, 2, CHUNKS>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((answer_tiles_kernel<P, 4, 4, CHUNKS>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

bool answer_sizes_ok(int64_t n, int64_t num_rows, int32_t dim, int32_t type, int32_t k)
{
    return n >= 0 && n <= (1 << 24) && num_rows > 0 && num_rows < (1ll << 31) && dim >= 1 && dim <= NE_OP_MAX_DIM && type_ok(type) && k >= 0 && k <= NE_TOP_MAX;
}

}  // namespace

extern "C" {

size_t ne_logprob_workspace_bytes(int64_t n, int64_t num_rows, int32_t dim, int32_t type, int32_t k, int32_t grad)
{
    if (!answer_sizes_ok(n, num_rows, dim, type, k) || n == 0) return 0;
    return grad ? logprob_grad_bytes(n, num_rows, dim, type) : answer_need(n, num_rows, dim, type, k);
}

ne_status ne_logprob(const void* h_dev, int64_t h_stride, const void* w_dev, int64_t w_stride, int32_t type, const int32_t* ids_dev, int64_t n,
                     int64_t num_rows, int32_t dim, int32_t k, float* logp_dev, float* lse_dev, float* entropy_dev, int32_t* top_ids_dev,
                     float* top_logp_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    if (!answer_sizes_ok(n, num_rows, dim, type, k)) return fail(NE_ERR_ARG, "ne_logprob: n, num_rows, dim, type or k out of range");
    if (h_stride < dim || w_stride < dim) return fail(NE_ERR_ARG, "ne_logprob: a row stride is smaller than dim");
    if (!w_dev || !aligned(w_dev, type_bytes(type))) return fail(NE_ERR_ARG, "ne_logprob: w_dev is NULL or misaligned");
    if (n == 0) return NE_OK;
    if (!h_dev || !aligned(h_dev, type_bytes(type))) return fail(NE_ERR_ARG, "ne_logprob: h_dev is NULL or misaligned");
    if (!aligned(ids_dev, 4)) return fail(NE_ERR_ARG, "ne_logprob: ids_dev is not 4-byte aligned");
    if (!lse_dev || !aligned(lse_dev, 4)) return fail(NE_ERR_ARG, "ne_logprob: lse_dev is NULL or misaligned");
    if (logp_dev && !ids_dev) return fail(NE_ERR_ARG, "ne_logprob: log probabilities need ids");
    if (!aligned(logp_dev, 4) || !aligned(entropy_dev, 4)) return fail(NE_ERR_ARG, "ne_logprob: logp_dev or entropy_dev is misaligned");
    if (k > 0 && (!top_ids_dev || !top_logp_dev || !aligned(top_ids_dev, 4) || !aligned(top_logp_dev, 4)))
        return fail(NE_ERR_ARG, "ne_logprob: top_ids_dev or top_logp_dev is NULL or misaligned");
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < answer_need(n, num_rows, dim, type, k))
        return fail(NE_ERR_ARG, "ne_logprob: workspace_dev is NULL, not 256-byte aligned, or smaller than ne_logprob_workspace_bytes()");
    const AnswerWs w = answer_layout(n, num_rows, dim, type, k, static_cast<char*>(workspace_dev));
    const SoftmaxCall x{h_dev, w_dev, h_stride, w_stride, n, num_rows, dim, type, ids_dev, nullptr};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool f32 = type == NE_F32;
    hipError_t e;
    if (w.few_blocks) e = f32 ? few_answers<float>(x, w, st) : few_answers<bf16_t>(x, w, st);
    else if (w.kind == kWide) e = f32 ? tile_answers<2, kWide>(x, w, st) : tile_answers<1, kWide>(x, w, st);
    else if (w.kind == kNarrow) e = f32 ? tile_answers<2, kNarrow>(x, w, st) : tile_answers<1, kNarrow>(x, w, st);
    else e = f32 ? tile_answers<2, kNone>(x, w, st) : tile_answers<1, kNone>(x, w, st);
    if (e == hipSuccess) {
        const FinishArgs f{h_dev, w_dev, h_stride, w_stride, ids_dev, n, static_cast<uint32_t>(num_rows), w.splits, w.few_blocks ? w.splits : 1,
                           static_cast<uint32_t>(k), dim, w.kind, w.stat, w.few_blocks ? w.norms : w.norm, f32 && !w.few_blocks ? w.shift : nullptr, w.best,
                           w.chunks, w.group, w.groups, w.group_tiles, w.per_split, w.row_tiles, w.large_scores ? 256u : 128u, w.late, logp_dev, lse_dev, entropy_dev,
                           top_ids_dev, top_logp_dev};
        auto launch = [&](auto kernel, int64_t groups, int threads) { hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(groups)), dim3(threads), 0, st, f); };
        if (n <= kTeamsOfMany && w.chunks <= kChunksOfFour) f32 ? launch(answers_kernel<float, 4>, n, 256) : launch(answers_kernel<bf16_t, 4>, n, 256);
        else if (n <= kTeamsOfMany) f32 ? launch(answers_kernel<float, 16>, n, 1024) : launch(answers_kernel<bf16_t, 16>, n, 1024);
        else f32 ? launch(answers_kernel<float, 1>, ceil_div(n, 4), kThreads) : launch(answers_kernel<bf16_t, 1>, ceil_div(n, 4), kThreads);
        e = hipGetLastError();
        if (e == hipSuccess && w.late) {
            f32 ? launch(late_answers_kernel<float>, std::min<int64_t>(n, kLateGroups), 1024) : launch(late_answers_kernel<bf16_t>, std::min<int64_t>(n, kLateGroups), 1024);
            e = hipGetLastError();
        }
    }
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("log probability launch: ") + hipGetErrorString(e));
    return NE_OK;
}

}  // extern "C"
