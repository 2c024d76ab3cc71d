// Answers from a whole table: log probabilities of given ids, entropies, and the best ids of every row (ne_logprob).
//
//     S = H . W^T [n x V],   lse_i = log sum_v exp S_iv,   logp_i = S_i,id - lse_i
//     entropy_i = - sum_v p_iv log p_iv = log sum_v e^x_iv - sum_v p_iv x_iv,   x_iv = S_iv - max S_i  (nothing large is subtracted)
//     top: the k ids of largest S_iv in falling order, of equal scores the lowest id first
//
// Scores are never kept.  One pass over them leaves, beside the maximum and the two sums of every row's softmax, one record of 8 bytes for every
// chunk of table rows (64 with tiles, 16 where the table streams) and row of H: the chunk's best score with its place in the low bits, and
// its second best.  A score is off by at most `off_by` from what 64 bits would give.  So, with t the k-th largest of the chunks' best, the answers are among
// the chunks' best of at least t - 2 off_by and, where a chunk's second best reaches that, too (4 chunks in 100 rows at k = 16 of 200 003), its
// other rows.  A workgroup for every row of H finds these in the records, takes their scores again with sums in 64 bits, and orders them: what
// it answers does not depend on how the table was cut into tiles, and equal rows tie exactly.
#include "ne_tiles.h"

namespace {

constexpr int kTileChunk = 6, kFewChunk = 4;           // log2 of a chunk's rows
constexpr int kMostFound = 2048;                       // candidates that a workgroup looks at together
constexpr float kNoScore = -1e30f;                     // below all scores: they are bounded by kMostScore
constexpr float kMostScore = 1e29f;

// A row's softmax so far: maximum and, relative to it, the sums of e^x and x e^x (all in powers of two).
struct Softmax {
    float top, sum, moment, unused;
};

__device__ __forceinline__ void join(Softmax& a, float top, float sum, float moment)
{
    const float now = fmaxf(a.top, top), da = a.top - now, db = top - now, ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
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

template <class T>
__device__ __forceinline__ void norms_of(const NormArgs& a, uint32_t block, uint32_t blocks, uint32_t* lds)
{
    float total = 0.0f, largest = 0.0f;
    uint32_t most = 0;
    int at = 0;
    for_eights(static_cast<const T*>(a.w), a.w_stride, a.num_rows, a.dim, a.dim, block, blocks, [&](int64_t, int e, const T (&x)[8]) {
        if (e != at) {
            total += __uint_as_float(most);
            most = 0;
            at = e;
        }
        float squares = 0.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float y = static_cast<float>(x[q]);
            squares = fmaf(y, y, squares);
            if (sizeof(T) == 4) largest = fmaxf(largest, finite_abs(y));
        }
        if (magnitude_bits(x) && squares < 0x1p-126f) squares = 0x1p-126f;      // (squares of small values may be 0)
        most = max(most, __float_as_uint(squares) & 0x7FFFFFFFu);
    });
    total += __uint_as_float(most);
    int lanes = 1;
    while (lanes < 64 && 8 * lanes < a.dim) lanes *= 2;
    for (int o = 1; o < lanes; o <<= 1) total += __shfl_xor(total, o, 64);
    const uint32_t all = block_max_bits(__float_as_uint(total) & 0x7FFFFFFFu, lds);
    if (threadIdx.x == 0) a.norms[block] = all;
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

__global__ void __launch_bounds__(kThreads) norms_kernel(NormArgs a)
{
    __shared__ uint32_t lds[kThreads / 64];
    norms_of<float>(a, blockIdx.x, gridDim.x, lds);
}

// bf16: rows of H into stages and the table's norms in one launch, and the table's rows where they cannot be used as they lie.
__global__ void __launch_bounds__(kThreads) prepare_kernel(PackJobs jobs, NormArgs a)
{
    __shared__ uint32_t lds[kThreads / 64];
    if (blockIdx.y == 0) norms_of<bf16_t>(a, blockIdx.x, gridDim.x, lds);
    else pack_rows<1, kThreads>(jobs.job[blockIdx.y - 1], blockIdx.x, gridDim.x, reinterpret_cast<float*>(lds));
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
};

template <int P, int W, int KS, bool TOP>
__global__ void __launch_bounds__(64 * W, 2) answer_tiles_kernel(TileArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * stage_bytes<W>()];
    constexpr int R = rows_of<W>(), MT = W / 2;
    const int lane = threadIdx.x & 63, m0 = first_row<W>(), n0 = first_col<W>();
    uint32_t token_tile, split;
    pair_of(by_xcd(blockIdx.x, gridDim.x), (a.tokens + R - 1) / R, a.splits, token_tile, split);
    const uint32_t per = (a.row_tiles + a.splits - 1) / a.splits, tile0 = split * per;
    const float factor = score_factor<P>(a.shift), to_log2 = kLog2e * factor;
    Softmax s[2] = {{kNoScore, 0.0f, 0.0f, 0.0f}, {kNoScore, 0.0f, 0.0f, 0.0f}};
    const float low = fmaxf(-3e38f, kNoScore / factor);          // (in units of the sums; below all of them)
    all_scores<P, W, KS>(a.w, a.h, token_tile, 0, tile0, min(tile0 + per, a.row_tiles), a.steps, lds, [&](uint32_t tile_row0, f32x16 (&acc)[MT][2]) {
        const uint32_t row0 = tile_row0 + m0;
        if (row0 + 32 * MT > a.num_rows) {
            const int left = static_cast<int>(a.num_rows - (row0 + lane_row()));     // (the difference is small where both are not)
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * im + sum_row(i) >= left) acc[im][0][i] = acc[im][1][i] = low;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float t = low;
            if constexpr (TOP) {
                const int64_t token = static_cast<int64_t>(token_tile) * R + n0 + 32 * j + (lane & 31);
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
                    const uint32_t chunk = (row0 >> kTileChunk) + c;
                    if (lane < 32 && token < a.n && chunk < a.chunks) a.best[token * a.chunks + chunk] = make_float2(b.first * factor, b.second * factor);
                }
            } else {
#pragma unroll
                for (int im = 0; im < MT; ++im)
#pragma unroll
                    for (int i = 0; i < 16; ++i) t = fmaxf(t, acc[im][j][i]);
            }
            const float now = fmaxf(s[j].top, t * to_log2), d = s[j].top - now, e = __builtin_amdgcn_exp2f(d);
            float sum = 0.0f, moment = 0.0f;
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = fmaf(acc[im][j][i], to_log2, -now), p = __builtin_amdgcn_exp2f(x);
                    sum += p;
                    moment = fmaf(p, x, moment);
                }
            s[j].moment = fmaf(fmaf(s[j].sum, d, s[j].moment), e, moment);
            s[j].sum = fmaf(s[j].sum, e, sum);
            s[j].top = now;
        }
    });
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
// blocks of 16 rows; fp32 operands are split into three bf16 parts.
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
            const float now = fmaxf(s[b].top, best.first * kLog2e), d = s[b].top - now, e = __builtin_amdgcn_exp2f(d);
            float sum = 0.0f, moment = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = fmaf(acc[i], kLog2e, -now), p = __builtin_amdgcn_exp2f(x);
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
    uint32_t num_rows, splits, norm_count, k;
    int32_t dim;
    const Softmax* stat;           // [n][splits]
    const uint32_t* norms;
    const int32_t* shift;          // NULL, or powers of two of W and H
    const float2* best;            // [n][chunks]
    int64_t chunks;
    float *logp, *lse, *entropy;   // logp, entropy: NULL where not wanted
    int32_t* top_ids;
    float* top_logp;
};

// What a workgroup holds of a row: candidates and, in front of them, the best so far.
struct Found {
    uint32_t ids[64 + kMostFound];
    double scores[64 + kMostFound];
    uint32_t count;
};

// Scores of found.ids[first ..], 16 lanes each, with products and sums in 64 bits, in an order that depends on dim alone.
template <class T>
__device__ __forceinline__ void exact_scores(const FinishArgs& a, const float* h, const uint32_t* ids, double* scores, uint32_t first, uint32_t count)
{
    const int lane = threadIdx.x & 15;
    constexpr int FLIGHT = 2;
    for (uint32_t c = first + (threadIdx.x >> 4) * FLIGHT; c < count; c += kThreads / 16 * FLIGHT) {
        double sum[FLIGHT] = {};
        const T* row[FLIGHT];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) row[f] = static_cast<const T*>(a.w) + static_cast<int64_t>(ids[min(c + f, count - 1)]) * a.w_stride;
        for (int e = lane * 8; e < a.dim; e += 128) {
            T x[FLIGHT][8];
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) load_eight(row[f], e, a.dim, x[f]);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const double y = e + q < a.dim ? static_cast<double>(h[e + q]) : 0.0;
#pragma unroll
                for (int f = 0; f < FLIGHT; ++f) sum[f] = fma(static_cast<double>(static_cast<float>(x[f][q])), y, sum[f]);
            }
        }
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) sum[f] += __shfl_xor(sum[f], o, 16);
            if (lane == 0 && c + f < count) scores[c + f] = sum[f];
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) answers_kernel(FinishArgs a, int chunk_log2)
{
    extern __shared__ __align__(16) float row_lds[];      // [dim]  the row of H
    __shared__ Found found;
    __shared__ Softmax stats[kThreads / 64];
    __shared__ double norms[kThreads / 64];
    __shared__ uint32_t bits[kThreads / 64];
    __shared__ __align__(16) float maxima[kThreads];
    __shared__ uint32_t next_ids[64], total;
    __shared__ double next_scores[64];
    __shared__ float threshold;
    const int64_t i = blockIdx.x;
    const uint32_t id = a.ids ? static_cast<uint32_t>(a.ids[i]) : 0xFFFFFFFFu, k = a.k;
    int32_t* top_ids = a.top_ids + i * k;
    float* top_logp = a.top_logp + i * k;
    if (a.ids && id >= a.num_rows) {
        if (threadIdx.x == 0) {
            a.lse[i] = 0.0f;
            if (a.logp) a.logp[i] = 0.0f;
            if (a.entropy) a.entropy[i] = 0.0f;
        }
        if (threadIdx.x < k) {
            top_ids[threadIdx.x] = -1;
            top_logp[threadIdx.x] = -INFINITY;
        }
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the row, its softmax and norm, and the table's largest norm
    double norm = 0.0;
    const T* h = static_cast<const T*>(a.h) + i * a.h_stride;
    for (int e = threadIdx.x; e < a.dim; e += kThreads) {
        const float x = static_cast<float>(h[e]);
        row_lds[e] = x;
        norm = fma(static_cast<double>(x), static_cast<double>(x), norm);
    }
    Softmax s{kNoScore, 0.0f, 0.0f, 0.0f};
    for (uint32_t p = threadIdx.x; p < a.splits; p += kThreads) {
        const Softmax q = a.stat[i * a.splits + p];
        join(s, q.top, q.sum, q.moment);
    }
    uint32_t largest = 0;
    for (uint32_t p = threadIdx.x; p < a.norm_count; p += kThreads) largest = max(largest, a.norms[p]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        join_lanes(s, o);
        norm += __shfl_xor(norm, o, 64);
    }
    if (lane == 0) {
        stats[wave] = s;
        norms[wave] = norm;
    }
    double w_norm = sqrt(static_cast<double>(__uint_as_float(block_max_bits(largest, bits))));
    if (w_norm > 0.0) w_norm += 0x1p-62 * sqrt(static_cast<double>(a.dim));        // (what squares of small values left out)
    s = stats[0];
    norm = norms[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) {
        join(s, stats[w].top, stats[w].sum, stats[w].moment);
        norm += norms[w];
    }
    const double product = sqrt(norm) * w_norm, lse = (static_cast<double>(s.top) + log2(static_cast<double>(s.sum))) * 0.693147180559945309;
    const bool bad = !(product < kMostScore);       // a value that is not finite, or scores that fp32 may not hold
    if (threadIdx.x == 0) {
        a.lse[i] = bad ? NAN : static_cast<float>(lse);
        if (a.entropy) a.entropy[i] = bad ? NAN : (log2f(s.sum) - s.moment / s.sum) * kLn2;
        if (bad && a.logp) a.logp[i] = NAN;
    }
    if (bad) {
        if (threadIdx.x < k) {
            top_ids[threadIdx.x] = -1;
            top_logp[threadIdx.x] = NAN;
        }
        return;
    }
    if (a.logp) {
        if (threadIdx.x == 0) next_ids[0] = id;
        __syncthreads();
        exact_scores<T>(a, row_lds, next_ids, next_scores, 0, 1);
        if (threadIdx.x == 0) a.logp[i] = static_cast<float>(next_scores[0] - lse);
    }
    if (k == 0) return;
    if (product == 0.0) {           // all scores are 0: the lowest ids
        if (threadIdx.x < k) {
            const bool is = threadIdx.x < a.num_rows;
            top_ids[threadIdx.x] = is ? static_cast<int32_t>(threadIdx.x) : -1;
            top_logp[threadIdx.x] = is ? static_cast<float>(-lse) : -INFINITY;
        }
        return;
    }
    // How far a score of the pass may be off: rounded products and sums (a chain of dim / 16 of them), and what halves of the rows leave out.
    float off_by = static_cast<float>((a.dim / 16 + 8) * 0x1p-23 * product);
    if (sizeof(T) == 4) off_by += static_cast<float>(0x1p-20 * product);
    if (a.shift) off_by += static_cast<float>(0x1p-36 * sqrt(static_cast<double>(a.dim)) * w_norm * (sqrt(norm) + ldexp(1.0, 14 - a.shift[1])));
    off_by = 2.0f * off_by + 1e-36f * a.dim;
    // t: the k-th largest of the threads' best, below the k-th largest of all
    const float2* best = a.best + i * a.chunks;
    float mine = kNoScore;
    for (int64_t c = threadIdx.x; c < a.chunks; c += kThreads) mine = fmaxf(mine, best[c].x);
    maxima[threadIdx.x] = mine;
    if (threadIdx.x == 0) {
        threshold = kNoScore;
        total = 0;
        found.count = 64;
    }
    __syncthreads();
    if (a.chunks >= k) {
        uint32_t rank = 0;
#pragma unroll 8
        for (uint32_t o = 0; o < kThreads; o += 4) {
            const float4 m = *reinterpret_cast<const float4*>(maxima + o);
            rank += (m.x > mine || (m.x == mine && o < threadIdx.x)) + (m.y > mine || (m.y == mine && o + 1 < threadIdx.x)) +
                    (m.z > mine || (m.z == mine && o + 2 < threadIdx.x)) + (m.w > mine || (m.w == mine && o + 3 < threadIdx.x));
        }
        if (rank == k - 1) threshold = mine;
    }
    __syncthreads();
    float t = threshold;
    if (t > kNoScore) t -= 2.0f * off_by + fabsf(t) * 0x1p-15f;
    // how many rows reach it
    uint32_t rows = 0;
    for (int64_t c = threadIdx.x; c < a.chunks; c += kThreads) {
        const float2 b = best[c];
        if (b.x >= t) rows += b.y >= t ? 1u << chunk_log2 : 1u;
    }
    atomicAdd(&total, rows);
    __syncthreads();
    // All of them together where there is room, otherwise so many chunks at a time that there is.
    const int64_t at_a_time = total <= kMostFound ? a.chunks : kMostFound >> chunk_log2;
    uint32_t have = 0;              // the best so far lie in front of the candidates: found.ids[64 - have ..]
    for (int64_t c0 = 0; c0 < a.chunks; c0 += at_a_time) {
        const int64_t c1 = min(c0 + at_a_time, a.chunks);
        for (int64_t c = c0 + threadIdx.x; c < c1; c += kThreads) {
            const float2 b = best[c];
            if (!(b.x >= t)) continue;
            const uint32_t row = static_cast<uint32_t>(c) << chunk_log2;
            if (b.y >= t) {
                const uint32_t some = min(1u << chunk_log2, a.num_rows - row), to = atomicAdd(&found.count, some);
                for (uint32_t r = 0; r < some; ++r) found.ids[to + r] = row + r;
            } else {
                found.ids[atomicAdd(&found.count, 1u)] = row + (__float_as_uint(b.x) & ((1u << chunk_log2) - 1));
            }
        }
        __syncthreads();
        const uint32_t count = found.count;
        exact_scores<T>(a, row_lds, found.ids, found.scores, 64, count);
        __syncthreads();
        const uint32_t all = have + count - 64, base = 64 - have;
        for (uint32_t c = threadIdx.x; c < all; c += kThreads) {
            const uint32_t my_id = found.ids[base + c];
            const double my_score = found.scores[base + c];
            uint32_t rank = 0;
            for (uint32_t o = 0; o < all; ++o) {
                const double other = found.scores[base + o];
                rank += other > my_score || (other == my_score && found.ids[base + o] < my_id);
            }
            if (rank < k) {
                next_ids[rank] = my_id;
                next_scores[rank] = my_score;
            }
        }
        __syncthreads();
        have = min(all, k);
        if (threadIdx.x < have) {
            found.ids[64 - have + threadIdx.x] = next_ids[threadIdx.x];
            found.scores[64 - have + threadIdx.x] = next_scores[threadIdx.x];
        }
        if (threadIdx.x == 0) found.count = 64;
        __syncthreads();
        if (have == k) {
            const float last = static_cast<float>(found.scores[63]);
            t = fmaxf(t, last - off_by - fabsf(last) * 0x1p-15f);
        }
    }
    if (threadIdx.x < k) {
        const bool is = threadIdx.x < have;
        top_ids[threadIdx.x] = is ? static_cast<int32_t>(found.ids[64 - have + threadIdx.x]) : -1;
        top_logp[threadIdx.x] = is ? static_cast<float>(found.scores[64 - have + threadIdx.x] - lse) : -INFINITY;
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct AnswerWs : Packs {
    uint32_t row_tiles, splits;
    int32_t few_blocks;
    int64_t chunks;
    uint32_t* norms;
    Softmax* stat;
    float2* best;
    size_t total;
};

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
    w.chunks = ceil_div(num_rows, 1 << (w.few_blocks ? kFewChunk : kTileChunk));
    Carver take{base};
    w.norms = take.get<uint32_t>(kMostPack);
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
    if (k) bytes += std::max(ceil_div(num_rows, 1 << kFewChunk) * few, ceil_div(num_rows, 1 << kTileChunk) * n) * 8;
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

template <int P, bool TOP>
hipError_t tile_answers(const SoftmaxCall& x, const AnswerWs& w, uint32_t* norm_count, hipStream_t st)
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
        *norm_count = kAmaxBlocks;
        hipLaunchKernelGGL(norms_kernel, dim3(kAmaxBlocks), dim3(kThreads), 0, st, norms);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(pack_kernel<2>, dim3(blocks, 2), dim3(kThreads), 0, st, jobs);
    } else {
        *norm_count = blocks;
        hipLaunchKernelGGL(prepare_kernel, dim3(blocks, direct ? 2 : 3), dim3(kThreads), 0, st, jobs, norms);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    TileArgs a{};
    a.w = packed_operand(w.w, x.num_rows, w.padded);
    if (direct) a.w = Operand{{static_cast<const uint16_t*>(x.w), nullptr}, x.w_stride, static_cast<uint32_t>(x.num_rows - 1), static_cast<uint32_t>(x.dim)};
    a.h = packed_operand(w.h, w.tokens, w.padded);
    a.shift = w.shift; a.n = x.n; a.num_rows = static_cast<uint32_t>(x.num_rows); a.row_tiles = w.row_tiles; a.splits = w.splits;
    a.tokens = static_cast<uint32_t>(w.tokens); a.steps = w.padded / step_of<P>(); a.stat = w.stat; a.best = w.best; a.chunks = w.chunks;
    const dim3 grid(static_cast<unsigned>(ceil_div(w.tokens, w.large_scores ? 256 : 128) * w.splits));
    const int held = held_stages(w, w.row_tiles, w.splits, a.steps);
    if (P == 1 && w.large_scores) hipLaunchKernelGGL((answer_tiles_kernel<1, 8, 0, TOP>), grid, dim3(512), 0, st, a);
    else if (held == 0) hipLaunchKernelGGL((answer_tiles_kernel<P, 4, 0, TOP>), grid, dim3(256), 0, st, a);
    else if (held == 2) hipLaunchKernelGGL((answer_tiles_kernel<P, 4, 2, TOP>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((answer_tiles_kernel<P, 4, 4, TOP>), grid, dim3(256), 0, st, a);
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
    uint32_t norm_count = w.splits;
    hipError_t e;
    if (w.few_blocks) e = type == NE_F32 ? few_answers<float>(x, w, st) : few_answers<bf16_t>(x, w, st);
    else if (k) e = type == NE_F32 ? tile_answers<2, true>(x, w, &norm_count, st) : tile_answers<1, true>(x, w, &norm_count, st);
    else e = type == NE_F32 ? tile_answers<2, false>(x, w, &norm_count, st) : tile_answers<1, false>(x, w, &norm_count, st);
    if (e == hipSuccess) {
        const FinishArgs f{h_dev, w_dev, h_stride, w_stride, ids_dev, static_cast<uint32_t>(num_rows), w.splits, norm_count, static_cast<uint32_t>(k), dim,
                           w.stat, w.norms, type == NE_F32 && !w.few_blocks ? w.shift : nullptr, w.best, w.chunks, logp_dev, lse_dev, entropy_dev,
                           top_ids_dev, top_logp_dev};
        const size_t lds = static_cast<size_t>(dim) * 4;
        const int chunk_log2 = w.few_blocks ? kFewChunk : kTileChunk;
        if (type == NE_F32) hipLaunchKernelGGL(answers_kernel<float>, dim3(static_cast<unsigned>(n)), dim3(kThreads), lds, st, f, chunk_log2);
        else hipLaunchKernelGGL(answers_kernel<bf16_t>, dim3(static_cast<unsigned>(n)), dim3(kThreads), lds, st, f, chunk_log2);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("log probability launch: ") + hipGetErrorString(e));
    return NE_OK;
}

}  // extern "C"
