// Softmax cross entropy against a whole table, without keeping the scores: ne_xent_loss, ne_xent_grad.
//
//     S = H . W^T [n x V],   lse_i = log sum_v exp S_iv,   loss_i = lse_i - S_i,target
//     G_iv = exp(S_iv - lse_i) - [v = target_i],   dH_i = scale c_i (G . W)_i,   dW = scale G^T . (c H)
// (c_i is in the rows of H for dW and applied in fp32 to the sums of dH, scale to the sums of both)
//
// Everything is a matrix product with something small around it, so the same loads to LDS, operand reads and matrix
// instructions serve all three products; they differ in where their operands lie and in what becomes of the sums:
//   scores   every lane of a tile's sums belongs to one row of H (table rows run along the registers), so the running
//            maximum and sum of a row's softmax are two registers, joined between lanes once at the end.
//   gradient the same product again for a piece of the table, whose G is written to the workspace (of sizes that
//            fill the machine, and in the 256 MB of last-level cache where that matters), then dH += G . W_piece and dW_piece = G^T . H in one launch.
// The scores are computed twice (8 n V d operations in training, where 6 would do with all scores kept: n V of them,
// 6.6 GB in fp32 at the sizes below, written once and read twice).
// With few rows of H all of it is bound by reading the table and writing its gradient, and other kernels let the table stream through
// registers once (few_rows_kernel, few_grad_kernel).
//
// Types: bf16 operands go to the matrix cores as they are.  G of bf16 tables is held in fp16, which keeps 11 bits where bf16 keeps 8.  dW
// multiplies it with H in fp16.  dH, for which the table would have to be turned into fp16, rounds it to bf16 in registers, but takes the
// target's coefficient whole.  So both gradients' errors are those of their own rounding: 0.0017.  (With G in bf16 0.0021, and dH 0.013 where the
// table's rows share a part ten times as large as what tells them apart: a row's coefficients add up to nothing, their roundings do not.)  Where entropies count the
// target's coefficient is not the only large one, and dH takes all of them with 11 bits (its error is 0.0017 to 0.0021 there).
// fp32 operands are split into two fp16 halves at a common power of two, x 2^k = hi + lo with 22 bits (of elements down to 2^-16 of the
// largest; smaller ones are off by up to 2^-38 of it, fp16 ending there), and a product is hi hi + hi lo + lo hi: about the error of an fp32
// product at three matrix instructions, 408 TF as a large library product runs (1225 TF in bf16), where one in fp32 makes 154.
//
// Bound by the matrix cores and by the loads from L2 that feed them.  Measured, 8192 rows, 200 003 of 512, bf16: loss
// 1.7 to 1.8 ms (950 TF; a copy of the kernel without loads took 0.87 of the time, without exponentials 0.90, without
// products 0.87: none of them hides the others completely), gradients of a piece of 15 616 table rows 167 us for G and
// 255 for both products (1.03 PF), 6.9 to 7.2 ms in all.
// 4096 rows, 10 000 of 128, fp32: scores 40 us, G 55, products 72, and 35 us for the small launches around them.
#include "ne_tiles.h"

namespace {

constexpr int kFewGradGroups = 1024;       // workgroups of the gradients; half as many where one takes more registers and LDS
// Bytes of G of one piece: at most, those from which on smaller pieces are not looked at, those that stay in the last-level cache beside the
// table and the sums, and what is written or read of these in a stage's time.
constexpr int64_t kGBytes = 512 << 20, kGLeast = 64 << 20, kGCached = 256 << 20, kStageBytes = 8 << 20;
// In stages: the fewest of a product's workgroup; what a tile takes besides (1, 4 and 8 choose alike); what a launch takes.
constexpr int kLeastShare = 8, kTileCost = 1, kLaunchCost = 10;
constexpr int kGShift = 14;            // fp16 halves of G are those of G 2^14
constexpr int64_t kHalfTable = 512;    // rows of H from which on a bf16 table becomes fp16 for dH where entropies count

// ---------------------------------------------------------------------------------------------
// scores: the softmax's maximum and sum of every row of H, and its target's score
// ---------------------------------------------------------------------------------------------
struct ScoreArgs {
    Operand w, h;                  // both by rows
    const int32_t* targets;
    const int32_t* shift;          // fp32 only: powers of two of W and H
    int64_t n;
    uint32_t num_rows, row_tiles, splits, tokens;   // tokens: padded n
    int32_t steps;                 // stages of a tile
    float2* stat;                  // [tokens][splits]  maximum and sum, in powers of two
    float* target_score;           // [tokens]
};

template <int P, int W, int KS>
__global__ void __launch_bounds__(64 * W, 2) scores_kernel(ScoreArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * stage_bytes<W>()];
    constexpr int R = rows_of<W>(), MT = W / 2;
    const int lane = threadIdx.x & 63, m0 = first_row<W>(), n0 = first_col<W>();
    uint32_t token_tile, split;
    pair_of(by_xcd(blockIdx.x, gridDim.x), (a.tokens + R - 1) / R, a.splits, token_tile, split);
    const uint32_t per = (a.row_tiles + a.splits - 1) / a.splits, tile0 = split * per;
    const float factor = score_factor<P>(a.shift), to_log2 = kLog2e * factor;
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
    uint32_t target[2];
    int64_t token[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        token[j] = static_cast<int64_t>(token_tile) * R + n0 + 32 * j + (lane & 31);
        target[j] = token[j] < a.n ? static_cast<uint32_t>(a.targets[token[j]]) : 0xFFFFFFFFu;
        if (target[j] >= a.num_rows) target[j] = 0xFFFFFFFFu;
    }
    all_scores<P, W, KS>(a.w, a.h, token_tile, 0, tile0, min(tile0 + per, a.row_tiles), a.steps, lds, [&](uint32_t tile_row0, f32x16 (&acc)[MT][2]) {
        const uint32_t row0 = tile_row0 + m0, lane_row0 = row0 + lane_row();
        if (row0 + 32 * MT > a.num_rows) {
            const int left = static_cast<int>(a.num_rows - lane_row0);     // (the difference is small where both are not)
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * im + sum_row(i) >= left) acc[im][0][i] = acc[im][1][i] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (__any(target[j] - row0 < 32 * MT)) {
#pragma unroll
                for (int im = 0; im < MT; ++im)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (target[j] - lane_row0 == 32 * im + sum_row(i)) a.target_score[token[j]] = acc[im][j][i] * factor;
            }
            float t = acc[0][j][0];
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i) t = fmaxf(t, acc[im][j][i]);
            const float now = fmaxf(top[j], t * to_log2);
            const float by = now == -INFINITY ? 0.0f : now;         // (nothing seen yet but scores of minus infinity)
            float part = 0.0f;
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i) part += __builtin_amdgcn_exp2f(fmaf(acc[im][j][i], to_log2, -by));
            sum[j] = fmaf(sum[j], __builtin_amdgcn_exp2f(top[j] - by), part);
            top[j] = now;
        }
    });
    // lanes l and l + 32 and the two wavefronts of a column have the same rows of H
    float2* join = reinterpret_cast<float2*>(lds);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        join_stat(top[j], sum[j], make_float2(__shfl_xor(top[j], 32, 64), __shfl_xor(sum[j], 32, 64)));
        if (lane < 32) join[(m0 ? R : 0) + n0 + 32 * j + lane] = make_float2(top[j], sum[j]);
    }
    __syncthreads();
    const uint32_t row = token_tile * R + threadIdx.x;
    if (threadIdx.x < R && row < a.tokens) {
        float2 p = join[threadIdx.x];
        join_stat(p.x, p.y, join[R + threadIdx.x]);
        a.stat[static_cast<int64_t>(row) * a.splits + split] = p;
    }
}

// Joins the splits of the table: lse and loss of every row, a wavefront each.
__global__ void __launch_bounds__(kThreads) loss_join_kernel(const float2* stat, const float* target_score, const int32_t* targets, int64_t n,
                                                             uint32_t num_rows, uint32_t splits, float* loss, float* lse)
{
    const int lane = threadIdx.x & 63;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
    if (i >= n) return;
    if (static_cast<uint32_t>(targets[i]) >= num_rows) {
        if (lane == 0) loss[i] = lse[i] = 0.0f;
        return;
    }
    float top = -INFINITY, sum = 0.0f;
#pragma unroll 4
    for (uint32_t s = lane; s < splits; s += 64) join_stat(top, sum, stat[i * splits + s]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) join_stat(top, sum, make_float2(__shfl_xor(top, o, 64), __shfl_xor(sum, o, 64)));
    if (lane == 0) {
        const float z = (top + log2f(sum)) * kLn2;
        lse[i] = z;
        loss[i] = z - target_score[i];
    }
}

// ---------------------------------------------------------------------------------------------
// few rows of H: the table streams through registers once, straight from memory
// ---------------------------------------------------------------------------------------------
// Bound by reading the table (one row against 200 003 of 256 bf16: 19.5 us, 5.2 TB/s; 23.6 with the launch that joins the workgroups'
// shares).  A wavefront has 16 table rows at a time, whose elements go from memory to the matrix cores' first
// operand as they lie (lane l: row l % 16, eight elements from (l / 16) * 8 on of every 32); H lies in LDS as second operands, in blocks
// of 16 rows.  fp32 operands are split into three bf16 parts (24 bits, no common scale to be found first: that would read the
// table twice), of whose nine products the six largest are taken.  Up to 32 rows the largest of them is added up apart from the others, and in two or
// four sums of every second or fourth step, which are joined at the end: fewer roundings, and of smaller numbers (losses of 16 rows of 1011 fp32 columns:
// off by 0.5e-6 root mean square, 2.2e-6 in one sum, where torch's fp32 product leads to 0.8e-6; times within 2 %.  64 rows: 1.7e-6 and torch's 3.0e-6,
// and sums apart cost 4 %).
struct FewArgs {
    const void *h, *w;
    int64_t h_stride, w_stride;
    const int32_t* targets;
    uint32_t n, num_rows;
    int32_t dim, steps;            // steps of 32 elements
    float2* stat;                  // [n][workgroups]
    float* target_score;
};

template <class T, int BLOCKS, int THREADS>
__global__ void __launch_bounds__(THREADS) few_rows_kernel(FewArgs a)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, AHEAD = sizeof(T) == 4 ? 4 : 8, CHAINS = BLOCKS == 1 ? 4 : BLOCKS == 2 ? 2 : 1;
    constexpr bool APART = PARTS > 1 && BLOCKS < 4;
    extern __shared__ __align__(16) unsigned char few_lds[];       // [blocks][steps][parts][64 lanes] 16 bytes
    bf16x8* hs = reinterpret_cast<bf16x8*>(few_lds);
    __shared__ float2 join[THREADS / 64][BLOCKS * 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    for (int i = wave; i < BLOCKS * a.steps; i += THREADS / 64) {
        const int block = i / a.steps, step = i % a.steps;
        const uint32_t t = block * 16 + col;
        T x[8];
        if (t < a.n && static_cast<uint32_t>(a.targets[t]) < a.num_rows) {
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
    float top[BLOCKS], sum[BLOCKS];
    uint32_t target[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        top[b] = -INFINITY;
        sum[b] = 0.0f;
        target[b] = b * 16 + col < a.n ? static_cast<uint32_t>(a.targets[b * 16 + col]) : 0xFFFFFFFFu;
    }
    __syncthreads();
    const uint32_t tiles = (a.num_rows + 15) / 16, stride = gridDim.x * (THREADS / 64);
    for (uint32_t tile = blockIdx.x * (THREADS / 64) + wave; tile < tiles; tile += stride) {
        const T* row = static_cast<const T*>(a.w) + static_cast<int64_t>(min(tile * 16 + col, a.num_rows - 1)) * a.w_stride;
        f32x4 sums[BLOCKS][CHAINS], small[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            small[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < CHAINS; ++c) sums[b][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        for (int s0 = 0; s0 < a.steps; s0 += AHEAD) {
            T x[AHEAD][8];
#pragma unroll
            for (int s = 0; s < AHEAD; ++s)
                if (s0 + s < a.steps) load_eight(row, (s0 + s) * 32 + quarter * 8, a.dim, x[s]);
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                if (s0 + s >= a.steps) break;
                bf16x8 w[PARTS];
                split_bf16<PARTS>(x[s], w);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    bf16x8 h[PARTS];
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) h[p] = hs[((b * a.steps + s0 + s) * PARTS + p) * 64 + lane];
                    // (the smallest products first)
#pragma unroll
                    for (int sum_of_parts = PARTS - 1; sum_of_parts >= 0; --sum_of_parts) {
                        f32x4& to = APART && sum_of_parts > 0 ? small[b] : sums[b][s % CHAINS];
#pragma unroll
                        for (int p = 0; p <= sum_of_parts; ++p) to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[p], h[sum_of_parts - p], to, 0, 0, 0);
                    }
                }
            }
        }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            f32x4& acc = sums[b][0];
#pragma unroll
            for (int c = 1; c < CHAINS; ++c) acc += sums[b][c];
            if (APART) acc += small[b];
            float now = top[b];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t r = tile * 16 + quarter * 4 + i;
                if (r == target[b] && r < a.num_rows) a.target_score[b * 16 + col] = acc[i];
                if (r >= a.num_rows) acc[i] = -INFINITY;
                now = fmaxf(now, acc[i] * kLog2e);
            }
            const float by = now == -INFINITY ? 0.0f : now;
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) part += __builtin_amdgcn_exp2f(fmaf(acc[i], kLog2e, -by));
            sum[b] = fmaf(sum[b], __builtin_amdgcn_exp2f(top[b] - by), part);
            top[b] = now;
        }
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) join_stat(top[b], sum[b], make_float2(__shfl_xor(top[b], o, 64), __shfl_xor(sum[b], o, 64)));
        if (lane < 16) join[wave][b * 16 + lane] = make_float2(top[b], sum[b]);
    }
    __syncthreads();
    if (threadIdx.x < a.n) {
        float2 p = join[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) join_stat(p.x, p.y, join[w][threadIdx.x]);
        a.stat[static_cast<int64_t>(threadIdx.x) * gridDim.x + blockIdx.x] = p;
    }
}

// ---------------------------------------------------------------------------------------------
// a bf16 table as fp16
// ---------------------------------------------------------------------------------------------
// Where entropies count, several of a row's coefficients are large and they add up to nothing, so where the table's rows share a part it is the roundings of
// all of them that is left of it in dH: with G in bf16 dH is off by 0.011 where that part is ten times what tells rows apart, with G's 11 bits by 0.002 (its own rounding
// 0.0017).  So dH's product takes G, in fp16, as the sum of two bf16 numbers; or, of kHalfTable rows of H and more, a bf16 table becomes fp16, too, piece by piece, where
// it was packed or would have been.  That costs passes over the table, which many rows share, instead of a fourth more matrix instructions (us of the
// gradients, G rounded to bf16, as two, table in fp16: 64 rows of 200 003 x 512 180, 191, 306; 300 rows 365, 429, 493; 600 rows 558, 661, 666; 1500 rows 1171, 1464,
// 1278; 400 of 199 999 x 300 447, 513, 494; 800 of 100 000 x 128 131, 141, 148).
// bf16 to fp16, times a power of two: exponents less `bias` (how much smaller fp16's are, for the largest to have fp16's largest), which lies in the places
// of both formats' exponents.  Elements keep all of their 8 bits from 2^-29 of the largest on; smaller ones are off by less than 2^-30 of it.
__device__ __forceinline__ s16x8 to_half(s16x8 x, uint16_t bias)
{
    typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
    const u16x8 u = __builtin_bit_cast(u16x8, x), sign = u & static_cast<uint16_t>(0x8000);
    return __builtin_bit_cast(s16x8, (__builtin_elementwise_sub_sat(u ^ sign, u16x8(bias)) << static_cast<uint16_t>(3)) | sign);
}

// That bias for a largest magnitude, and the power of two that it makes.
__device__ __forceinline__ int half_bias(float largest) { return max(static_cast<int>(__float_as_uint(largest) >> 23) - 30, 0); }
__device__ __forceinline__ int half_shift(int bias) { return 112 - bias; }

struct TableArgs {
    const void* in;
    uint16_t* out;                 // (may be in)
    int64_t in_stride, out_stride, rows;
    int32_t width;                 // a multiple of 8
    const int32_t* shift;
};

// Bound by memory (8192 rows of H against 200 003 x 512: 13 launches of 7.2 us, and 42 us for the table's largest magnitude, which packing finds; as G need not be turned in
// registers the gradients take 80 us more in all, of 7430. Turning the table there, in the place of G, took 2200: a large tile has twice as many operands of it.)
__global__ void __launch_bounds__(kThreads) table_kernel(TableArgs a)
{
    const uint16_t bias = static_cast<uint16_t>((half_shift(0) - *a.shift) << 7);
    for_eights(static_cast<const bf16_t*>(a.in), a.in_stride, a.rows, a.width, a.width, blockIdx.x, gridDim.x, [&](int64_t r, int e, const bf16_t (&x)[8]) {
        s16x8 y;
        __builtin_memcpy(&y, x, 16);
        *reinterpret_cast<s16x8*>(a.out + r * a.out_stride + e) = to_half(y, bias);
    });
}

// ---------------------------------------------------------------------------------------------
// G of a piece of the table
// ---------------------------------------------------------------------------------------------
// The scores again, with the exponentials written as operands of the next products instead of added up: of bf16 tables G 2^14 in fp16, off by 2^-12 of
// itself from 2^-28 on and by 2^-39 below; of fp32 ones two fp16 halves of it, which keep 22 bits of 2^-16 and more (and 2^-39 of less).  By far
// the largest coefficient of most rows is the target's: what dH's product does not see of it in bf16 is kept, and given to dH with the target's row of the
// table when its sums are rounded.
// 8192 x 15 616 x 512 bf16: 167 us (0.78 PF, 256 MB written); 4096 x 10 000 x 128 fp32: 55 us (164 MB written).
// A row's coefficients where its entropy counts: p (a + b x) 2^14 - target at the target, for p 2^14 = 2^x.
struct Mix {
    float a, b, target, unused;
};

struct CoefArgs {
    Operand w, h;                  // both by rows
    const int32_t* targets;
    const int32_t* shift;
    const float* lse;
    int64_t n, g_stride;
    uint32_t num_rows, row_base, row_tiles, splits, tokens;
    int32_t steps;
    uint16_t* g[2];                // [tokens][g_stride], table rows of the piece side by side
    uint32_t blocks;               // workgroups that make G; bf16: further ones of the first piece bring c H into fp16 (1000 x 3000 x 64: 37 us with a
                                   // launch of its own, 32 so)
    PackArgs hc;
    float* rest;                   // bf16 only: [tokens]  what rounding takes from the target's coefficient: to bf16, or where entropies count to fp16
    const Mix* mix;                // with entropies only: [n]
    const float* table_max;        // NULL, or `maxima` largest magnitudes of the table, ...
    int32_t maxima;
    int32_t* table_shift;          // ... which leave the power of two behind that it takes as fp16
};

// ENTROPY: one multiply-add and one product more a score, beside the exponential (4096 rows against 10 000 x 128 fp32: 61 us, 8192 against 200 003 x 512 bf16:
// 13 pieces of 181).
template <int P, int W, int KS, bool ENTROPY>
__global__ void __launch_bounds__(64 * W, 2) coef_kernel(CoefArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * stage_bytes<W>()];
    constexpr int R = rows_of<W>(), MT = W / 2;
    if (P == 1 && blockIdx.x >= a.blocks) {
        pack_rows<1, 64 * W>(a.hc, blockIdx.x - a.blocks, gridDim.x - a.blocks, reinterpret_cast<float*>(lds));
        return;
    }
    if (ENTROPY && P == 1 && a.table_max && blockIdx.x == 0) {
        float top = 0.0f;
        for (int i = threadIdx.x; i < a.maxima; i += 64 * W) top = fmaxf(top, a.table_max[i]);
        top = block_max<64 * W>(top, reinterpret_cast<float*>(lds));
        if (threadIdx.x == 0) *a.table_shift = half_shift(half_bias(top));
        __syncthreads();
    }
    const int lane = threadIdx.x & 63, m0 = first_row<W>(), n0 = first_col<W>();
    uint32_t token_tile, split;
    pair_of(by_xcd(blockIdx.x, a.blocks), (a.tokens + R - 1) / R, a.splits, token_tile, split);
    const uint32_t per = (a.row_tiles + a.splits - 1) / a.splits, tile0 = split * per;
    const float to_log2 = kLog2e * score_factor<P>(a.shift);
    uint32_t target[2];
    float by[2];
    Mix mix[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t token = static_cast<int64_t>(token_tile) * R + n0 + 32 * j + (lane & 31);
        const bool all = ENTROPY && !a.targets;      // (rows that have no ids all count)
        target[j] = token < a.n && !all ? static_cast<uint32_t>(a.targets[token]) : 0xFFFFFFFFu;
        if (target[j] >= a.num_rows) target[j] = 0xFFFFFFFFu;
        const bool counts = all ? token < a.n : target[j] != 0xFFFFFFFFu;
        // (G 2^14; a row without a target: 2 to the minus infinity)
        by[j] = counts ? fmaf(a.lse[token], kLog2e, -static_cast<float>(kGShift)) : INFINITY;
        mix[j] = ENTROPY && counts ? a.mix[token] : Mix{0.0f, 0.0f, 0x1p14f, 0.0f};
    }
    all_scores<P, W, KS>(a.w, a.h, token_tile, a.row_base, tile0, min(tile0 + per, a.row_tiles), a.steps, lds, [&](uint32_t tile_row0, f32x16 (&acc)[MT][2]) {
        const uint32_t row0 = tile_row0 + m0, lane_row0 = row0 + lane_row();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (token_tile * R + n0 + 32 * j >= a.tokens) continue;     // (tokens: a multiple of 32)
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x = fmaf(acc[im][j][i], to_log2, -by[j]);
                    if (ENTROPY) x = x < -1000.0f ? -1000.0f : x;       // (0 times infinity is no coefficient)
                    acc[im][j][i] = __builtin_amdgcn_exp2f(x);
                    if (ENTROPY) acc[im][j][i] *= fmaf(mix[j].b, x, mix[j].a);
                }
            if (__any(target[j] - row0 < 32 * MT)) {
#pragma unroll
                for (int im = 0; im < MT; ++im)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (target[j] - lane_row0 == 32 * im + sum_row(i)) {
                            acc[im][j][i] -= ENTROPY ? mix[j].target : 0x1p14f;
                            if (P == 1) {
                                const float g = acc[im][j][i];
                                const float stored = static_cast<float>(static_cast<f16_t>(g));
                                a.rest[token_tile * R + n0 + 32 * j + (lane & 31)] = g - (ENTROPY ? stored : static_cast<float>(static_cast<bf16_t>(stored)));
                            }
                        }
            }
            if (row0 + 32 * MT > a.num_rows) {
                const int left = static_cast<int>(a.num_rows - lane_row0);     // (the difference is small where both are not)
#pragma unroll
                for (int im = 0; im < MT; ++im)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (32 * im + sum_row(i) >= left) acc[im][j][i] = 0.0f;
            }
            const int64_t to = (static_cast<int64_t>(token_tile) * R + n0 + 32 * j + (lane & 31)) * a.g_stride + (row0 - a.row_base) + 8 * (lane >> 5);
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int q = 0; q < 4; q += 2) {
                    u32x2 hi[2], lo[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const f32x4 x = {acc[im][j][4 * (q + r)], acc[im][j][4 * (q + r) + 1], acc[im][j][4 * (q + r) + 2], acc[im][j][4 * (q + r) + 3]};
                        const f16x4 xh = __builtin_convertvector(x, f16x4);
                        hi[r] = __builtin_bit_cast(u32x2, xh);
                        if constexpr (P == 2) lo[r] = __builtin_bit_cast(u32x2, __builtin_convertvector(x - __builtin_convertvector(xh, f32x4), f16x4));
                    }
                    *reinterpret_cast<u32x4*>(a.g[0] + to + 32 * im + 8 * q) = eight_of(hi[0], hi[1]);
                    if constexpr (P == 2) *reinterpret_cast<u32x4*>(a.g[1] + to + 32 * im + 8 * q) = eight_of(lo[0], lo[1]);
                }
        }
    });
}

// ---------------------------------------------------------------------------------------------
// dH += G . W_piece and dW_piece = G^T . H
// ---------------------------------------------------------------------------------------------
struct ProductArgs {
    Operand g_rows, w;             // dH: G by rows (contraction along them), W across
    Operand g_cols, h;             // dW: G across, H across
    float* dh;                     // [h_splits][tokens][cols]  sums over the pieces
    float* dw;                     // [w_splits][piece rows][cols], or NULL: one split, whose sums are dW
    void* out;                     // dW of the piece
    int64_t out_stride;
    uint32_t tokens, piece_rows, cols;      // multiples of 32 or 64, of 256, of 32
    uint32_t h_tiles, w_tiles, col_tiles;   // tiles over tokens, piece rows, columns
    uint32_t h_splits, w_splits, h_share, w_share;      // splits of the contraction, stages of each
    uint32_t h_stages, w_stages;
    int32_t add;                   // dh: added to what earlier pieces left
    uint32_t rows;                 // table rows of the piece that there are
    int32_t dim;
    float scale;
    const int32_t* shift;          // power of two of the rows of H
};

// Both products of a piece are one launch: either alone leaves places empty.  (8192 x 15 616 x 512 bf16, large tiles: 255 us, 1.03 PF; 4096 x 10 000 x
// 128 fp32, small tiles: 72 us, 0.87 PF of half products.)
// (The gradients' columns are the first operand, so that they run along a lane's registers and are written side by side.)
// (bf16: turning G from fp16 to bf16 in registers takes up to 4 % of the gradients' time, 8192 x 200 003 x 512 5180 -> 5370 us; W in fp16 would
// take a pass over the table.)
// DH: how dH's product takes G and the table.
template <int P, int W, Kind DH>
__global__ void __launch_bounds__(64 * W, 2) products_kernel(ProductArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * stage_bytes<W>()];
    const int lane = threadIdx.x & 63;
    const uint32_t h_blocks = a.h_tiles * a.col_tiles * a.h_splits;
    // (dH's workgroups first, then dW's: a CU that has two has one of either, which differ in how long they take)
    uint32_t b = blockIdx.x;
    const bool dh = b < h_blocks;
    if (!dh) b -= h_blocks;
    const uint32_t splits = dh ? a.h_splits : a.w_splits, share = dh ? a.h_share : a.w_share, stages = dh ? a.h_stages : a.w_stages;
    const uint32_t col = b % a.col_tiles, split = b / a.col_tiles % splits, tile = b / a.col_tiles / splits;
    const uint32_t s0 = min(split * share, stages), s1 = min(s0 + share, stages);
    constexpr int R = rows_of<W>(), MT = W / 2;
    f32x16 acc[MT][2];
    if (dh) product_tile<P, W, true, DH>(a.w, a.g_rows, col * R, tile * R, s0, s1, lds, acc);
    else product_tile<P, W, false, P == 1 ? kHalf : kPlain>(a.h, a.g_cols, col * R, tile * R, s0, s1, lds, acc);
    const uint32_t row0 = tile * R + first_col<W>() + (lane & 31), col0 = col * R + first_row<W>() + 4 * (lane >> 5);
    if (!dh && !a.dw) {
        const int k = -(*a.shift + kGShift);
        typedef typename std::conditional<P == 2, float, bf16_t>::type T;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (row0 + 32 * j >= a.rows) continue;
            T* to = static_cast<T*>(a.out) + static_cast<int64_t>(row0 + 32 * j) * a.out_stride + col0;
#pragma unroll
            for (int im = 0; im < MT; ++im)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = ldexpf(acc[im][j][4 * q + e], k) * a.scale;
                    store_some<T, 4>(to + 32 * im + 8 * q, a.dim - static_cast<int>(col0 + 32 * im + 8 * q), x);
                }
        }
        return;
    }
    float* out = dh ? a.dh + static_cast<int64_t>(split) * a.tokens * a.cols : a.dw + static_cast<int64_t>(split) * a.piece_rows * a.cols;
    const bool add = dh && a.add;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (row0 + 32 * j >= (dh ? a.tokens : a.piece_rows)) continue;
        float* to = out + static_cast<int64_t>(row0 + 32 * j) * a.cols + col0;
#pragma unroll
        for (int im = 0; im < MT; ++im)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (col0 + 32 * im + 8 * q >= a.cols) continue;
                float4 x = make_float4(acc[im][j][4 * q], acc[im][j][4 * q + 1], acc[im][j][4 * q + 2], acc[im][j][4 * q + 3]);
                float4* at = reinterpret_cast<float4*>(to + 32 * im + 8 * q);
                if (add) {
                    const float4 old = *at;
                    x = make_float4(old.x + x.x, old.y + x.y, old.z + x.z, old.w + x.w);
                }
                *at = x;
            }
    }
}

// Sums the splits and rounds once (2 x 8192 x 512, 42 MB: 8 us, 11 with the targets' rows).  dH: rows without a target become zeros, the others
// take their factor, and in bf16 what the target's coefficient lost.
struct ReduceArgs {
    const float* in;               // [splits][rows_in][cols]
    int64_t split_stride;
    uint32_t splits, cols;
    int64_t rows;
    int32_t dim;
    void* out;
    int64_t out_stride;
    const int32_t* targets;        // dH only
    uint32_t num_targets;
    const float* c;
    float scale;
    const int32_t* shift;          // NULL, or power of two of the other operand
    const float* rest;             // dH in bf16 only: what the targets' coefficients lost, ...
    const bf16_t* w;               // ... and the table, whose rows of the targets take it
    int64_t w_stride;
};

// A workgroup has 256 columns of a row; where there are many splits its wavefronts share them, and their sums are added in order.
template <class T>
__global__ void __launch_bounds__(kThreads) reduce_kernel(ReduceArgs a)
{
    __shared__ float4 lds[kThreads];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t parts = a.splits >= 16 ? 4 : 1;           // wavefronts of a row
    const int64_t r = static_cast<int64_t>(blockIdx.x) * (4 / parts) + (parts == 4 ? 0 : wave);
    const int e = blockIdx.y * 256 + lane * 4;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const bool in = r < a.rows && e < static_cast<int>(a.cols);
    bool counts = in;
    float c = 1.0f, rest = 0.0f, x[4] = {};
    if (in && (a.targets || a.c)) {      // (fetched ahead of the sums)
        const uint32_t target = a.targets ? static_cast<uint32_t>(a.targets[r]) : 0;
        counts = !a.targets || target < a.num_targets;
        if (counts && a.c) c = a.c[r];
        if (counts && a.rest) {
            rest = a.rest[r];
            const bf16_t* w = a.w + target * a.w_stride + e;
            if (e + 4 <= a.dim) {
                load_vec<bf16_t, 4>(w, x);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = e + q < a.dim ? static_cast<float>(w[q]) : 0.0f;
            }
        }
    }
    if (in) {
        const float* from = a.in + r * a.cols + e;
        const uint32_t step = parts;
        uint32_t s = parts == 4 ? wave : 0;
        for (; s + 7 * step < a.splits; s += 8 * step) {
            float4 x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = *reinterpret_cast<const float4*>(from + (s + q * step) * a.split_stride);
#pragma unroll
            for (int q = 0; q < 8; ++q) sum = make_float4(sum.x + x[q].x, sum.y + x[q].y, sum.z + x[q].z, sum.w + x[q].w);
        }
        for (; s < a.splits; s += step) {
            const float4 x = *reinterpret_cast<const float4*>(from + s * a.split_stride);
            sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
        }
    }
    if (parts == 4) {
        lds[threadIdx.x] = sum;
        __syncthreads();
        if (wave != 0) return;
        for (int w = 1; w < 4; ++w) {
            const float4 x = lds[w * 64 + lane];
            sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
        }
    }
    if (!in) return;
    const int k = -((a.shift ? *a.shift : 0) + kGShift);
    const float all[4] = {sum.x, sum.y, sum.z, sum.w};
    auto whole = [&](float sum, float w) {
        if (a.rest && a.shift) return fmaf(ldexpf(rest, -kGShift), w, ldexpf(sum, k));      // (the table's power of two is not the coefficient's)
        return ldexpf(a.rest ? fmaf(rest, w, sum) : sum, k);
    };
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = counts ? whole(all[q], x[q]) * a.scale * c : 0.0f;
    store_some<T, 4>(static_cast<T*>(a.out) + r * a.out_stride + e, a.dim - e, x);
}

// ---------------------------------------------------------------------------------------------
// few rows of H: both gradients in one pass over the table
// ---------------------------------------------------------------------------------------------
// Bound by reading the table and writing its gradient.  A workgroup has 16 table rows at a time, of which a wavefront has CT groups of 16
// columns: its share of the scores goes to the others through LDS, then every wavefront has all coefficients and makes dW of its columns, which
// leaves at once, and adds to dH of its columns, which stays in registers to the end.  All products are fp32 matrix
// instructions: with few rows of H they take less time than the table does, and no operand has to be split or scaled, so nothing reads the table
// twice (200 003 x 256 fp32, 410 MB read and written: one row 92 us, 4.4 TB/s; 16 rows 102; in bf16 81, by then bound by the tile's chain of
// LDS exchanges and products).
// Contraction indices are taken in the order in which a lane has them side by side: 16 indices in four instructions, instruction i with index
// 4 q + i in quarter q of the wavefront.
struct FewGradArgs {
    const void *h, *w;
    int64_t h_stride, w_stride;
    const int32_t* targets;
    const float *lse, *c;          // c: NULL, or factors of the rows
    uint32_t n, num_rows, cols;
    int32_t dim;
    float scale;
    float* dh;                     // NULL, or [workgroups][n][cols]
    void* dw;                      // NULL, or the table's gradient
    int64_t dw_stride;
    const Mix* mix;                // with entropies only: [n]
};

template <int CT, int WAVES> constexpr int few_stride() { return WAVES * CT * 16 + 4; }        // of a row of H in LDS: quarters in different banks
template <int BLOCKS, int CT, int WAVES> constexpr size_t few_grad_lds() { return size_t{16} * BLOCKS * few_stride<CT, WAVES>() * 4; }

template <class T, int BLOCKS, int CT, int WAVES, bool ENTROPY>
__global__ void __launch_bounds__(64 * WAVES) few_grad_kernel(FewGradArgs a)
{
    constexpr int STRIDE = few_stride<CT, WAVES>();
    extern __shared__ __align__(16) float few_h[];      // [16 BLOCKS][STRIDE]
    __shared__ __align__(16) float part[2][WAVES][BLOCKS][256], turn[WAVES][BLOCKS][256];      // [row of H][row of the table]
    __shared__ __align__(16) float crossing[WAVES][2][16][20];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    for (int i = threadIdx.x; i < 16 * BLOCKS * STRIDE; i += 64 * WAVES) {
        const uint32_t t = i / STRIDE;
        const int e = i % STRIDE;
        const bool in = t < a.n && e < a.dim && ((ENTROPY && !a.targets) || static_cast<uint32_t>(a.targets[t]) < a.num_rows);
        few_h[i] = in ? static_cast<float>(static_cast<const T*>(a.h)[t * a.h_stride + e]) : 0.0f;
    }
    uint32_t target[BLOCKS];
    float by[BLOCKS], c[BLOCKS];
    Mix mix[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        const uint32_t t = b * 16 + col;
        const bool all = ENTROPY && !a.targets;
        target[b] = t < a.n && !all ? static_cast<uint32_t>(a.targets[t]) : 0xFFFFFFFFu;
        const bool counts = all ? t < a.n : target[b] < a.num_rows;     // (otherwise 2 to the minus infinity)
        by[b] = counts ? a.lse[t] * kLog2e : INFINITY;
        c[b] = counts && a.c ? a.c[t] : 1.0f;
        mix[b] = Mix{};
        if (ENTROPY && counts) {
            mix[b] = a.mix[t];
            mix[b].a = fmaf(mix[b].b, static_cast<float>(kGShift), mix[b].a);      // (p = 2^x here)
            mix[b].target *= 0x1p-14f;
        }
    }
    f32x4 dh[BLOCKS][CT];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int g = 0; g < CT; ++g) dh[b][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t tiles = (a.num_rows + 15) / 16, last = a.num_rows - 1;
    const int first_col = wave * CT * 16;
    const T* w = static_cast<const T*>(a.w);
    // row `col` of a tile, columns 4 quarter .. + 3 of each group: zeros beyond the last column
    auto load = [&](uint32_t tile, float (&x)[CT][4]) {
        const T* row = w + min(tile * 16 + col, last) * a.w_stride;
#pragma unroll
        for (int g = 0; g < CT; ++g) {
            const int e = first_col + g * 16 + quarter * 4;
            if (e + 4 <= a.dim) {
                load_vec<T, 4>(row + e, x[g]);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) x[g][q] = e + q < a.dim ? static_cast<float>(row[e + q]) : 0.0f;
            }
        }
    };
    float x[CT][4];
    load(blockIdx.x, x);
    __syncthreads();
    uint32_t turns = 0;
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x, turns ^= 1) {
        float next[CT][4];
        if (tile + gridDim.x < tiles) load(tile + gridDim.x, next);
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int g = 0; g < CT; ++g) {
                const f32x4 h = *reinterpret_cast<const f32x4*>(few_h + (b * 16 + col) * STRIDE + first_col + g * 16 + quarter * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[g][i], h[i], s, 0, 0, 0);
            }
            *reinterpret_cast<f32x4*>(&part[turns][wave][b][col * 16 + quarter * 4]) = s;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // (loads travel on; the other half of `part` is for the next tile)
        // coefficients of row `col` of H and rows 4 quarter .. + 3 of the table
        f32x4 coef[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            f32x4 s = *reinterpret_cast<const f32x4*>(&part[turns][0][b][col * 16 + quarter * 4]);
#pragma unroll
            for (int v = 1; v < WAVES; ++v) s += *reinterpret_cast<const f32x4*>(&part[turns][v][b][col * 16 + quarter * 4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t row = tile * 16 + quarter * 4 + i;
                float x = fmaf(s[i], kLog2e, -by[b]);
                if (ENTROPY) x = x < -1000.0f ? -1000.0f : x;
                float p = __builtin_amdgcn_exp2f(x);
                if (ENTROPY) p *= fmaf(mix[b].b, x, mix[b].a);
                if (row == target[b]) p -= ENTROPY ? mix[b].target : 1.0f;
                coef[b][i] = row <= last ? p * c[b] : 0.0f;
            }
            if (a.dw) *reinterpret_cast<f32x4*>(&turn[wave][b][col * 16 + quarter * 4]) = coef[b];
        }
        if (a.dh) {     // the tile with its rows along the registers, by way of LDS
            float across[CT][4];
#pragma unroll
            for (int g = 0; g < CT; ++g) {
                float (&at)[16][20] = crossing[wave][g & 1];
                *reinterpret_cast<f32x4*>(&at[col][quarter * 4]) = f32x4{x[g][0], x[g][1], x[g][2], x[g][3]};
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int i = 0; i < 4; ++i) across[g][i] = at[quarter * 4 + i][col];
            }
#pragma unroll
            for (int g = 0; g < CT; ++g)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) dh[b][g] = __builtin_amdgcn_mfma_f32_16x16x4f32(coef[b][i], across[g][i], dh[b][g], 0, 0, 0);
        }
        if (a.dw) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            float turned[BLOCKS][4];        // of rows 4 quarter .. + 3 of H and row `col` of the table
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) turned[b][i] = turn[wave][b][(quarter * 4 + i) * 16 + col];
            T* to = static_cast<T*>(a.dw) + static_cast<int64_t>(tile * 16 + col) * a.dw_stride;
#pragma unroll
            for (int g = 0; g < CT; ++g) {
                f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sum = __builtin_amdgcn_mfma_f32_16x16x4f32(few_h[(b * 16 + quarter * 4 + i) * STRIDE + first_col + g * 16 + col], turned[b][i], sum, 0, 0, 0);
                const int e = first_col + g * 16 + quarter * 4;
                const float out[4] = {sum[0] * a.scale, sum[1] * a.scale, sum[2] * a.scale, sum[3] * a.scale};
                if (tile * 16 + col <= last) store_some<T, 4>(to + e, a.dim - e, out);
            }
        }
#pragma unroll
        for (int g = 0; g < CT; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[g][i] = next[g][i];
    }
    if (!a.dh) return;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t t = b * 16 + quarter * 4 + i;
            if (t >= a.n) continue;
            float* to = a.dh + (static_cast<int64_t>(blockIdx.x) * a.n + t) * a.cols;
#pragma unroll
            for (int g = 0; g < CT; ++g)
                if (first_col + g * 16 + col < a.dim) to[first_col + g * 16 + col] = dh[b][g][i];
        }
}

// dH from the workgroups' shares, added in their order: 64 columns of a row, 64 shares at a time.
struct FewJoinArgs {
    const float* in;               // [shares][n][cols]
    uint32_t shares, n, num_targets, cols;
    const int32_t* targets;
    int32_t dim;
    float scale;
    void* out;
    int64_t out_stride;
};

template <class T>
__global__ void __launch_bounds__(1024) few_join_kernel(FewJoinArgs a)
{
    __shared__ __align__(16) float lds[64][64];
    const uint32_t group = threadIdx.x >> 4, t = blockIdx.x;
    const int e = blockIdx.y * 64 + (threadIdx.x & 15) * 4;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (e < static_cast<int>(a.cols)) {
        const float* from = a.in + static_cast<int64_t>(t) * a.cols + e;
        const int64_t step = static_cast<int64_t>(a.n) * a.cols;
#pragma unroll 8
        for (uint32_t v = group; v < a.shares; v += 64) sum += *reinterpret_cast<const f32x4*>(from + v * step);
    }
    *reinterpret_cast<f32x4*>(&lds[group][(threadIdx.x & 15) * 4]) = sum;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    float all = 0.0f;
#pragma unroll 16
    for (int v = 0; v < 64; ++v) all += lds[v][threadIdx.x];
    const int at = blockIdx.y * 64 + threadIdx.x;
    if (at >= a.dim) return;
    const bool counts = !a.targets || static_cast<uint32_t>(a.targets[t]) < a.num_targets;
    static_cast<T*>(a.out)[t * a.out_stride + at] = from_float<T>(counts ? all * a.scale : 0.0f);
}

// Gradients of sum_i l_i logp_i + e_i entropy_i: with f = |l| + 8 |e|, a = l / f and b = e / f the coefficient of table row v is
//     - f [ p (a + b (s - lse + entropy)) - a [v = id] ],
// the bracket at most 1 in magnitude (p |log p| < 0.37, p entropy < 6 for tables of less than 2^31 rows), as that of the loss alone is.  (A launch: 3 to 5 us.)
struct MixArgs {
    const int32_t* ids;            // NULL: no log probabilities, and all rows count
    const float *logp_grad, *entropy_grad, *entropy;      // the gradients: NULL for 1; the entropies are there
    float logp_scale, entropy_scale;
    int64_t n;
    uint32_t num_rows;
    Mix* mix;                      // [n]
    float* c;                      // [n]  - f
};

__global__ void __launch_bounds__(kThreads) mix_kernel(MixArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= a.n) return;
    const bool counts = !a.ids || static_cast<uint32_t>(a.ids[i]) < a.num_rows;
    const float l = counts && a.ids ? a.logp_scale * (a.logp_grad ? a.logp_grad[i] : 1.0f) : 0.0f;
    const float e = counts ? a.entropy_scale * (a.entropy_grad ? a.entropy_grad[i] : 1.0f) : 0.0f;
    const float f = fabsf(l) + 8.0f * fabsf(e), u = f == 0.0f ? 0.0f : l / f, v = f == 0.0f ? 0.0f : e / f;
    a.mix[i] = counts ? Mix{fmaf(v, a.entropy[i] - kGShift * kLn2, u), v * kLn2, u * 0x1p14f, 0.0f} : Mix{};
    a.c[i] = -f;
}

template <class T>
__global__ void __launch_bounds__(kThreads) zero_kernel(T* out, int64_t stride, int64_t rows, int32_t dim)
{
    const int64_t total = rows * dim;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * kThreads)
        out[i / dim * stride + i % dim] = from_float<T>(0.0f);
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct XentWs : Packs {
    uint32_t row_tiles, splits;        // of the scores, or of a piece's coefficients
    int32_t few_blocks;                // > 0: few rows of H, so many blocks of 16
    int32_t few_waves, few_groups;     // of their gradients: wavefronts of a workgroup, groups of 16 columns of each
    int64_t piece;                     // table rows of a piece
    bool large_products;               // tiles of 256 x 256
    uint32_t h_splits, w_splits, w_share, w_stages;
    float2* stat;
    float* target_score;
    uint16_t* g[2];
    float *dh, *dw, *rest;
    float* table_max;                  // with entropies: largest magnitudes of a bf16 table
    size_t total;
};

bool xent_sizes_ok(int64_t n, int64_t num_rows, int32_t dim, int32_t type)
{
    return n >= 0 && n <= (1 << 24) && num_rows > 0 && num_rows < (1ll << 31) && dim >= 1 && dim <= NE_OP_MAX_DIM && type_ok(type);
}

// When a launch ends, in stages: `first` workgroups of `first_time` stages begin in order, then `second` ones, and `slots` run at once.
int64_t launch_time(int64_t first, int64_t first_time, int64_t second, int64_t second_time, int64_t slots)
{
    // the second kind finds `late` slots that are free one round of the first after the others
    const int64_t begin = first / slots * first_time, late = first % slots;
    int64_t early_rounds = std::max<int64_t>(0, second / slots - first_time / second_time - 2), late_rounds = early_rounds;
    while ((slots - late) * early_rounds + late * late_rounds < second) {
        if (begin + early_rounds * second_time <= begin + first_time + late_rounds * second_time) ++early_rounds;
        else ++late_rounds;
    }
    return std::max(begin + early_rounds * second_time, late ? begin + first_time + late_rounds * second_time : 0);
}

// Splits the contractions of a piece's two products, which are one launch of two kinds of workgroups, into shares of about the same length, as many
// as fill the machine; of these shares the one with which the launch is over first, as a workgroup too many takes a whole round more (1500 x
// 100 003 x 200 bf16: 257 workgroups 97 us a piece, 251 longer ones 66).  Returns its time in stages of small tiles.
int64_t split_products(XentWs& w, int32_t dim, bool large)
{
    const int64_t edge = large ? 256 : 128, step = w.parts == 1 ? step_of<1>() : step_of<2>();
    const int64_t cols = ceil_div(dim, edge), h_tiles = ceil_div(w.tokens, edge) * cols, w_tiles = ceil_div(w.piece, edge) * cols;
    const int64_t h_stages = w.piece / step, w_stages = w.tokens / step;
    w.large_products = large;
    w.w_stages = static_cast<uint32_t>(w_stages);
    const int64_t even = std::max<int64_t>(kLeastShare, ceil_div(h_tiles * h_stages + w_tiles * w_stages, slots_of(large)));
    int64_t best = INT64_MAX;
    for (int64_t share = even; share <= 2 * even; share += ceil_div(even, 32)) {
        const int64_t hs = ceil_div(h_stages, share), ws = ceil_div(w_stages, share);
        const int64_t time = launch_time(h_tiles * hs, ceil_div(h_stages, hs) + kTileCost, w_tiles * ws, ceil_div(w_stages, ws) + kTileCost, slots_of(large));
        if (time >= best) continue;
        best = time;
        w.h_splits = static_cast<uint32_t>(hs);
        w.w_splits = static_cast<uint32_t>(ws);
        w.w_share = static_cast<uint32_t>(ceil_div(w_stages, ws));
    }
    return large ? 2 * best : best;
}

// The pieces of the table: large ones mean few launches, some sizes fill the machine and others just miss it, and G of a small one stays in the
// last-level cache, which narrow tables need, whose products are over faster than G is read.  Of up to seventeen numbers of pieces the
// one whose launches take the least time, by their stages and by G's bytes.  (Gradients, us, and with pieces of always 128 MB: 8192 x 200 003 x
// 512 bf16 5220 and 5580, 4096 x 100 000 x 256 795 and 910, 8192 x 100 000 x 128 fp32 2595 and 3100, 1000 x 500 000 x 128 bf16 833 and 818,
// x 64 680 and 625: the estimate is not always right.  The bf16 figures, here and below, are those before G was held in fp16, which costs both sides
// up to 4 %.)
void choose_pieces(XentWs& w, int64_t n, int64_t num_rows, int32_t dim)
{
    const int64_t row_tiles = ceil_div(num_rows, 256), bytes = row_tiles * 256 * 2 * w.parts * w.tokens;
    const int64_t side = w.large_scores ? 256 : 128, steps = w.padded / (w.parts == 1 ? step_of<1>() : step_of<2>());
    const int64_t fewest = std::min<int64_t>(ceil_div(bytes, kGBytes), row_tiles);
    int64_t best = INT64_MAX;
    XentWs chosen = w;
    for (int64_t pieces = fewest; pieces <= 5 * fewest && pieces <= row_tiles && pieces * kGLeast <= bytes + kGLeast; pieces += ceil_div(fewest, 4)) {
        w.piece = ceil_div(row_tiles, pieces) * 256;
        // Large tiles of products (bf16, of more than 128 columns): where dW needs no partial sums with them, or where they have few more columns
        // than small tiles (4096 x 50 000, gradients: of 640 columns 1070 us, small tiles 1118; of 300, which become 512: 768 and 641; 6000 x 30 000
        // x 200: 386 and 440; 1024 x 50 000 x 384, no partial sums: 182 and 205).
        int64_t time = split_products(w, dim, w.parts == 1 && dim > 128 && n >= 256);
        if (w.large_products && w.w_splits > 1 && round_up(dim, 256) * 5 > round_up(dim, 128) * 6) time = split_products(w, dim, false);
        const int64_t g_tiles = ceil_div(w.piece, side), g_splits = splits_of(g_tiles, ceil_div(w.tokens, side), w.large_scores);
        const int64_t g_bytes = w.piece * 2 * w.parts * w.tokens, g_time = g_bytes / (g_bytes <= kGCached ? kStageBytes : kStageBytes / 2);
        time = std::max(time, 2 * g_time) + std::max(ceil_div(g_tiles, g_splits) * steps * (w.large_scores ? 2 : 1), g_time) + 2 * kLaunchCost;
        time *= ceil_div(num_rows, w.piece);
        if (time >= best) continue;
        best = time;
        chosen = w;
    }
    w = chosen;
}

// Whether both gradients take one pass over the table, and how.  Up to 32 rows in fp32, where the other way makes halves of the table first (us at
// 200 003 x 256: 16 rows 102 and 280, 32 rows 149 and 281), and up to 16 in bf16 where columns are few (100 000 x 100: 33 and 48; 200 003 x 256:
// 80 and 90; 100 000 x 512: 102 and 86; 17 rows of 256: 132 and 90).
bool few_grad(XentWs& w, int64_t n, int32_t dim)
{
    if (n > 32 || (w.parts == 1 && (n > 16 || dim > 256))) return false;
    const int64_t groups = ceil_div(dim, 16);
    w.few_blocks = n <= 16 ? 1 : 2;
    w.few_waves = groups <= 32 ? 4 : 8;
    w.few_groups = 1;
    while (w.few_groups * w.few_waves < groups) w.few_groups *= 2;
    if (w.few_groups <= 8 && (w.few_blocks == 1 || w.few_waves == 4)) return true;
    w.few_blocks = 0;
    return false;
}

// The workspace has room for packed copies whether or not this call's alignment needs them.
XentWs xent_layout(int64_t n, int64_t num_rows, int32_t dim, int32_t type, bool grad, char* base)
{
    XentWs w{};
    w.parts = type == NE_F32 ? 2 : 1;
    w.padded = static_cast<int32_t>(round_up(dim, w.parts == 1 ? step_of<1>() : step_of<2>()));
    w.cols = static_cast<int32_t>(round_up(dim, 32));
    const int64_t step = w.parts == 1 ? step_of<1>() : step_of<2>();
    w.tokens = round_up(n, step);
    w.large_scores = large_scores(n, num_rows, dim, w.parts);
    const int64_t side = w.large_scores ? 256 : 128, token_tiles = ceil_div(w.tokens, side);
    w.row_tiles = static_cast<uint32_t>(ceil_div(num_rows, side));
    Carver take{base};
    if (!grad && (w.few_blocks = few_blocks_of(n, num_rows, dim, w.parts)) > 0) {
        const bool alone = few_bytes_of(w.few_blocks, dim, w.parts) > kFewBytes;        // (a tile of 16 rows for each wavefront, at most)
        w.splits = static_cast<uint32_t>(std::min<int64_t>(ceil_div(num_rows, alone ? 128 : 64), alone ? 256 : kFewGroups));
        w.stat = take.get<float2>(static_cast<size_t>(w.splits) * n);
        w.target_score = take.get<float>(static_cast<size_t>(n));
        w.total = take.total();
        return w;
    }
    if (grad && few_grad(w, n, dim)) {
        const int64_t most = w.few_blocks == 1 && w.few_groups <= 4 ? kFewGradGroups : kFewGradGroups / 2;
        w.splits = static_cast<uint32_t>(std::min(ceil_div(num_rows, 16), most));
        w.dh = take.get<float>(static_cast<size_t>(w.splits) * n * w.cols);
        w.total = take.total();
        return w;
    }
    w.amax = take.get<float>(3 * kAmaxBlocks);
    w.shift = take.get<int32_t>(3);
    for (int p = 0; p < w.parts; ++p) {
        w.h[p] = take.get<uint16_t>(static_cast<size_t>(w.tokens) * w.padded);
        w.w[p] = take.get<uint16_t>(static_cast<size_t>(num_rows) * w.padded);
    }
    if (!grad) {
        w.splits = splits_of(w.row_tiles, token_tiles, w.large_scores);
        w.stat = take.get<float2>(static_cast<size_t>(w.splits) * w.tokens);
        w.target_score = take.get<float>(static_cast<size_t>(w.tokens));
    } else {
        choose_pieces(w, n, num_rows, dim);
        for (int p = 0; p < w.parts; ++p) {
            w.hc[p] = take.get<uint16_t>(static_cast<size_t>(w.tokens) * w.padded);
            w.g[p] = take.get<uint16_t>(static_cast<size_t>(w.tokens) * w.piece);
        }
        w.dh = take.get<float>(static_cast<size_t>(w.h_splits) * w.tokens * w.cols);
        w.dw = w.w_splits > 1 ? take.get<float>(static_cast<size_t>(w.w_splits) * w.piece * w.cols) : nullptr;
        w.rest = w.parts == 1 ? take.get<float>(static_cast<size_t>(w.tokens)) : nullptr;
    }
    w.total = take.total();
    return w;
}

// Bytes of a workspace for up to n rows: bounds of what xent_layout takes, each growing with n, as what it takes itself need not (few rows take no
// copies, a larger n may have smaller pieces or fewer splits).
size_t xent_bytes(int64_t n, int64_t num_rows, int32_t dim, int32_t type, bool grad)
{
    XentWs w{};
    w.parts = type == NE_F32 ? 2 : 1;
    const int64_t step = w.parts == 1 ? step_of<1>() : step_of<2>();
    const int64_t tokens = round_up(n, step), padded = round_up(dim, step), cols = round_up(dim, 32), rows = round_up(num_rows, 256);
    int64_t bytes = 16 << 10;                                   // alignment, largest magnitudes
    if (!grad) {
        // shares of few rows; of tiles: as many workgroups as run in four rounds, or one for every tile
        bytes += (std::min<int64_t>(ceil_div(num_rows, 64), kFewGroups) * std::min<int64_t>(n, 192) + tokens +
                  std::min<int64_t>(ceil_div(num_rows, 128) * tokens, 4 * 512 * 128)) * 8 + tokens * 4;
        if (few_blocks_of(n, num_rows, dim, w.parts)) return static_cast<size_t>(bytes);
    } else {
        const int64_t few = ceil_div(num_rows, 16);
        const int64_t narrow = std::min<int64_t>(few, kFewGradGroups) * std::min<int64_t>(n, 16);
        const int64_t wide = std::min<int64_t>(few, kFewGradGroups / 2) * std::min<int64_t>(n, 32);
        bytes += std::max(narrow, wide) * cols * 4;
        if (few_grad(w, n, dim)) return static_cast<size_t>(bytes);
        // G of a piece; partial sums: a share has kLeastShare stages, and all workgroups but one for each tile have a place at once
        const int64_t row_bytes = 2 * w.parts * tokens, places = int64_t{256} * 256 * 256;
        const int64_t all_h = round_up(n, 256) * round_up(dim, 256), all_w = rows * round_up(dim, 256);
        bytes += std::min(rows * row_bytes, kGBytes + 256 * row_bytes);
        bytes += std::min(ceil_div(rows / step, kLeastShare) * tokens * cols, places + all_h) * 4;
        if (tokens / step > kLeastShare) bytes += std::min(ceil_div(tokens / step, kLeastShare) * rows * cols, places + std::min(all_w, places)) * 4;
        bytes += w.parts * tokens * padded * 2 + (w.parts == 1 ? tokens * 4 : 0);
    }
    return static_cast<size_t>(bytes + w.parts * 2 * padded * (tokens + num_rows));
}

hipError_t join_losses(const SoftmaxCall& x, const XentWs& w, float* loss, float* lse, hipStream_t st)
{
    hipLaunchKernelGGL(loss_join_kernel, dim3(static_cast<unsigned>(ceil_div(x.n, kThreads / 64))), dim3(kThreads), 0, st, w.stat, w.target_score,
                       x.targets, x.n, static_cast<uint32_t>(x.num_rows), w.splits, loss, lse);
    return hipGetLastError();
}

template <class T>
hipError_t run_few(const SoftmaxCall& x, const XentWs& w, float* loss, float* lse, hipStream_t st)
{
    FewArgs a{};
    a.w = x.w; a.h_stride = x.h_stride; a.w_stride = x.w_stride; a.num_rows = static_cast<uint32_t>(x.num_rows); a.dim = x.dim;
    a.steps = static_cast<int32_t>(ceil_div(x.dim, 32));
    const size_t lds = static_cast<size_t>(few_bytes_of(w.few_blocks, x.dim, w.parts));
    auto launch = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(w.splits), dim3(threads), lds, st, a); };
    for (int64_t base = 0; base < x.n; base += 16 * w.few_blocks) {
        a.h = static_cast<const T*>(x.h) + base * x.h_stride; a.targets = x.targets + base;
        a.n = static_cast<uint32_t>(std::min<int64_t>(x.n - base, 16 * w.few_blocks));
        a.stat = w.stat + base * w.splits; a.target_score = w.target_score + base;
        if (lds > kFewBytes) {
            if (w.few_blocks == 1) launch(few_rows_kernel<T, 1, 512>, 512);
            else if (w.few_blocks == 2) launch(few_rows_kernel<T, 2, 512>, 512);
            else launch(few_rows_kernel<T, 4, 512>, 512);
        } else {
            if (w.few_blocks == 1) launch(few_rows_kernel<T, 1, 256>, 256);
            else if (w.few_blocks == 2) launch(few_rows_kernel<T, 2, 256>, 256);
            else launch(few_rows_kernel<T, 4, 256>, 256);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return join_losses(x, w, loss, lse, st);
}

template <int P>
hipError_t run_loss(const SoftmaxCall& x, const XentWs& w, float* loss, float* lse, hipStream_t st)
{
    ScoreArgs a{};
    Operand unused;
    hipError_t e = pack(x, w, false, &a.h, &unused, &a.w, nullptr, nullptr, nullptr, st);
    if (e != hipSuccess) return e;
    a.targets = x.targets; a.shift = w.shift; a.n = x.n; a.num_rows = static_cast<uint32_t>(x.num_rows); a.row_tiles = w.row_tiles;
    a.splits = w.splits; a.tokens = static_cast<uint32_t>(w.tokens); a.steps = w.padded / step_of<P>(); a.stat = w.stat; a.target_score = w.target_score;
    const dim3 grid(static_cast<unsigned>(ceil_div(w.tokens, w.large_scores ? 256 : 128) * w.splits));
    const int held = held_stages(w, w.row_tiles, w.splits, a.steps);
    if (P == 1 && w.large_scores) hipLaunchKernelGGL((scores_kernel<1, 8, 0>), grid, dim3(512), 0, st, a);
    else if (held == 0) hipLaunchKernelGGL((scores_kernel<P, 4, 0>), grid, dim3(256), 0, st, a);
    else if (held == 2) hipLaunchKernelGGL((scores_kernel<P, 4, 2>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((scores_kernel<P, 4, 4>), grid, dim3(256), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    return join_losses(x, w, loss, lse, st);
}

template <class T, int BLOCKS, bool ENTROPY = false>
hipError_t run_few_grad(const SoftmaxCall& x, const XentWs& w, const Mix* mix, const float* lse, float scale, void* dh, int64_t dh_stride, void* dw, int64_t dw_stride, hipStream_t st)
{
    FewGradArgs a{};
    a.h = x.h; a.w = x.w; a.h_stride = x.h_stride; a.w_stride = x.w_stride; a.targets = x.targets; a.lse = lse; a.c = x.c;
    a.n = static_cast<uint32_t>(x.n); a.num_rows = static_cast<uint32_t>(x.num_rows); a.cols = static_cast<uint32_t>(w.cols); a.dim = x.dim;
    a.scale = scale; a.dh = dh ? w.dh : nullptr; a.dw = dw; a.dw_stride = dw_stride; a.mix = mix;
    const dim3 grid(w.splits);
    if (w.few_groups == 1) hipLaunchKernelGGL((few_grad_kernel<T, BLOCKS, 1, 4, ENTROPY>), grid, dim3(256), (few_grad_lds<BLOCKS, 1, 4>()), st, a);
    else if (w.few_groups == 2) hipLaunchKernelGGL((few_grad_kernel<T, BLOCKS, 2, 4, ENTROPY>), grid, dim3(256), (few_grad_lds<BLOCKS, 2, 4>()), st, a);
    else if (w.few_groups == 4) hipLaunchKernelGGL((few_grad_kernel<T, BLOCKS, 4, 4, ENTROPY>), grid, dim3(256), (few_grad_lds<BLOCKS, 4, 4>()), st, a);
    if constexpr (sizeof(T) == 4) {
        if (BLOCKS == 1 && w.few_waves == 8) hipLaunchKernelGGL((few_grad_kernel<T, 1, 8, 8, ENTROPY>), grid, dim3(512), (few_grad_lds<1, 8, 8>()), st, a);
        else if (w.few_groups == 8) hipLaunchKernelGGL((few_grad_kernel<T, BLOCKS, 8, 4, ENTROPY>), grid, dim3(256), (few_grad_lds<BLOCKS, 8, 4>()), st, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dh) return e;
    FewJoinArgs j{w.dh, w.splits, a.n, a.num_rows, a.cols, x.targets, x.dim, scale, dh, dh_stride};
    hipLaunchKernelGGL(few_join_kernel<T>, dim3(a.n, static_cast<unsigned>(ceil_div(x.dim, 64))), dim3(1024), 0, st, j);
    return hipGetLastError();
}

template <int P, class T, bool ENTROPY = false>
hipError_t run_grad(const SoftmaxCall& x, const XentWs& w, const Mix* mix, const float* lse, float scale, void* dh, int64_t dh_stride, void* dw, int64_t dw_stride, hipStream_t st)
{
    CoefArgs ca{};
    ProductArgs pa{};
    const bool halves = P == 1 && ENTROPY && dh && x.n >= kHalfTable;      // dH's product takes the table as fp16
    hipError_t e = pack(x, w, dw != nullptr, &ca.h, &pa.h, &ca.w, &ca.hc, halves ? w.table_max : nullptr, &ca.maxima, st);
    if (e != hipSuccess) return e;
    const Operand all = ca.w;
    ca.targets = x.targets; ca.shift = w.shift; ca.lse = lse; ca.n = x.n; ca.g_stride = w.piece; ca.rest = w.rest; ca.mix = mix;
    ca.num_rows = static_cast<uint32_t>(x.num_rows); ca.steps = w.padded / step_of<P>();
    const int64_t side = w.large_scores ? 256 : 128, edge = w.large_products ? 256 : 128;
    const uint32_t token_tiles = static_cast<uint32_t>(ceil_div(w.tokens, side));
    pa.dh = w.dh; pa.dw = w.dw; pa.tokens = static_cast<uint32_t>(w.tokens); pa.piece_rows = static_cast<uint32_t>(w.piece);
    pa.cols = static_cast<uint32_t>(w.cols); pa.col_tiles = static_cast<uint32_t>(ceil_div(x.dim, edge));
    pa.h_splits = w.h_splits; pa.w_splits = w.w_splits; pa.w_share = w.w_share;
    pa.w_stages = w.w_stages;
    pa.out_stride = dw_stride; pa.dim = x.dim; pa.scale = scale; pa.shift = w.shift + (x.c ? 2 : 1);
    ca.table_max = halves ? w.table_max : nullptr;
    ca.table_shift = w.shift;
    auto reduce = [&](ReduceArgs r) {
        r.cols = pa.cols; r.dim = x.dim; r.scale = scale;
        const dim3 grid(static_cast<unsigned>(ceil_div(r.rows, r.splits >= 16 ? 1 : 4)), static_cast<unsigned>(ceil_div(x.dim, 256)));
        hipLaunchKernelGGL(reduce_kernel<T>, grid, dim3(kThreads), 0, st, r);
        return hipGetLastError();
    };
    for (int64_t base = 0; base < x.num_rows; base += w.piece) {
        const int64_t rows = std::min<int64_t>(w.piece, x.num_rows - base);
        ca.row_base = static_cast<uint32_t>(base);
        ca.row_tiles = static_cast<uint32_t>(ceil_div(rows, side));
        ca.splits = splits_of(ca.row_tiles, token_tiles, w.large_scores);
        ca.tokens = static_cast<uint32_t>(w.tokens);
        for (int p = 0; p < P; ++p) ca.g[p] = w.g[p];
        ca.blocks = token_tiles * ca.splits;
        const dim3 grid(ca.blocks + (P == 1 && dw && base == 0 ? pack_blocks(w, w.tokens, w.large_scores ? 512 : 256, 256) : 0));
        const int held = held_stages(w, ca.row_tiles, ca.splits, ca.steps);
        if (P == 1 && w.large_scores) hipLaunchKernelGGL((coef_kernel<1, 8, 0, ENTROPY>), grid, dim3(512), 0, st, ca);
        else if (held == 0) hipLaunchKernelGGL((coef_kernel<P, 4, 0, ENTROPY>), grid, dim3(256), 0, st, ca);
        else if (held == 2) hipLaunchKernelGGL((coef_kernel<P, 4, 2, ENTROPY>), grid, dim3(256), 0, st, ca);
        else hipLaunchKernelGGL((coef_kernel<P, 4, 4, ENTROPY>), grid, dim3(256), 0, st, ca);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        pa.g_rows = Operand{{w.g[0], w.g[1]}, w.piece, static_cast<uint32_t>(w.tokens - 1), static_cast<uint32_t>(w.piece)};
        pa.g_cols = pa.g_rows;
        pa.w = all;
        if (halves) {
            const TableArgs t{all.part[0] + base * all.stride, w.w[0] + base * w.padded, all.stride, w.padded, rows, static_cast<int32_t>(all.width), w.shift};
            hipLaunchKernelGGL(table_kernel, dim3(pack_blocks(w, rows, kThreads, kMostPack)), dim3(kThreads), 0, st, t);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            pa.w.part[0] = w.w[0];
            pa.w.stride = w.padded;
        }
        for (int p = 0; p < P; ++p) pa.w.part[p] += base * pa.w.stride;
        pa.w.last = static_cast<uint32_t>(rows - 1);
        pa.h_tiles = dh ? static_cast<uint32_t>(ceil_div(w.tokens, edge)) : 0;
        pa.w_tiles = dw ? static_cast<uint32_t>(ceil_div(rows, edge)) : 0;
        pa.h_stages = static_cast<uint32_t>(ceil_div(rows, step_of<P>()));      // (no stage begins beyond the last row)
        pa.h_share = static_cast<uint32_t>(ceil_div(pa.h_stages, w.h_splits));
        pa.add = base > 0;
        pa.rows = static_cast<uint32_t>(rows);
        pa.out = dw ? static_cast<T*>(dw) + base * dw_stride : nullptr;
        const uint32_t blocks = (pa.h_tiles * pa.h_splits + pa.w_tiles * pa.w_splits) * pa.col_tiles;
        if (!blocks) continue;
        constexpr Kind DH = P == 2 ? kPlain : ENTROPY ? kToTwoBf16 : kToBf16, DH_HALVES = P == 1 && ENTROPY ? kHalf : DH;
        if (P == 1 && w.large_products && halves) hipLaunchKernelGGL((products_kernel<1, 8, ENTROPY ? kHalf : kToBf16>), dim3(blocks), dim3(512), 0, st, pa);
        else if (P == 1 && w.large_products) hipLaunchKernelGGL((products_kernel<1, 8, ENTROPY ? kToTwoBf16 : kToBf16>), dim3(blocks), dim3(512), 0, st, pa);
        else if (halves) hipLaunchKernelGGL((products_kernel<P, 4, DH_HALVES>), dim3(blocks), dim3(256), 0, st, pa);
        else hipLaunchKernelGGL((products_kernel<P, 4, DH>), dim3(blocks), dim3(256), 0, st, pa);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (dw && w.dw) {
            ReduceArgs r{};
            r.in = w.dw; r.split_stride = w.piece * pa.cols; r.splits = w.w_splits; r.rows = rows;
            r.out = static_cast<T*>(dw) + base * dw_stride; r.out_stride = dw_stride;
            r.shift = w.shift + (x.c ? 2 : 1);
            e = reduce(r);
            if (e != hipSuccess) return e;
        }
    }
    if (dh) {
        ReduceArgs r{};
        r.in = w.dh; r.split_stride = w.tokens * pa.cols; r.splits = w.h_splits; r.rows = x.n; r.out = dh; r.out_stride = dh_stride;
        r.targets = x.targets; r.num_targets = ca.num_rows; r.c = x.c; r.shift = P == 2 || halves ? w.shift : nullptr;
        r.rest = x.targets ? w.rest : nullptr; r.w = static_cast<const bf16_t*>(x.w); r.w_stride = x.w_stride;
        return reduce(r);
    }
    return hipSuccess;
}

ne_status check_xent(const SoftmaxCall& x, const char* who)
{
    const std::string name(who);
    if (!xent_sizes_ok(x.n, x.num_rows, x.dim, x.type)) return fail(NE_ERR_ARG, name + ": n, num_rows, dim or type out of range");
    if (x.h_stride < x.dim || x.w_stride < x.dim) return fail(NE_ERR_ARG, name + ": a row stride is smaller than dim");
    if (!x.w || !aligned(x.w, type_bytes(x.type))) return fail(NE_ERR_ARG, name + ": w_dev is NULL or misaligned");
    if (x.n == 0) return NE_OK;
    if (!x.h || !aligned(x.h, type_bytes(x.type))) return fail(NE_ERR_ARG, name + ": h_dev is NULL or misaligned");
    if (!x.targets || !aligned(x.targets, 4)) return fail(NE_ERR_ARG, name + ": targets_dev is NULL or not 4-byte aligned");
    return NE_OK;
}

// Gradients through whichever way the sizes take; with a mix, those of log probabilities and entropies.
hipError_t gradients(const SoftmaxCall& x, const XentWs& w, const Mix* mix, const float* lse, float scale, void* dh, int64_t dh_stride, void* dw,
                     int64_t dw_stride, hipStream_t st)
{
    auto run = [&](auto grad) { return grad(x, w, mix, lse, scale, dh, dh_stride, dw, dw_stride, st); };
    const bool f32 = x.type == NE_F32;
    if (mix) {
        return w.few_blocks == 1 ? (f32 ? run(run_few_grad<float, 1, true>) : run(run_few_grad<bf16_t, 1, true>))
               : w.few_blocks == 2 ? run(run_few_grad<float, 2, true>)
               : f32 ? run(run_grad<2, float, true>) : run(run_grad<1, bf16_t, true>);
    }
    return w.few_blocks == 1 ? (f32 ? run(run_few_grad<float, 1>) : run(run_few_grad<bf16_t, 1>))
           : w.few_blocks == 2 ? run(run_few_grad<float, 2>)
           : f32 ? run(run_grad<2, float>) : run(run_grad<1, bf16_t>);
}

hipError_t clear_gradient(void* dw, int64_t stride, int64_t rows, int32_t dim, int32_t type, hipStream_t st)
{
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ceil_div(rows * dim, kThreads), 4096)));
    if (type == NE_F32) hipLaunchKernelGGL(zero_kernel<float>, grid, dim3(kThreads), 0, st, static_cast<float*>(dw), stride, rows, dim);
    else hipLaunchKernelGGL(zero_kernel<bf16_t>, grid, dim3(kThreads), 0, st, static_cast<bf16_t*>(dw), stride, rows, dim);
    return hipGetLastError();
}

size_t xent_need(int64_t n, int64_t num_rows, int32_t dim, int32_t type, bool grad)
{
    return std::max(xent_bytes(n, num_rows, dim, type, grad), xent_layout(n, num_rows, dim, type, grad, nullptr).total);
}

// Rows' factors and the table's largest magnitudes lie in front of the gradients' workspace.
size_t mix_bytes(int64_t n) { return static_cast<size_t>(round_up(n * static_cast<int64_t>(sizeof(Mix)), 256) + round_up(n * 4, 256) + kMostPack * 4); }

}  // namespace

size_t logprob_grad_bytes(int64_t n, int64_t num_rows, int32_t dim, int32_t type) { return mix_bytes(n) + xent_need(n, num_rows, dim, type, true); }

extern "C" {

size_t ne_xent_workspace_bytes(int64_t n, int64_t num_rows, int32_t dim, int32_t type, int32_t grad)
{
    if (!xent_sizes_ok(n, num_rows, dim, type) || n == 0) return 0;
    return xent_need(n, num_rows, dim, type, grad != 0);
}

ne_status ne_xent_loss(const void* h_dev, int64_t h_stride, const void* w_dev, int64_t w_stride, int32_t type,
                       const int32_t* targets_dev, int64_t n, int64_t num_rows, int32_t dim, float* loss_dev,
                       float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    const SoftmaxCall x{h_dev, w_dev, h_stride, w_stride, n, num_rows, dim, type, targets_dev, nullptr};
    const ne_status rc = check_xent(x, "ne_xent_loss");
    if (rc != NE_OK || n == 0) return rc;
    if (!loss_dev || !lse_dev || !aligned(loss_dev, 4) || !aligned(lse_dev, 4)) return fail(NE_ERR_ARG, "ne_xent_loss: loss_dev or lse_dev is NULL or misaligned");
    const XentWs w = xent_layout(n, num_rows, dim, type, false, static_cast<char*>(workspace_dev));
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < std::max(xent_bytes(n, num_rows, dim, type, false), w.total))
        return fail(NE_ERR_ARG, "ne_xent_loss: workspace_dev is NULL, not 256-byte aligned, or smaller than ne_xent_workspace_bytes()");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = w.few_blocks ? (type == NE_F32 ? run_few<float>(x, w, loss_dev, lse_dev, st) : run_few<bf16_t>(x, w, loss_dev, lse_dev, st))
                                      : (type == NE_F32 ? run_loss<2>(x, w, loss_dev, lse_dev, st) : run_loss<1>(x, w, loss_dev, lse_dev, st));
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("cross entropy launch: ") + hipGetErrorString(e));
    return NE_OK;
}

ne_status ne_xent_grad(const void* h_dev, int64_t h_stride, const void* w_dev, int64_t w_stride, int32_t type,
                       const int32_t* targets_dev, const float* lse_dev, const float* loss_grad_dev, float scale,
                       int64_t n, int64_t num_rows, int32_t dim, void* dh_dev, int64_t dh_stride, void* dw_dev,
                       int64_t dw_stride, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    const SoftmaxCall x{h_dev, w_dev, h_stride, w_stride, n, num_rows, dim, type, targets_dev, loss_grad_dev};
    const ne_status rc = check_xent(x, "ne_xent_grad");
    if (rc != NE_OK) return rc;
    if (!std::isfinite(scale)) return fail(NE_ERR_ARG, "ne_xent_grad: scale is not finite");
    if ((dh_dev && dh_stride < dim) || (dw_dev && dw_stride < dim)) return fail(NE_ERR_ARG, "ne_xent_grad: a row stride is smaller than dim");
    if (!aligned(dh_dev, type_bytes(type)) || !aligned(dw_dev, type_bytes(type))) return fail(NE_ERR_ARG, "ne_xent_grad: dh_dev or dw_dev is misaligned");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (n == 0) {
        if (!dw_dev) return NE_OK;
        NE_HIP_CHECK(clear_gradient(dw_dev, dw_stride, num_rows, dim, type, st));
        return NE_OK;
    }
    if (!lse_dev || !aligned(lse_dev, 4) || !aligned(loss_grad_dev, 4)) return fail(NE_ERR_ARG, "ne_xent_grad: lse_dev is NULL, or it or loss_grad_dev misaligned");
    const XentWs w = xent_layout(n, num_rows, dim, type, true, static_cast<char*>(workspace_dev));
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < std::max(xent_bytes(n, num_rows, dim, type, true), w.total))
        return fail(NE_ERR_ARG, "ne_xent_grad: workspace_dev is NULL, not 256-byte aligned, or smaller than ne_xent_workspace_bytes()");
    if (!dh_dev && !dw_dev) return NE_OK;
    const hipError_t e = gradients(x, w, nullptr, lse_dev, scale, dh_dev, dh_stride, dw_dev, dw_stride, st);
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("cross entropy gradient launch: ") + hipGetErrorString(e));
    return NE_OK;
}

ne_status ne_logprob_grad(const void* h_dev, int64_t h_stride, const void* w_dev, int64_t w_stride, int32_t type, const int32_t* ids_dev,
                          const float* lse_dev, const float* entropy_dev, const float* logp_grad_dev, const float* entropy_grad_dev, float logp_scale,
                          float entropy_scale, int64_t n, int64_t num_rows, int32_t dim, void* dh_dev, int64_t dh_stride, void* dw_dev,
                          int64_t dw_stride, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    const std::string who = "ne_logprob_grad: ";
    if (!xent_sizes_ok(n, num_rows, dim, type)) return fail(NE_ERR_ARG, who + "n, num_rows, dim or type out of range");
    if (h_stride < dim || w_stride < dim || (dh_dev && dh_stride < dim) || (dw_dev && dw_stride < dim))
        return fail(NE_ERR_ARG, who + "a row stride is smaller than dim");
    const size_t size = type_bytes(type);
    if (!w_dev || !aligned(w_dev, size)) return fail(NE_ERR_ARG, who + "w_dev is NULL or misaligned");
    if (!aligned(dh_dev, size) || !aligned(dw_dev, size)) return fail(NE_ERR_ARG, who + "dh_dev or dw_dev is misaligned");
    if (!std::isfinite(logp_scale) || !std::isfinite(entropy_scale)) return fail(NE_ERR_ARG, who + "logp_scale or entropy_scale is not finite");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (n == 0) {
        if (dw_dev) NE_HIP_CHECK(clear_gradient(dw_dev, dw_stride, num_rows, dim, type, st));
        return NE_OK;
    }
    if (!h_dev || !aligned(h_dev, size)) return fail(NE_ERR_ARG, who + "h_dev is NULL or misaligned");
    if (!aligned(ids_dev, 4)) return fail(NE_ERR_ARG, who + "ids_dev is not 4-byte aligned");
    if (!ids_dev && logp_scale != 0.0f) return fail(NE_ERR_ARG, who + "log probabilities need ids");
    if (!lse_dev || !aligned(lse_dev, 4)) return fail(NE_ERR_ARG, who + "lse_dev is NULL or misaligned");
    if (!aligned(entropy_dev, 4) || (!entropy_dev && entropy_scale != 0.0f)) return fail(NE_ERR_ARG, who + "entropy_dev is NULL or misaligned");
    if (!aligned(logp_grad_dev, 4) || !aligned(entropy_grad_dev, 4)) return fail(NE_ERR_ARG, who + "logp_grad_dev or entropy_grad_dev is misaligned");
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < logprob_grad_bytes(n, num_rows, dim, type))
        return fail(NE_ERR_ARG, who + "workspace_dev is NULL, not 256-byte aligned, or smaller than ne_logprob_workspace_bytes()");
    if (!dh_dev && !dw_dev) return NE_OK;
    if (!ids_dev && entropy_scale == 0.0f) {        // (of nothing; entropy_dev may be NULL)
        if (dh_dev) NE_HIP_CHECK(clear_gradient(dh_dev, dh_stride, n, dim, type, st));
        if (dw_dev) NE_HIP_CHECK(clear_gradient(dw_dev, dw_stride, num_rows, dim, type, st));
        return NE_OK;
    }
    XentWs w = xent_layout(n, num_rows, dim, type, true, static_cast<char*>(workspace_dev) + mix_bytes(n));
    SoftmaxCall x{h_dev, w_dev, h_stride, w_stride, n, num_rows, dim, type, ids_dev, logp_grad_dev};
    hipError_t e;
    if (entropy_scale == 0.0f) {                    // the loss's gradient with its sign turned
        e = gradients(x, w, nullptr, lse_dev, -logp_scale, dh_dev, dh_stride, dw_dev, dw_stride, st);
    } else {
        Carver take{static_cast<char*>(workspace_dev)};
        Mix* mix = take.get<Mix>(static_cast<size_t>(n));
        float* c = take.get<float>(static_cast<size_t>(n));
        w.table_max = take.get<float>(kMostPack);
        const MixArgs a{ids_dev, logp_grad_dev, entropy_grad_dev, entropy_dev, logp_scale, entropy_scale, n, static_cast<uint32_t>(num_rows), mix, c};
        hipLaunchKernelGGL(mix_kernel, dim3(static_cast<unsigned>(ceil_div(n, kThreads))), dim3(kThreads), 0, st, a);
        e = hipGetLastError();
        x.c = c;
        if (e == hipSuccess) e = gradients(x, w, mix, lse_dev, 1.0f, dh_dev, dh_stride, dw_dev, dw_stride, st);
    }
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("log probability gradient launch: ") + hipGetErrorString(e));
    return NE_OK;
}

}  // extern "C"
