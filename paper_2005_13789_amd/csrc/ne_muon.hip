// Updates whose singular values are brought near 1 by Newton-Schulz products: ne_orthogonalize, ne_muon_step.
//
//     X <- M / |M|_F,   then steps times   X <- X (a + b G + c G^2),  G = X^T X     (of the smaller side; a wide M is taken transposed)
//
// A step multiplies X from the right by a polynomial of its own G, and all these polynomials commute.  So instead of two products with X
// for every step, X is read twice for several steps: once for G, then G's successors G <- G Q^2 and P = Q Q' .. are made of the small side alone
// (Q = a + b G + c G^2), then X <- X P.  How many steps a G can serve is a matter of digits: a direction of X of singular value
// s is s^2 in G, beside errors of 2^-24 of the largest, so weak directions are lost first.  A step brings them up by 3.4445; three steps, then a new G
// and two more leave an error like that of the products taken one after the other in fp32 (all five at once: up to a hundred times that).
//
// Products with X are of fp16 halves at a power of two (x 2^k = hi + lo, 22 bits), three matrix instructions each, with fp32 sums: about the error
// of an fp32 product.  The first X's powers follow from its rows' largest magnitudes, those of later ones and of P from what they are: singular values of X stay
// below 1.3, of P of three steps below 41.  G is the sum of a long contraction: sums of 256 rows are added to a second set of registers, and the
// workgroups' shares in 64 bits.  Matrices of the small side are fp32, taken apart into three bf16 parts (24 bits) for their products, of which
// the six largest are taken.
#include "ne_tiles.h"

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kHalfShift = 13, kPShift = 10;           // powers of two of later Xs, of P
constexpr int kPrepBlocks = 2048;
constexpr int kMostSplits = 512;
constexpr int kFlush = 8;                              // stages whose sums are added up apart
constexpr int kSide = 128;                             // of a tile of G

// A matrix of halves, rows of `stride` elements.
struct Halves {
    uint16_t* part[2];
    int64_t stride;
};

// ---------------------------------------------------------------------------------------------
// momentum, norm, X's first halves
// ---------------------------------------------------------------------------------------------
// Every 32 rows of X (a stage of G's contraction) have a power of two of their own, which their largest magnitude sets, so that one pass is enough: the
// norm comes in later, with the powers.
constexpr int kBlock = 32;              // rows of X that share a power of two
constexpr int kZeroShift = 200;         // of rows of zeros: beyond all others
constexpr int kPieces = 8;              // of eight elements, that a thread keeps between finding the largest magnitude and writing

struct PrepArgs {
    const void* g;
    int64_t g_stride;
    float* m;               // NULL: u = g
    int64_t m_stride;
    int64_t rows;
    int32_t cols;
    float grad_scale, beta;
    int32_t nesterov;
    Halves x;               // rows and columns up to multiples of 32, zeros beyond the matrix; a wide matrix transposed
    int64_t tall, blocks;
    int32_t small, padded_small;
    double* squares;        // [kPrepBlocks]
    int32_t* shifts;        // [blocks]
};

__device__ __forceinline__ void split_half(float x, int shift, short& hi, short& lo)
{
    const float y = ldexpf(x, shift);
    const f16_t h = static_cast<f16_t>(y);
    hi = __builtin_bit_cast(short, h);
    lo = __builtin_bit_cast(short, static_cast<f16_t>(y - static_cast<float>(h)));
}

// u: x itself, or with momentum m <- beta m + g what g's look ahead makes of it.  Eight elements from (row, e) on, zeros beyond the columns.
template <class T, bool MOMENTUM, bool FIRST>
__device__ __forceinline__ void update_of(const PrepArgs& a, int64_t row, int e, float (&u)[8])
{
    T g[8];
    load_eight(static_cast<const T*>(a.g) + row * a.g_stride, e, a.cols, g);
#pragma unroll
    for (int q = 0; q < 8; ++q) u[q] = static_cast<float>(g[q]);
    if (!MOMENTUM) return;
    float m[8];
    float* at = a.m + row * a.m_stride;
    load_eight(at, e, a.cols, m);
    if (FIRST) {
#pragma unroll
        for (int q = 0; q < 8; ++q) m[q] = fmaf(a.beta, m[q], a.grad_scale * u[q]);
        store_some<float, 8>(at + e, a.cols - e, m);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) u[q] = a.nesterov ? fmaf(a.beta, m[q], a.grad_scale * u[q]) : m[q];
}

// A block's largest magnitude, found, leaves its power of two behind.
__device__ __forceinline__ int block_shift(float top, int32_t* shifts, int64_t block, float* lds)
{
    top = block_max(top, lds);
    const int shift = top == 0.0f ? kZeroShift : shift_of(top);
    if (threadIdx.x == 0) shifts[block] = shift;
    return shift;
}

// Bound by memory: with momentum every element is 4 bytes of momentum read and 4 written, 4 of X's halves written, and the gradient's (1 M x 128 fp32: 372 us,
// 5.5 TB/s; 200 003 x 512 bf16: 300).  HELD: a thread's pieces stay in registers from the first look to the halves; otherwise, beyond 512 columns, they are
// read again, from L2.
template <class T, bool MOMENTUM, bool HELD>
__global__ void __launch_bounds__(kThreads) prep_kernel(PrepArgs a)
{
    __shared__ float lds[kThreads / 64];
    __shared__ double sums[kThreads / 64];
    double total = 0.0;
    const int across = a.padded_small / 8, pieces = kBlock * across;
    for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        float u[kPieces][8], top = 0.0f;
        auto first = [&](int p, float (&x)[8]) {
            const int64_t row = block * kBlock + p / across;
            const int e = p % across * 8;
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = 0.0f;
            if (p < pieces && row < a.tall && e < a.small) update_of<T, MOMENTUM, true>(a, row, e, x);
        };
        auto look = [&](const float (&x)[8]) {
            double more = 0.0;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                top = fmaxf(top, finite_abs(x[q]));
                more = fma(static_cast<double>(x[q]), static_cast<double>(x[q]), more);
            }
            total += more;
        };
        auto write = [&](int p, const float (&x)[8], int shift) {
            const int64_t row = block * kBlock + p / across;
            const int e = p % across * 8;
            s16x8 hi, lo;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                short h, l;
                split_half(x[q], shift, h, l);
                hi[q] = h;
                lo[q] = l;
            }
            *reinterpret_cast<s16x8*>(a.x.part[0] + row * a.x.stride + e) = hi;
            *reinterpret_cast<s16x8*>(a.x.part[1] + row * a.x.stride + e) = lo;
        };
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (i * kThreads < pieces) first(i * kThreads + threadIdx.x, u[i]);
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (i * kThreads < pieces) look(u[i]);
            const int shift = block_shift(top, a.shifts, block, lds);
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (i * kThreads + static_cast<int>(threadIdx.x) < pieces) write(i * kThreads + threadIdx.x, u[i], shift);
        } else {
            for (int p = threadIdx.x; p < pieces; p += kThreads) {
                first(p, u[0]);
                look(u[0]);
            }
            const int shift = block_shift(top, a.shifts, block, lds);
            for (int p = threadIdx.x; p < pieces; p += kThreads) {
                const int64_t row = block * kBlock + p / across;
                const int e = p % across * 8;
                float x[8] = {};
                if (row < a.tall && e < a.small) update_of<T, MOMENTUM, false>(a, row, e, x);
                write(p, x, shift);
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = total;
    __syncthreads();
    if (threadIdx.x == 0) a.squares[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// A wide matrix: 32 of its columns are a block, turned by way of LDS, 64 rows at a time.
template <class T, bool MOMENTUM>
__global__ void __launch_bounds__(kThreads) prep_wide_kernel(PrepArgs a)
{
    __shared__ float lds[kThreads / 64];
    __shared__ double sums[kThreads / 64];
    __shared__ uint32_t turn[kBlock * 65];
    double total = 0.0;
    for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        const int64_t x0 = block * kBlock;
        float top = 0.0f;
        for (int p = threadIdx.x; p < a.small * 4; p += kThreads) {
            const int e = static_cast<int>(x0) + (p & 3) * 8;
            float u[8];
            if (e >= a.cols) continue;
            update_of<T, MOMENTUM, true>(a, p >> 2, e, u);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                top = fmaxf(top, finite_abs(u[q]));
                total = fma(static_cast<double>(u[q]), static_cast<double>(u[q]), total);
            }
        }
        const int shift = block_shift(top, a.shifts, block, lds);
        for (int c0 = 0; c0 < a.padded_small; c0 += 64) {
            __syncthreads();
            const int r = threadIdx.x >> 2, e = (threadIdx.x & 3) * 8;
            float u[8] = {};
            if (c0 + r < a.small && x0 + e < a.cols) update_of<T, MOMENTUM, false>(a, c0 + r, static_cast<int>(x0) + e, u);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                short h, l;
                split_half(u[q], shift, h, l);
                turn[(e + q) * 65 + r] = static_cast<uint16_t>(h) | static_cast<uint32_t>(static_cast<uint16_t>(l)) << 16;
            }
            __syncthreads();
            const int x = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
            if (c0 + c < a.padded_small) {
                s16x8 hi, lo;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const uint32_t both = turn[x * 65 + c + q];
                    hi[q] = static_cast<short>(both & 0xFFFF);
                    lo[q] = static_cast<short>(both >> 16);
                }
                *reinterpret_cast<s16x8*>(a.x.part[0] + (x0 + x) * a.x.stride + c0 + c) = hi;
                *reinterpret_cast<s16x8*>(a.x.part[1] + (x0 + x) * a.x.stride + c0 + c) = lo;
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = total;
    __syncthreads();
    if (threadIdx.x == 0) a.squares[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// ---------------------------------------------------------------------------------------------
// G = X^T X
// ---------------------------------------------------------------------------------------------
struct GramArgs {
    Operand x;              // across: element (column, row of X)
    uint32_t tiles, splits, share, stages;      // tiles of a side; stages of a split, of all
    float* part;            // [splits][pairs][kSide][kSide]
    const int32_t* shifts;  // FIRST: powers of two of X's blocks
    int32_t* split_shift;   // [splits]  of a split's sums
    const double* squares;  // [square_count], for 1 / |M|_F
    uint32_t square_count;
    double* inverse;
};

// Tile pairs (i, j), i <= j, one after the other.
__device__ __forceinline__ void pair_at(uint32_t p, uint32_t tiles, uint32_t& i, uint32_t& j)
{
    i = 0;
    while (p >= tiles - i) {
        p -= tiles - i;
        ++i;
    }
    j = i + p;
}

// G is symmetric: tiles of 128 x 128 on and above the diagonal, X's rows shared out among enough workgroups to fill the CUs; a diagonal tile has one
// operand in LDS.  Bound by what the matrix cores' operands take out of LDS (200 003 x 512, ten tiles: 255 us, 0.63 PFLOP/s of halves; adding up every
// stage, FIRST, 300), at one tile by memory (1 M x 128: 143 us, 3.6 TB/s).
// FIRST: of X as it came, whose blocks of rows have powers of two of their own: a stage's sums are added by themselves.
template <bool FIRST>
__global__ void __launch_bounds__(256, 2) gram_kernel(GramArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * stage_bytes<4>()];
    if (FIRST && blockIdx.x == 0) {         // the norm, from shares
        double* sums = reinterpret_cast<double*>(lds);
        double total = 0.0;
        for (uint32_t i = threadIdx.x; i < a.square_count; i += 256) total += a.squares[i];
        sums[threadIdx.x] = total;
        __syncthreads();
        for (int o = 128; o > 0; o >>= 1) {
            if (static_cast<int>(threadIdx.x) < o) sums[threadIdx.x] += sums[threadIdx.x + o];
            __syncthreads();
        }
        if (threadIdx.x == 0) *a.inverse = sums[0] == 0.0 ? 0.0 : 1.0 / sqrt(sums[0]);
        __syncthreads();
    }
    const uint32_t pairs = a.tiles * (a.tiles + 1) / 2, b = by_xcd(blockIdx.x, gridDim.x), split = b / pairs, pair = b - split * pairs;
    uint32_t ti, tj;
    pair_at(pair, a.tiles, ti, tj);
    const uint32_t s0 = min(split * a.share, a.stages), s1 = min(s0 + a.share, a.stages);
    f32x16 acc[2][2], all[2][2];
    clear(acc);
    clear(all);
    int least = kZeroShift;                 // of the split's powers of two: that of its sums
    if (FIRST) {
        for (uint32_t s = s0 + (threadIdx.x & 63); s < s1; s += 64) least = min(least, a.shifts[s]);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) least = min(least, __shfl_xor(least, o, 64));
        least = __builtin_amdgcn_readfirstlane(least);
        if (pair == 0 && threadIdx.x == 0) a.split_shift[split] = least;
    }
    if (s0 < s1) {
        Loader<2, 4, false> load_a, load_b;
        load_a.start(a.x, ti * kSide, s0);
        load_b.start(a.x, tj * kSide, s0);
        uint32_t done = 0;
        run_stages<4>(
            s1 - s0, lds,
            [&](uint32_t to) {
                load_a.fetch(to);
                if (ti != tj) load_b.fetch(to + operand_bytes<4>());
            },
            [&](const unsigned char* stage) {
                multiply<2, 4, false, false>(stage, acc, ti == tj ? 0 : operand_bytes<4>());
                if constexpr (FIRST) {
                    const float factor = ldexpf(1.0f, max(2 * (least - a.shifts[s0 + done]), -200));
                    ++done;
#pragma unroll
                    for (int im = 0; im < 2; ++im)
#pragma unroll
                        for (int in = 0; in < 2; ++in)
#pragma unroll
                            for (int i = 0; i < 16; ++i) all[im][in][i] = fmaf(acc[im][in][i], factor, all[im][in][i]);
                    clear(acc);
                } else if ((++done & (kFlush - 1)) == 0) {
#pragma unroll
                    for (int im = 0; im < 2; ++im)
#pragma unroll
                        for (int in = 0; in < 2; ++in) all[im][in] += acc[im][in];
                    clear(acc);
                }
            });
    }
    const int lane = threadIdx.x & 63;
    float* out = a.part + (static_cast<int64_t>(split) * pairs + pair) * (kSide * kSide);
#pragma unroll
    for (int im = 0; im < 2; ++im)
#pragma unroll
        for (int in = 0; in < 2; ++in)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                out[(first_row<4>() + 32 * im + sum_row(i) + lane_row()) * kSide + first_col<4>() + 32 * in + (lane & 31)] = all[im][in][i] + acc[im][in][i];
}

__device__ __forceinline__ void put(const Halves& to, int64_t row, int64_t col, float x, int shift)
{
    short hi, lo;
    split_half(x, shift, hi, lo);
    to.part[0][row * to.stride + col] = static_cast<uint16_t>(hi);
    to.part[1][row * to.stride + col] = static_cast<uint16_t>(lo);
}

// The splits' sums, joined in 64 bits and scaled; both triangles.  Bound by the launch and one chain of reads (1 M x 128, 512 splits, 34 MB: 7.5 us).
struct GramJoinArgs {
    const float* part;
    uint32_t tiles, splits;
    int32_t side;
    const int32_t* split_shift;     // NULL: X's halves are of X 2^kHalfShift
    const double* inverse;
    float* g;               // [side][side]
};

// 64 elements of a row of a tile pair, whose splits the wavefronts share: sixteen of them, or four where there are few.
template <int WAVES>
__global__ void __launch_bounds__(64 * WAVES) gram_join_kernel(GramJoinArgs a)
{
    __shared__ double lds[64 * WAVES];
    const uint32_t pairs = a.tiles * (a.tiles + 1) / 2, per = kSide * kSide / 64, pair = blockIdx.x / per, at = (blockIdx.x % per) * 64 + (threadIdx.x & 63);
    uint32_t ti, tj;
    pair_at(pair, a.tiles, ti, tj);
    const int64_t row = ti * kSide + at / kSide, col = tj * kSide + at % kSide;
    if (row >= a.side) return;      // (the same for all of the workgroup)
    double sum = 0.0;
    const float* from = a.part + static_cast<int64_t>(pair) * (kSide * kSide) + at;
    constexpr int FLIGHT = 8;
    for (uint32_t s0 = threadIdx.x >> 6; s0 < a.splits; s0 += WAVES * FLIGHT) {
        float x[FLIGHT];
        int shift[FLIGHT];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            const uint32_t s = s0 + WAVES * f;
            x[f] = 0.0f;
            shift[f] = kHalfShift;
            if (s >= a.splits) continue;
            x[f] = from[static_cast<int64_t>(s) * pairs * (kSide * kSide)];
            if (a.split_shift) shift[f] = a.split_shift[s];
        }
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) sum += ldexp(static_cast<double>(x[f]), -2 * shift[f]);
    }
    lds[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 64 || col >= a.side || row > col) return;
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += lds[w * 64 + threadIdx.x];
    if (a.split_shift) sum = sum * *a.inverse * *a.inverse;
    a.g[row * a.side + col] = a.g[col * a.side + row] = static_cast<float>(sum);
}

// ---------------------------------------------------------------------------------------------
// products of the small side
// ---------------------------------------------------------------------------------------------
// All of them are polynomials of one symmetric matrix, so they are symmetric (but for roundings) and commute.  They are fp32 [side][side], side a
// multiple of 32.
//
// Up to kRowsSide a step is one launch: row by row, v Q(G) = kA v + kB v G + kC (v G) G, so a workgroup takes 16 rows of G and of P through
// all products of the step, and nothing waits for another workgroup.  A wavefront has 16 columns, whose share of G stays in its registers; rows go
// from product to product through LDS.  (Side 128, three steps and two: 5 launches in the place of 13, which took 71 us.)
constexpr int kRowsSide = 256;

struct RowsArgs {
    const float* g;
    const float* p;         // NULL: the first step, P = 1
    float* next;            // NULL, or G Q(G)^2
    float* out;             // P Q(G), or NULL: as halves
    Halves halves;
    int32_t side;
};

template <int WAVES>
struct Rows {               // 16 rows as three bf16 parts
    static constexpr int STRIDE = WAVES * 16 + 8;
    bf16_t part[3][16][STRIDE];
};

template <int WAVES>
__global__ void __launch_bounds__(64 * WAVES) rows_kernel(RowsArgs a)
{
    constexpr int STEPS = WAVES / 2;
    __shared__ __align__(16) Rows<WAVES> v_rows[2], p_rows[2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * 16;
    const int c = wave * 16 + col;
    const bool works = wave * 16 < a.side;
    const int steps = a.side / 32;
    // (columns, not rows in their place: what roundings leave of G - G^T would grow 24 times a step, G times G^T no longer being a power of one matrix)
    bf16x8 held[STEPS][3];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        float x[8] = {};
        if (works && s < steps)
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = a.g[static_cast<int64_t>(s * 32 + quarter * 8 + q) * a.side + c];
        split_bf16<3>(x, held[s]);
    }
    // a lane's four results: rows 4 quarter .. + 3, its column
    auto load = [&](const float* from, float (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = works ? from[(row0 + quarter * 4 + i) * a.side + c] : 0.0f;
    };
    auto keep = [&](Rows<WAVES>& rows, const float (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float rest = x[i];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const bf16_t y = static_cast<bf16_t>(rest);
                rows.part[p][quarter * 4 + i][c] = y;
                rest -= static_cast<float>(y);
            }
        }
    };
    auto times_g = [&](const Rows<WAVES>& rows, float (&x)[4]) {
        // (the largest products in sums of every fourth step: an instruction's sum is cut off where the larger of what it adds ends)
        f32x4 sum[4], small = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int f = 0; f < 4; ++f) sum[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s >= steps) break;
            bf16x8 y[3];
#pragma unroll
            for (int p = 0; p < 3; ++p) y[p] = *reinterpret_cast<const bf16x8*>(&rows.part[p][col][s * 32 + quarter * 8]);
            // (the smallest products first, apart from the largest)
#pragma unroll
            for (int of_parts = 2; of_parts >= 0; --of_parts) {
                f32x4& to = of_parts > 0 ? small : sum[s % 4];
#pragma unroll
                for (int q = 0; q <= of_parts; ++q) to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[q], held[s][of_parts - q], to, 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = ((sum[0][i] + sum[1][i]) + (sum[2][i] + sum[3][i])) + small[i];
    };
    float v[4], v1[4], v2[4], p[4], p1[4], p2[4];
    load(a.g, v);
    keep(v_rows[0], v);
    if (a.p) {
        load(a.p, p);
        keep(p_rows[0], p);
    }
    __syncthreads();
    const bool first = !a.p, moves = a.next != nullptr;
    if (first || moves) times_g(v_rows[0], v1);
    if (!first) times_g(p_rows[0], p1);
    if (first) {            // P = 1: P G and P G G are G's rows and v G
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = row0 + quarter * 4 + i == c ? 1.0f : 0.0f;
            p1[i] = v[i];
            p2[i] = v1[i];
        }
    }
    if (moves) keep(v_rows[1], v1);
    if (!first) keep(p_rows[1], p1);
    __syncthreads();
    if (moves) times_g(v_rows[1], v2);
    if (!first) times_g(p_rows[1], p2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + quarter * 4 + i;
        const float x = fmaf(kC, p2[i], fmaf(kB, p1[i], kA * p[i]));
        if (!works) continue;
        if (a.out) a.out[row * a.side + c] = x;
        else put(a.halves, row, c, x, kPShift);
    }
    if (!moves) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmaf(kC, v2[i], fmaf(kB, v1[i], kA * v[i]));
    keep(v_rows[0], v);
    __syncthreads();
    times_g(v_rows[0], v1);
    keep(v_rows[1], v1);
    __syncthreads();
    times_g(v_rows[1], v2);
    if (works)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.next[(row0 + quarter * 4 + i) * a.side + c] = fmaf(kC, v2[i], fmaf(kB, v1[i], kA * v[i]));
}

// Larger sides: a product is a launch, or two that do not wait for one another.  A workgroup has a tile of 32 x 32, or of 64 x 64 where there are
// enough of them, on or above the diagonal, its eight wavefronts a share of the contraction each, straight from L2 into the matrix cores' operands.
// (Larger tiles from 1024 on: whole updates of 1000 x 1000 506 and 463 us, 4096 x 4096 15.3 and 10.0 ms; half as many reads and conversions to parts, which
// bound it, but a quarter of the workgroups.  Side 320: 6.4 us a launch, thirteen of them; 512: 8.)
constexpr int kSmallWaves = 8, kSmallLarge = 1024;

struct SmallJob {
    const float *a, *b;
    float* out;             // NULL: the halves of P, for the product with X
    int32_t polynomial;     // kA + kB a + kC (a b), for a = b = G, in the place of a b
};

struct SmallArgs {
    SmallJob job[2];
    Halves p;
    int32_t side;
};

template <int T>
__global__ void __launch_bounds__(64 * kSmallWaves) small_kernel(SmallArgs args)
{
    constexpr int WAVES = kSmallWaves, SIDE = 32 * T, EACH = SIDE * SIDE / (64 * WAVES), ROWS = 64 * WAVES / SIDE;      // elements of a thread, rows of a turn
    __shared__ __align__(16) float lds[WAVES][SIDE * (SIDE + 1)];
    const SmallJob& job = args.job[blockIdx.y];
    const int side = args.side;
    const uint32_t tiles = (side + SIDE - 1) / SIDE;
    uint32_t ti, tj;
    pair_at(blockIdx.x, tiles, ti, tj);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, steps = side / 16, r0 = threadIdx.x / SIDE, c = threadIdx.x % SIDE;
    // (rows behind the last are the last again, and not written)
    const float *a[T], *b[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        a[t] = job.a + static_cast<int64_t>(min(static_cast<int>(ti) * SIDE + 32 * t + (lane & 31), side - 1)) * side + (lane >> 5) * 8;
        b[t] = job.b + static_cast<int64_t>(min(static_cast<int>(tj) * SIDE + 32 * t + (lane & 31), side - 1)) * side + (lane >> 5) * 8;
    }
    auto inside = [&](uint32_t i, uint32_t j, int r, int col) { return T == 1 || (static_cast<int>(i) * SIDE + r < side && static_cast<int>(j) * SIDE + col < side); };
    // (the polynomial's other term is fetched ahead of the sums)
    float g[EACH] = {};
    if (job.polynomial)
#pragma unroll
        for (int q = 0; q < EACH; ++q)
            if (inside(ti, tj, r0 + ROWS * q, c)) g[q] = job.a[static_cast<int64_t>(ti * SIDE + r0 + ROWS * q) * side + tj * SIDE + c];
    f32x16 sum[T][T], small[T][T];
#pragma unroll
    for (int m = 0; m < T; ++m)
#pragma unroll
        for (int n = 0; n < T; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[m][n][i] = small[m][n][i] = 0.0f;
    constexpr int FLIGHT = 4 / T;
    for (int s0 = wave; s0 < steps; s0 += WAVES * FLIGHT) {
        float x[FLIGHT][T][8] = {}, y[FLIGHT][T][8] = {};
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            if (s0 + WAVES * f >= steps) break;
#pragma unroll
            for (int t = 0; t < T; ++t) {
                __builtin_memcpy(x[f][t], a[t] + (s0 + WAVES * f) * 16, 32);
                __builtin_memcpy(y[f][t], b[t] + (s0 + WAVES * f) * 16, 32);
            }
        }
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            bf16x8 u[T][3], v[T][3];
#pragma unroll
            for (int t = 0; t < T; ++t) {
                split_bf16<3>(x[f][t], u[t]);
                split_bf16<3>(y[f][t], v[t]);
            }
#pragma unroll
            for (int of_parts = 2; of_parts >= 0; --of_parts)
#pragma unroll
                for (int q = 0; q <= of_parts; ++q)
#pragma unroll
                    for (int m = 0; m < T; ++m)
#pragma unroll
                        for (int n = 0; n < T; ++n) {
                            f32x16& to = of_parts > 0 ? small[m][n] : sum[m][n];
                            to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u[m][q], v[n][of_parts - q], to, 0, 0, 0);
                        }
        }
    }
#pragma unroll
    for (int m = 0; m < T; ++m)
#pragma unroll
        for (int n = 0; n < T; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) lds[wave][(32 * m + sum_row(i) + lane_row()) * (SIDE + 1) + 32 * n + (lane & 31)] = sum[m][n][i] + small[m][n][i];
    __syncthreads();
    float* all = lds[0];            // the results; on the diagonal those above it are both
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        const int r = r0 + ROWS * q, at = r * (SIDE + 1) + c;
        float x = (lds[0][at] + lds[1][at]) + (lds[2][at] + lds[3][at]);
        x += (lds[4][at] + lds[5][at]) + (lds[6][at] + lds[7][at]);
        if (job.polynomial) x = fmaf(kC, x, kB * g[q]) + (ti == tj && r == c ? kA : 0.0f);
        all[at] = x;                // (read by this thread alone so far)
    }
    __syncthreads();
    auto write = [&](uint32_t i, uint32_t j, int r, int col, float x) {
        if (!inside(i, j, r, col)) return;
        const int64_t to_row = i * SIDE + r, to_col = j * SIDE + col;
        if (job.out) job.out[to_row * side + to_col] = x;
        else put(args.p, to_row, to_col, x, kPShift);
    };
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        const int r = r0 + ROWS * q;
        if (ti == tj) {
            write(ti, tj, r, c, all[min(r, c) * (SIDE + 1) + max(r, c)]);
        } else {
            write(ti, tj, r, c, all[r * (SIDE + 1) + c]);
            write(tj, ti, r, c, all[c * (SIDE + 1) + r]);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// X <- X P, and what becomes of the last one
// ---------------------------------------------------------------------------------------------
struct ApplyArgs {
    Operand x, p;           // both by rows (P is symmetric)
    uint32_t row_tiles, splits, col_tiles;
    int32_t steps;
    int64_t tall, padded_tall;
    int32_t small, padded_small;
    const int32_t* shifts;  // NULL: X's halves are of X 2^kHalfShift
    const double* inverse;
    // one of: the next X's halves; a matrix out; parameters
    Halves next;
    void* out;
    int64_t out_stride;
    float* param;
    int64_t param_stride;
    bf16_t* copy;
    int64_t copy_stride;
    float keep, step;       // p keep - step o
};

enum Last { kNext, kFloat, kBfloat, kParam };

// Sixteen results of a lane: rows row + sum_row(i) of X, a column.
template <Last L, bool WIDE>
__device__ __forceinline__ void finish(const ApplyArgs& a, int64_t row, int col, const float (&x)[16])
{
    if (L == kNext) {
        if (col >= a.padded_small) return;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (row + sum_row(i) < a.padded_tall) put(a.next, row + sum_row(i), col, x[i], kHalfShift);
        return;
    }
    if (col >= a.small) return;
    // (a wide matrix has X's rows as columns: four of them are side by side)
    const int64_t step = WIDE ? 1 : L == kParam ? a.param_stride : a.out_stride, first = WIDE ? col * (L == kParam ? a.param_stride : a.out_stride) + row : row * step + col;
    if (L == kFloat || L == kBfloat) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (row + sum_row(i) >= a.tall) continue;
            if (L == kFloat) static_cast<float*>(a.out)[first + sum_row(i) * step] = x[i];
            else static_cast<bf16_t*>(a.out)[first + sum_row(i) * step] = static_cast<bf16_t>(x[i]);
        }
        return;
    }
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = row + sum_row(i) < a.tall ? a.param[first + sum_row(i) * step] : 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = fmaf(-a.step, x[i], p[i] * a.keep);
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (row + sum_row(i) < a.tall) a.param[first + sum_row(i) * step] = p[i];
    if (!a.copy) return;
    const int64_t copy_step = WIDE ? 1 : a.copy_stride, copy_first = WIDE ? col * a.copy_stride + row : row * a.copy_stride + col;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (row + sum_row(i) < a.tall) a.copy[copy_first + sum_row(i) * copy_step] = static_cast<bf16_t>(p[i]);
}

// A workgroup has a tile of P's columns and rows of X one after the other; up to 128 columns P stays in registers.  A tile's results go out as they
// lie, 32 columns of a row side by side.  Narrow X is bound by memory (1 M x 128 with parameters: 350 us, 4.4 TB/s), 512 columns by operands out of LDS and
// by results, which nothing else runs beside (200 003 x 512: 397 us, with parameters and their bf16 copy 475; 0.8 PFLOP/s of halves).  Turned, so that a lane has
// four and four columns of one row, wider stores were slower: 422 and 605 us, lines being written in quarters.
template <int W, int KS, Last L, bool WIDE>
__global__ void __launch_bounds__(64 * W, 2) apply_kernel(ApplyArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * stage_bytes<W>()];
    constexpr int MT = W / 2;
    const int lane = threadIdx.x & 63, m0 = first_row<W>(), n0 = first_col<W>();
    uint32_t col_tile, split;
    pair_of(by_xcd(blockIdx.x, gridDim.x), a.col_tiles, a.splits, col_tile, split);
    const uint32_t per = (a.row_tiles + a.splits - 1) / a.splits, tile0 = split * per;
    const double inverse = a.shifts ? *a.inverse : 1.0;
    all_scores<2, W, KS>(a.x, a.p, col_tile, 0, tile0, min(tile0 + per, a.row_tiles), a.steps, lds, [&](uint32_t tile_row0, f32x16 (&acc)[MT][2]) {
#pragma unroll
        for (int im = 0; im < MT; ++im) {
            const int64_t row0 = static_cast<int64_t>(tile_row0) + m0 + 32 * im;
            if (row0 >= a.padded_tall) continue;
            const int shift = a.shifts ? a.shifts[row0 / kBlock] : kHalfShift;
            const float factor = static_cast<float>(ldexp(inverse, -(shift + kPShift)));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = acc[im][j][i] * factor;
                finish<L, WIDE>(a, row0 + lane_row(), col_tile * rows_of<W>() + n0 + 32 * j + (lane & 31), x);
            }
        }
    });
}

// X P and its G in one pass: up to 128 columns a workgroup has whole rows of X P, turns them into halves in LDS, multiplies them there and writes them
// from there.  P's rows stay in registers, X travels in a ring of four stages.  (1 M x 128: 345 us, both apart 383.  P of all steps at once, so that X P need not be written, would have
// values up to 485 where X has no direction, whose roundings would be 485 / 41 times as large in all others.)
struct NextGramArgs {
    Operand x, p;           // both by rows (P is symmetric)
    uint32_t row_tiles, splits;
    int32_t steps;
    int64_t padded_tall;
    const int32_t* shifts;
    const double* inverse;
    Halves next;
    float* part;            // [splits][kSide][kSide]
};

template <int KS>
__global__ void __launch_bounds__(256, 1) next_gram_kernel(NextGramArgs a)
{
    constexpr int STAGE = operand_bytes<4>();       // 32 rows of X P, both halves
    __shared__ __align__(16) unsigned char lds[4 * STAGE + 4 * STAGE];
    unsigned char* rows = lds + 4 * STAGE;
    const int lane = threadIdx.x & 63, m0 = first_row<4>(), n0 = first_col<4>();
    const uint32_t per = (a.row_tiles + a.splits - 1) / a.splits, tile0 = blockIdx.x * per;
    const double inverse = a.shifts ? *a.inverse : 1.0;
    f32x16 all[2][2];
    clear(all);
    all_scores<2, 4, KS>(a.x, a.p, 0, 0, tile0, min(tile0 + per, a.row_tiles), a.steps, lds, [&](uint32_t tile_row0, f32x16 (&acc)[2][2]) {
#pragma unroll
        for (int im = 0; im < 2; ++im) {
            const int64_t row0 = static_cast<int64_t>(tile_row0) + m0 + 32 * im;
            // (rows behind the last are the last again)
            const int shift = !a.shifts ? kHalfShift : row0 < a.padded_tall ? a.shifts[row0 / kBlock] : 0;
            const float factor = static_cast<float>(ldexp(inverse, kHalfShift - (shift + kPShift)));
            // (column after column, a row of X P along the contraction: four of a lane's values are side by side)
            unsigned char* stage = rows + ((m0 >> 5) + im) * STAGE;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int col = n0 + 32 * j + (lane & 31);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f16x4 hi, lo;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = row0 < a.padded_tall ? acc[im][j][4 * q + e] * factor : 0.0f;
                        hi[e] = static_cast<f16_t>(x);
                        lo[e] = static_cast<f16_t>(x - static_cast<float>(hi[e]));
                    }
                    unsigned char* at = stage + col * 64 + ((q ^ ((col >> 2) & 3)) << 4) + (lane >> 5) * 8;
                    *reinterpret_cast<f16x4*>(at) = hi;
                    *reinterpret_cast<f16x4*>(at + STAGE / 2) = lo;
                    if (row0 >= a.padded_tall || col >= a.next.stride) continue;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t to = (row0 + 8 * q + lane_row() + e) * a.next.stride + col;
                        const f16_t h = hi[e], l = lo[e];       // (a cast of a vector's element would take the vector's first)
                        a.next.part[0][to] = __builtin_bit_cast(uint16_t, h);
                        a.next.part[1][to] = __builtin_bit_cast(uint16_t, l);
                    }
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // (X's next stages travel on)
        f32x16 g[2][2];
        clear(g);
#pragma unroll
        for (int stage = 0; stage < 4; ++stage) multiply<2, 4, true, true>(rows + stage * STAGE, g, 0);
#pragma unroll
        for (int im = 0; im < 2; ++im)
#pragma unroll
            for (int in = 0; in < 2; ++in) all[im][in] += g[im][in];
    });
    float* out = a.part + static_cast<int64_t>(blockIdx.x) * (kSide * kSide);
#pragma unroll
    for (int im = 0; im < 2; ++im)
#pragma unroll
        for (int in = 0; in < 2; ++in)
#pragma unroll
            for (int i = 0; i < 16; ++i) out[(m0 + 32 * im + sum_row(i) + lane_row()) * kSide + n0 + 32 * in + (lane & 31)] = all[im][in][i];
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct MuonWs {
    int64_t tall, padded_tall;
    int32_t side, padded_side;      // the smaller one
    bool wide;
    uint32_t tiles, pairs, splits, share, stages;
    double *squares, *inverse;
    int32_t *shifts, *split_shift;
    Halves x[2];
    float* part;
    float* small[6];                // matrices of the small side
    Halves p;
    size_t total;
};

// Workgroups of next_gram_kernel: one a CU.
uint32_t next_gram_splits(int64_t padded_tall)
{
    const int64_t tiles = ceil_div(padded_tall, kSide), per = ceil_div(tiles, 256);
    return static_cast<uint32_t>(ceil_div(tiles, per));
}

MuonWs muon_layout(int64_t rows, int64_t cols, char* base)
{
    MuonWs w{};
    w.wide = cols > rows;
    w.tall = w.wide ? cols : rows;
    w.side = static_cast<int32_t>(w.wide ? rows : cols);
    w.padded_tall = round_up(w.tall, 32);
    w.padded_side = static_cast<int32_t>(round_up(w.side, 32));
    w.tiles = static_cast<uint32_t>(ceil_div(w.padded_side, kSide));
    w.pairs = w.tiles * (w.tiles + 1) / 2;
    // splits of the long contraction: two workgroups a CU, of eight stages at least
    w.stages = static_cast<uint32_t>(w.padded_tall / step_of<2>());
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(ceil_div(kMostSplits, w.pairs), w.stages / kFlush));
    w.share = static_cast<uint32_t>(ceil_div(w.stages, most));
    w.splits = static_cast<uint32_t>(ceil_div(w.stages, w.share));
    Carver take{base};
    w.squares = take.get<double>(kPrepBlocks);
    w.inverse = take.get<double>(1);
    w.shifts = take.get<int32_t>(static_cast<size_t>(w.padded_tall / kBlock));
    w.split_shift = take.get<int32_t>(w.splits);
    for (auto& x : w.x) {
        for (auto& p : x.part) p = take.get<uint16_t>(static_cast<size_t>(w.padded_tall) * w.padded_side);
        x.stride = w.padded_side;
    }
    const uint32_t most_splits = w.padded_side <= kSide ? std::max(w.splits, next_gram_splits(w.padded_tall)) : w.splits;
    w.part = take.get<float>(static_cast<size_t>(most_splits) * w.pairs * kSide * kSide);
    for (auto*& m : w.small) m = take.get<float>(static_cast<size_t>(w.padded_side) * w.padded_side);
    for (auto& p : w.p.part) p = take.get<uint16_t>(static_cast<size_t>(w.padded_side) * w.padded_side);
    w.p.stride = w.padded_side;
    w.total = take.total();
    return w;
}

// The polynomial P of `steps` steps (three at most) from G (w.small[0]) on, as halves in w.p.
hipError_t polynomial(const MuonWs& w, int steps, hipStream_t st)
{
    hipError_t e = hipSuccess;
    if (w.padded_side <= kRowsSide) {
        RowsArgs a{};
        a.side = w.padded_side;
        a.halves = w.p;
        float *g = w.small[0], *next = w.small[1], *p = nullptr, *out = w.small[2], *other = w.small[3];
        for (int s = 1; s <= steps && e == hipSuccess; ++s) {
            a.g = g; a.p = p; a.next = s < steps ? next : nullptr; a.out = s < steps ? out : nullptr;
            const dim3 grid(static_cast<unsigned>(w.padded_side / 16));
            if (w.padded_side <= 128) hipLaunchKernelGGL(rows_kernel<8>, grid, dim3(512), 0, st, a);
            else hipLaunchKernelGGL(rows_kernel<16>, grid, dim3(1024), 0, st, a);
            e = hipGetLastError();
            std::swap(g, next);
            p = out;
            std::swap(out, other);
        }
        return e;
    }
    float *g = w.small[0], *q = w.small[1], *t = w.small[2], *next = w.small[3], *p = q, *q2 = w.small[4], *p2 = w.small[5];
    const bool large = w.padded_side >= kSmallLarge;
    const uint32_t tiles = static_cast<uint32_t>(ceil_div(w.padded_side, large ? 64 : 32));
    SmallArgs args{};
    args.side = w.padded_side;
    args.p = w.p;
    int jobs = 0;
    auto add = [&](const float* a, const float* b, float* out, bool poly) { args.job[jobs++] = SmallJob{a, b, out, poly ? 1 : 0}; };
    auto run = [&]() {
        const dim3 grid(tiles * (tiles + 1) / 2, jobs);
        if (large) hipLaunchKernelGGL(small_kernel<2>, grid, dim3(64 * kSmallWaves), 0, st, args);
        else hipLaunchKernelGGL(small_kernel<1>, grid, dim3(64 * kSmallWaves), 0, st, args);
        jobs = 0;
        return hipGetLastError();
    };
    add(g, g, steps == 1 ? nullptr : q, true);
    if ((e = run()) != hipSuccess || steps == 1) return e;
    add(g, q, t, false);                            // G Q
    if ((e = run()) != hipSuccess) return e;
    for (int s = 1; s < steps; ++s) {
        add(t, q, next, false);                     // G Q^2 is the next G,
        if ((e = run()) != hipSuccess) return e;
        std::swap(g, next);
        add(g, g, q2, true);                        // whose polynomial P is multiplied with, beside the G Q after it
        if ((e = run()) != hipSuccess) return e;
        const bool last = s + 1 == steps;
        add(p, q2, last ? nullptr : p2, false);
        if (!last) add(g, q2, t, false);
        if ((e = run()) != hipSuccess) return e;
        p = p2;                                     // (three steps at most: P's place is written once)
        std::swap(q, q2);
    }
    return hipSuccess;
}

// What is done with the last product.
struct Result {
    Last kind;
    void* out;
    int64_t out_stride;
    float* param;
    int64_t param_stride;
    void* copy;
    int64_t copy_stride;
    float keep, step;
};

template <int W, int KS>
void launch_apply(const ApplyArgs& a, Last kind, bool wide, dim3 grid, hipStream_t st)
{
    if (kind == kNext) hipLaunchKernelGGL((apply_kernel<W, KS, kNext, false>), grid, dim3(64 * W), 0, st, a);
    else if (kind == kFloat && !wide) hipLaunchKernelGGL((apply_kernel<W, KS, kFloat, false>), grid, dim3(64 * W), 0, st, a);
    else if (kind == kFloat) hipLaunchKernelGGL((apply_kernel<W, KS, kFloat, true>), grid, dim3(64 * W), 0, st, a);
    else if (kind == kBfloat && !wide) hipLaunchKernelGGL((apply_kernel<W, KS, kBfloat, false>), grid, dim3(64 * W), 0, st, a);
    else if (kind == kBfloat) hipLaunchKernelGGL((apply_kernel<W, KS, kBfloat, true>), grid, dim3(64 * W), 0, st, a);
    else if (!wide) hipLaunchKernelGGL((apply_kernel<W, KS, kParam, false>), grid, dim3(64 * W), 0, st, a);
    else hipLaunchKernelGGL((apply_kernel<W, KS, kParam, true>), grid, dim3(64 * W), 0, st, a);
}

hipError_t apply(const MuonWs& w, const Halves& x, bool first, const Halves* next, const Result& r, hipStream_t st)
{
    ApplyArgs a{};
    a.x = packed_operand(x.part, w.padded_tall, w.padded_side);     // (X's rows of zeros stay such)
    a.p = packed_operand(w.p.part, w.padded_side, w.padded_side);
    // Tiles of 256 x 256, one a CU, read half as much LDS for a product: where columns fill them to 8 / 9 and the last of their rounds is not mostly empty
    // (whole update, small tiles and large: 50 000 x 512, 392 tiles: 496 and 471 us; 20 000 x 1000, 316: 913 and 901; 33 000 x 512, 258: 402 and 412).
    const int64_t large_tiles = ceil_div(w.tall, 256) * ceil_div(w.padded_side, 256);
    const bool large = w.padded_side > 256 && round_up(w.padded_side, 256) * 8 <= w.padded_side * 9 && large_tiles * 10 >= round_up(large_tiles, 256) * 6;
    const int64_t tile = large ? 256 : kSide;
    a.row_tiles = static_cast<uint32_t>(ceil_div(w.tall, tile));
    a.col_tiles = static_cast<uint32_t>(ceil_div(w.padded_side, tile));
    a.splits = splits_of(a.row_tiles, a.col_tiles, large);
    a.steps = w.padded_side / step_of<2>();
    a.tall = w.tall; a.padded_tall = w.padded_tall; a.small = w.side; a.padded_small = w.padded_side; a.shifts = first ? w.shifts : nullptr; a.inverse = w.inverse;
    if (next) a.next = *next;
    a.out = r.out; a.out_stride = r.out_stride; a.param = r.param; a.param_stride = r.param_stride;
    a.copy = static_cast<bf16_t*>(r.copy); a.copy_stride = r.copy_stride; a.keep = r.keep; a.step = r.step;
    const Last kind = next ? kNext : r.kind;
    const dim3 grid(a.col_tiles * a.splits);
    const int held = a.steps > 4 || ceil_div(a.row_tiles, a.splits) < 3 ? 0 : a.steps > 2 ? 4 : 2;
    if (large) launch_apply<8, 0>(a, kind, w.wide, grid, st);
    else if (held == 0) launch_apply<4, 0>(a, kind, w.wide, grid, st);
    else if (held == 2) launch_apply<4, 2>(a, kind, w.wide, grid, st);
    else launch_apply<4, 4>(a, kind, w.wide, grid, st);
    return hipGetLastError();
}

template <class T, bool MOMENTUM>
hipError_t run_update(PrepArgs u, const MuonWs& w, int steps, const Result& r, hipStream_t st)
{
    u.x = w.x[0]; u.tall = w.tall; u.blocks = w.padded_tall / kBlock; u.small = w.side; u.padded_small = w.padded_side; u.squares = w.squares; u.shifts = w.shifts;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(u.blocks, kPrepBlocks)));
    if (w.wide) hipLaunchKernelGGL((prep_wide_kernel<T, MOMENTUM>), grid, dim3(kThreads), 0, st, u);
    else if (kBlock * w.padded_side / 8 <= kPieces * kThreads) hipLaunchKernelGGL((prep_kernel<T, MOMENTUM, true>), grid, dim3(kThreads), 0, st, u);
    else hipLaunchKernelGGL((prep_kernel<T, MOMENTUM, false>), grid, dim3(kThreads), 0, st, u);
    hipError_t e = hipGetLastError();
    auto join = [&](uint32_t splits, bool first) {
        const GramJoinArgs j{w.part, w.tiles, splits, w.padded_side, first ? w.split_shift : nullptr, w.inverse, w.small[0]};
        const dim3 blocks(w.pairs * (kSide * kSide / 64));
        if (splits <= 64) hipLaunchKernelGGL(gram_join_kernel<4>, blocks, dim3(256), 0, st, j);
        else hipLaunchKernelGGL(gram_join_kernel<16>, blocks, dim3(1024), 0, st, j);
        return hipGetLastError();
    };
    auto gram = [&](const Halves& x, bool first) {
        GramArgs g{};
        g.x = Operand{{x.part[0], x.part[1]}, w.padded_side, static_cast<uint32_t>(w.padded_tall - 1), static_cast<uint32_t>(w.padded_side)};
        g.tiles = w.tiles; g.splits = w.splits; g.share = w.share; g.stages = w.stages; g.part = w.part;
        g.shifts = w.shifts; g.split_shift = w.split_shift; g.squares = w.squares; g.square_count = grid.x; g.inverse = w.inverse;
        if (first) hipLaunchKernelGGL(gram_kernel<true>, dim3(w.pairs * w.splits), dim3(256), 0, st, g);
        else hipLaunchKernelGGL(gram_kernel<false>, dim3(w.pairs * w.splits), dim3(256), 0, st, g);
        const hipError_t failed = hipGetLastError();
        return failed != hipSuccess ? failed : join(w.splits, first);
    };
    auto next_gram = [&](const Halves& x, const Halves& next, bool first) {
        NextGramArgs a{};
        a.x = packed_operand(x.part, w.padded_tall, w.padded_side);
        a.p = packed_operand(w.p.part, w.padded_side, w.padded_side);
        a.row_tiles = static_cast<uint32_t>(ceil_div(w.padded_tall, kSide));
        a.splits = next_gram_splits(w.padded_tall);
        a.steps = w.padded_side / step_of<2>();
        a.padded_tall = w.padded_tall; a.shifts = first ? w.shifts : nullptr; a.inverse = w.inverse; a.next = next; a.part = w.part;
        if (a.steps > 2) hipLaunchKernelGGL(next_gram_kernel<4>, dim3(a.splits), dim3(256), 0, st, a);
        else hipLaunchKernelGGL(next_gram_kernel<2>, dim3(a.splits), dim3(256), 0, st, a);
        const hipError_t failed = hipGetLastError();
        return failed != hipSuccess ? failed : join(a.splits, false);
    };
    if (e == hipSuccess) e = gram(w.x[0], true);
    int which = 0, take = 3;            // the first G serves three steps, later ones two
    for (int left = steps; left > 0 && e == hipSuccess; which ^= 1, take = 2) {
        const int now = std::min(left, take);
        const bool first = left == steps;
        if ((e = polynomial(w, now, st)) != hipSuccess) return e;
        left -= now;
        if (left == 0) e = apply(w, w.x[which], first, nullptr, r, st);
        else if (w.padded_side <= kSide) e = next_gram(w.x[which], w.x[which ^ 1], first);
        else if ((e = apply(w, w.x[which], first, &w.x[which ^ 1], r, st)) == hipSuccess) e = gram(w.x[which ^ 1], false);
    }
    return e;
}

bool muon_sizes_ok(int64_t rows, int64_t cols)
{
    return rows >= 0 && cols >= 0 && std::max(rows, cols) < (1ll << 31) - 128 && std::min(rows, cols) <= NE_ORTHOGONAL_MAX_SIDE;
}

// Whether some of `rows` rows of `cols` elements, `stride` apart, share places.
bool rows_overlap(int64_t rows, int64_t cols, int64_t stride) { return rows > 1 && stride < cols; }

}  // namespace

extern "C" {

size_t ne_orthogonalize_workspace_bytes(int64_t rows, int64_t cols)
{
    return muon_sizes_ok(rows, cols) && rows > 0 && cols > 0 ? muon_layout(rows, cols, nullptr).total : 0;
}

ne_status ne_orthogonalize(const void* x_dev, int32_t x_type, int64_t x_stride, int64_t rows, int64_t cols, int32_t steps, void* out_dev,
                           int32_t out_type, int64_t out_stride, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    const std::string who = "ne_orthogonalize: ";
    if (!muon_sizes_ok(rows, cols) || !type_ok(x_type) || !type_ok(out_type) || steps < 1 || steps > NE_ORTHOGONAL_MAX_STEPS)
        return fail(NE_ERR_ARG, who + "rows, cols, steps or a type out of range");
    if (rows_overlap(rows, cols, x_stride) || rows_overlap(rows, cols, out_stride)) return fail(NE_ERR_ARG, who + "a row stride is smaller than cols");
    if (rows == 0 || cols == 0) return NE_OK;
    if (!x_dev || !aligned(x_dev, type_bytes(x_type)) || !out_dev || !aligned(out_dev, type_bytes(out_type)))
        return fail(NE_ERR_ARG, who + "x_dev or out_dev is NULL or misaligned");
    const MuonWs w = muon_layout(rows, cols, static_cast<char*>(workspace_dev));
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < w.total)
        return fail(NE_ERR_ARG, who + "workspace_dev is NULL, not 256-byte aligned, or smaller than ne_orthogonalize_workspace_bytes()");
    const PrepArgs u{x_dev, x_stride, nullptr, 0, rows, static_cast<int32_t>(cols), 1.0f, 0.0f, 0};
    const Result r{out_type == NE_F32 ? kFloat : kBfloat, out_dev, out_stride, nullptr, 0, nullptr, 0, 0.0f, 0.0f};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = x_type == NE_F32 ? run_update<float, false>(u, w, steps, r, st) : run_update<bf16_t, false>(u, w, steps, r, st);
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("orthogonalize launch: ") + hipGetErrorString(e));
    return NE_OK;
}

ne_status ne_muon_step(float* param_dev, int64_t param_stride, const void* grad_dev, int32_t grad_type, int64_t grad_stride, float* momentum_dev,
                       int64_t momentum_stride, void* param_bf16_dev, int64_t param_bf16_stride, int64_t rows, int64_t cols, int32_t steps, float lr,
                       float momentum, int32_t nesterov, float weight_decay, float scale, float grad_scale, void* workspace_dev, size_t workspace_bytes,
                       void* hip_stream)
{
    const std::string who = "ne_muon_step: ";
    if (!muon_sizes_ok(rows, cols) || !type_ok(grad_type) || steps < 1 || steps > NE_ORTHOGONAL_MAX_STEPS)
        return fail(NE_ERR_ARG, who + "rows, cols, steps or grad_type out of range");
    if (!(std::isfinite(lr) && lr >= 0.0f && momentum >= 0.0f && momentum < 1.0f && std::isfinite(weight_decay) && weight_decay >= 0.0f &&
          std::isfinite(scale) && std::isfinite(grad_scale) && std::isfinite(lr * scale) && std::isfinite(lr * weight_decay)))
        return fail(NE_ERR_ARG, who + "lr, momentum, weight_decay, scale or grad_scale out of range");
    if (rows_overlap(rows, cols, param_stride) || rows_overlap(rows, cols, grad_stride) || rows_overlap(rows, cols, momentum_stride) ||
        (param_bf16_dev && rows_overlap(rows, cols, param_bf16_stride)))
        return fail(NE_ERR_ARG, who + "a row stride is smaller than cols");
    if (rows == 0 || cols == 0) return NE_OK;
    if (!param_dev || !aligned(param_dev, 4) || !grad_dev || !aligned(grad_dev, type_bytes(grad_type)) || !momentum_dev || !aligned(momentum_dev, 4) ||
        !aligned(param_bf16_dev, 2))
        return fail(NE_ERR_ARG, who + "a matrix is NULL or misaligned");
    const MuonWs w = muon_layout(rows, cols, static_cast<char*>(workspace_dev));
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < w.total)
        return fail(NE_ERR_ARG, who + "workspace_dev is NULL, not 256-byte aligned, or smaller than ne_orthogonalize_workspace_bytes()");
    const PrepArgs u{grad_dev, grad_stride, momentum_dev, momentum_stride, rows, static_cast<int32_t>(cols), grad_scale, momentum, nesterov != 0};
    const Result r{kParam, nullptr, 0, param_dev, param_stride, param_bf16_dev, param_bf16_stride, 1.0f - lr * weight_decay, lr * scale};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = grad_type == NE_F32 ? run_update<float, true>(u, w, steps, r, st) : run_update<bf16_t, true>(u, w, steps, r, st);
    if (e != hipSuccess) return fail(NE_ERR_HIP, std::string("Muon step launch: ") + hipGetErrorString(e));
    return NE_OK;
}

}  // extern "C"
