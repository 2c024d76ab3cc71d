// Matrix products of tiles, and what scores of rows against a whole table are made with: stages of operands that travel to LDS a stage
// ahead, their reads and matrix instructions, packing into operands, tiles of scores.
//
// Operands in LDS are 16-byte pieces placed so that reads are free of bank conflicts (an XOR of the piece's
// index with the row's); they come from memory straight to LDS, 16 bytes a lane, and the XOR is applied to the
// address that a lane reads.  Operands whose rows run along the contraction are read with the transposing LDS read.
#pragma once
#include <type_traits>

#include "ne_internal.h"
#include "ne_ops.h"

namespace {

typedef _Float16 f16_t;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kAmaxBlocks = 1024, kMostPack = 2048;      // (bf16: each of the packing workgroups leaves a maximum, in the room of three times 1024)
static_assert(kMostPack <= 3 * kAmaxBlocks);
constexpr int64_t kMostStride = 1 << 22;   // elements: a tile's 256 rows are within 32 bits of its first
constexpr int kFewBytes = 65536, kFewBytesAlone = 153600;     // LDS of H for the loss: of a workgroup of 4 wavefronts, and of one of 8 that is alone on its CU
constexpr int kFewGroups = 1024;
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

template <int P> constexpr int step_of() { return P == 1 ? 64 : 32; }   // contraction indices of a stage

// A tile of sums is 128 x 128, of four wavefronts (W = 4) with 64 x 64 each, or 256 x 256, of eight (W = 8) with 128 x 64 each.  Two stages
// of a large tile fill LDS (128 KB), so one workgroup runs on a CU; of small tiles two run, and one multiplies while the other
// takes exponentials or waits.  Per operation a large tile fetches half as much from L2, which is what bounds the small ones.
template <int W> constexpr int rows_of() { return W == 8 ? 256 : 128; }
template <int W> constexpr int operand_bytes() { return rows_of<W>() * 128; }   // one operand's share of a stage in LDS (all its parts)
template <int W> constexpr int stage_bytes() { return 2 * operand_bytes<W>(); }
constexpr int slots_of(bool large) { return large ? 256 : 512; }        // workgroups that run at once

// An operand of a product.  ROWS: element (row, k) at row * stride + k.  Otherwise (row, k) at k * stride + row.
struct Operand {
    const uint16_t* part[2];
    int64_t stride;
    uint32_t last;      // ROWS: last row; otherwise: last k
    uint32_t width;     // elements of a row that there are: a multiple of 8
};

// ---------------------------------------------------------------------------------------------
// a stage: rows_of<W>() rows x step_of<P>() contraction indices of each operand's P parts
// ---------------------------------------------------------------------------------------------
// Loads go from memory to LDS directly, and are waited for once a stage (stage_done), before the barrier that hands the stage
// over: a stage is in flight while the one before it is multiplied.  They are written in assembly because the compiler waits for
// loads of this kind before every LDS read that follows.  The address is a uniform base and a lane's offset, which stays the same
// from stage to stage.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"     // (m0 is reserved: nothing is allocated to it, which is no reason not to name it)
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits for all but the last LATER loads of this wavefront, and for the other wavefronts.
template <int LATER = 0>
__device__ __forceinline__ void stage_done() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory"); }

__device__ __forceinline__ uint32_t lds_address(const unsigned char* p)
{
    return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) unsigned char*)p)));
}

// Rows row0 .. row0 + rows_of<W>() - 1 of an operand, stage after stage, in pieces of 1 KB.
template <int P, int W, bool ROWS>
struct Loader {
    static constexpr int R = rows_of<W>(), kPieces = 4 / P;     // pieces of a wavefront, per part
    const unsigned char* base[P];
    int64_t advance;               // bytes from one stage to the next
    uint32_t offset[kPieces];
    uint32_t stride, ks;           // bytes of a row; contraction indices that are left

    __device__ __forceinline__ static int piece(int q) { return q * W + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)); }

    // ROWS: which 16 bytes of its row a lane fetches: those that are read from the lane's place in LDS.  (Pieces of rows 0, 2, 4 .. lie at
    // the index XOR 0, 1, 2 ..; half-length rows 0, 4, 8 ..: so the 16 rows that LDS serves at a time are in different banks.)
    __device__ __forceinline__ static uint32_t place_in_row()
    {
        const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        return P == 1 ? (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4)) : (lane & 3) ^ (lane >> 4);
    }

    // Otherwise: which contraction index of the stage.
    __device__ __forceinline__ static uint32_t k_of(int q)
    {
        const int lane = threadIdx.x & 63;
        return R == 128 ? piece(q) * 4 + (lane >> 4) : piece(q) * 2 + (lane >> 5);
    }

    __device__ __forceinline__ void start(const Operand& o, uint32_t row0, uint32_t stage)
    {
        const int lane = threadIdx.x & 63;
        stride = static_cast<uint32_t>(o.stride * 2);
        const int64_t first = ROWS ? static_cast<int64_t>(row0) * o.stride + stage * step_of<P>() : static_cast<int64_t>(stage) * step_of<P>() * o.stride;
        advance = ROWS ? step_of<P>() * 2 : static_cast<int64_t>(step_of<P>()) * o.stride * 2;
        ks = (ROWS ? o.width : o.last + 1) - stage * step_of<P>();
#pragma unroll
        for (int p = 0; p < P; ++p) base[p] = reinterpret_cast<const unsigned char*>(o.part[p] + first);
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
            if (ROWS) {
                const uint32_t row = P == 1 ? piece(q) * 8 + (lane >> 3) : piece(q) * 16 + (lane >> 2);
                offset[q] = min(row, o.last - row0) * stride + place_in_row() * 16;
            } else {        // (the 32 bytes u of row k lie at u XOR 2 (k % 4))
                const uint32_t k = k_of(q), col = row0 + (((lane & (R / 8 - 1)) ^ ((k & 3) << 2)) << 3);
                offset[q] = k * stride + min(col, o.width - 8) * 2;
            }
        }
    }

    // (contraction indices beyond the last ones are those again: the other operand has zeros there)
    __device__ __forceinline__ void fetch(uint32_t lds)
    {
        uint32_t back[kPieces] = {};
        if (ks < static_cast<uint32_t>(step_of<P>()))
#pragma unroll
            for (int q = 0; q < kPieces; ++q) {
                const uint32_t k = ROWS ? 8 * place_in_row() : k_of(q);
                back[q] = ROWS ? (k - min(k, ks - 8)) * 2 : (k - min(k, ks - 1)) * stride;
            }
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int q = 0; q < kPieces; ++q) load_to_lds(base[p], offset[q] - back[q], lds + p * (operand_bytes<W>() / P) + piece(q) * 1024);
            base[p] += advance;
        }
        ks -= step_of<P>();
    }
};

// What lane l supplies for rows r0 .. r0 + 31 and contraction indices 16 kk .. + 15 of a stage: row l % 32, the eight
// indices from (l / 32) * 8 on.
template <int P, int W, bool ROWS>
__device__ __forceinline__ s16x8 fragment(const unsigned char* lds, int part, int r0, int kk)
{
    constexpr int R = rows_of<W>();
    const int lane = threadIdx.x & 63;
    const unsigned char* base = lds + part * (operand_bytes<W>() / P);
    if (ROWS) {
        const int row = r0 + (lane & 31), piece = kk * 2 + (lane >> 5);
        const int at = P == 1 ? row * 128 + ((piece ^ ((row >> 1) & 7)) << 4) : row * 64 + ((piece ^ ((row >> 2) & 3)) << 4);
        return *reinterpret_cast<const s16x8*>(base + at);
    }
    // 16 lanes get 16 columns of 4 rows: lane i points to the i % 4-th 8 bytes of row i / 4 and receives column i
    const int i = lane & 15, g = lane >> 4;
    const int k = kk * 16 + (g >> 1) * 8 + (i >> 2), unit = (r0 >> 4) + (g & 1);
    const int at = k * (2 * R) + ((unit ^ ((i >> 2) << 1)) << 5) + ((i & 3) << 3);
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + at));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + at + 8 * R));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// What operands hold: as their parts say (one: bf16, two: fp16 halves), fp16, or the second one fp16 that becomes bf16 for its products, rounded or as the sum of two.
enum Kind { kPlain, kHalf, kToBf16, kToTwoBf16 };

__device__ __forceinline__ s16x8 to_bf16(s16x8 x)
{
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(s16x8, __builtin_convertvector(__builtin_convertvector(__builtin_bit_cast(f16x8, x), f32x8), bf16x8));
}

// Returns what rounding leaves out, which bf16 holds exactly.
__device__ __forceinline__ s16x8 to_two_bf16(s16x8& x)
{
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    const f32x8 whole = __builtin_convertvector(__builtin_bit_cast(f16x8, x), f32x8);
    const bf16x8 most = __builtin_convertvector(whole, bf16x8);
    x = __builtin_bit_cast(s16x8, most);
    return __builtin_bit_cast(s16x8, __builtin_convertvector(whole - __builtin_convertvector(most, f32x8), bf16x8));
}

template <int P, Kind K = kPlain>
__device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
{
    if (P == 1 && K != kHalf) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Where a wavefront's share of a tile begins.
template <int W> __device__ __forceinline__ int first_row() { return static_cast<int>(threadIdx.x >> 6) / (W / 2) * (rows_of<W>() / 2); }
template <int W> __device__ __forceinline__ int first_col() { return static_cast<int>(threadIdx.x >> 6) % (W / 2) * 64; }

// acc[im][in] += A B^T over one stage (b_at: where B lies behind A, 0 where A is B).
template <int P, int W, bool AROWS, bool BROWS, Kind K = kPlain>
__device__ __forceinline__ void multiply(const unsigned char* stage, f32x16 (&acc)[W / 2][2], int b_at = operand_bytes<W>())
{
    constexpr int MT = W / 2, KK = step_of<P>() / 16;
    const int m0 = first_row<W>(), n0 = first_col<W>();
    const unsigned char* A = stage;
    const unsigned char* B = stage + b_at;
    // Operands of the next 16 indices are read while these are multiplied: a read takes as long as four products.  (The compiler would
    // reuse the registers at once and wait for every read.)
    s16x8 a[2][P][MT], b[2][P][2], more[2][2];
    auto read = [&](int kk) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int i = 0; i < MT; ++i) a[kk & 1][p][i] = fragment<P, W, AROWS>(A, p, m0 + 32 * i, kk);
#pragma unroll
            for (int i = 0; i < 2; ++i) b[kk & 1][p][i] = fragment<P, W, BROWS>(B, p, n0 + 32 * i, kk);
        }
    };
    // (in the middle of the products before: they have been read by then, and the other half hides it)
    auto convert = [&](int kk) {
        if (K == kToBf16)
#pragma unroll
            for (int in = 0; in < 2; ++in) b[kk & 1][0][in] = to_bf16(b[kk & 1][0][in]);
        if (K == kToTwoBf16)
#pragma unroll
            for (int in = 0; in < 2; ++in) more[kk & 1][in] = to_two_bf16(b[kk & 1][0][in]);
    };
    read(0);
    convert(0);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        if (kk + 1 < KK) read(kk + 1);
        __builtin_amdgcn_sched_barrier(0);
        const int at = kk & 1;
#pragma unroll
        for (int im = 0; im < MT; ++im) {
            if (im == MT / 2 && kk + 1 < KK) convert(kk + 1);
#pragma unroll
            for (int in = 0; in < 2; ++in) {
                acc[im][in] = mfma<P, K>(a[at][0][im], b[at][0][in], acc[im][in]);
                if (K == kToTwoBf16) acc[im][in] = mfma<P>(a[at][0][im], more[at][in], acc[im][in]);
                if (P == 2) {
                    acc[im][in] = mfma<P>(a[at][0][im], b[at][P - 1][in], acc[im][in]);
                    acc[im][in] = mfma<P>(a[at][P - 1][im], b[at][0][in], acc[im][in]);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int MT>
__device__ __forceinline__ void clear(f32x16 (&acc)[MT][2])
{
#pragma unroll
    for (int im = 0; im < MT; ++im)
#pragma unroll
        for (int in = 0; in < 2; ++in)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[im][in][i] = 0.0f;
}

// All stages of a workgroup, one travelling while the one before it is used: get(lds) fetches the next, use(stage) multiplies one.
template <int W, class Get, class Use>
__device__ __forceinline__ void run_stages(uint32_t stages, unsigned char* lds, Get get, Use use)
{
    const uint32_t lds0 = lds_address(lds);
    if (stages) get(lds0);
    stage_done();
    for (uint32_t s = 0; s < stages; ++s) {
        if (s + 1 < stages) get(lds0 + ((s + 1) & 1) * stage_bytes<W>());
        use(lds + (s & 1) * stage_bytes<W>());
        stage_done();
    }
}

// Workgroups go to the eight XCDs in turn, and each XCD has an L2 of its own: this numbers them so that an XCD's have
// consecutive numbers, and what neighbours share is fetched into one L2.
__device__ __forceinline__ uint32_t by_xcd(uint32_t block, uint32_t blocks)
{
    const uint32_t xcd = block & 7, per = blocks >> 3, more = blocks & 7;
    return xcd * per + min(xcd, more) + (block >> 3);
}

// Number b of tiles_a x tiles_b pairs, eight of a against one of b after the other: neighbours share their operands with one another, and with
// by_xcd in one L2 (all scores of 8192 x 200 003 x 512: 1.97 ms in plain order, 1.79 so).
__device__ __forceinline__ void pair_of(uint32_t b, uint32_t tiles_a, uint32_t tiles_b, uint32_t& ta, uint32_t& tb)
{
    const uint32_t group = b / (8 * tiles_b), rest = b - group * 8 * tiles_b, size = min(8u, tiles_a - group * 8);
    tb = rest / size;
    ta = group * 8 + rest - tb * size;
}

// Row (of 32) of a lane's i-th sum, without the lane's own share of it.
constexpr int sum_row(int i) { return (i & 3) + 8 * (i >> 2); }
__device__ __forceinline__ uint32_t lane_row() { return 4 * ((threadIdx.x & 63) >> 5); }

// ---------------------------------------------------------------------------------------------
// packing
// ---------------------------------------------------------------------------------------------
// Largest finite magnitudes, kAmaxBlocks of each: of W, of H's rows with a target, of the same rows times c_i.
struct AmaxArgs {
    const float* h;
    const float* w;
    const int32_t* targets;
    const float* c;
    int64_t h_stride, w_stride, n, num_rows;
    int32_t dim;
    float* amax;        // [3][kAmaxBlocks]
};

__device__ __forceinline__ float finite_abs(float x)
{
    x = fabsf(x);
    return x < INFINITY ? x : 0.0f;     // (false for a NaN)
}

template <int THREADS = kThreads>
__device__ __forceinline__ float block_max(float v, float* lds)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v = fmaxf(v, lds[w]);
    return v;
}

// Eight elements from index e on, zeros beyond dim.
template <class T>
__device__ __forceinline__ void load_eight(const T* row, int e, int dim, T (&x)[8])
{
    if (e + 8 <= dim) {
        __builtin_memcpy(x, row + e, 8 * sizeof(T));
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = e + q < dim ? row[e + q] : from_float<T>(0.0f);
    }
}

// Rows of `dim` elements, eight a lane: use(row, e, x) for a lane group's rows, two of them in flight.
template <int THREADS = kThreads, class T, class Use>
__device__ __forceinline__ void for_eights(const T* in, int64_t stride, int64_t rows, int dim, int width, uint32_t block, uint32_t blocks, Use use)
{
    int lanes_log2 = 0;
    while (lanes_log2 < 6 && (8 << lanes_log2) < width) ++lanes_log2;
    const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t groups = static_cast<int64_t>(blocks) * (THREADS >> lanes_log2);
    const int64_t first = static_cast<int64_t>(block) * (THREADS >> lanes_log2) + (threadIdx.x >> lanes_log2);
    for (int e = lane * 8; e < width; e += 8 * lanes)
        for (int64_t r = first; r < rows; r += 4 * groups) {
            T x[4][8];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (r + q * groups < rows) load_eight(in + (r + q * groups) * stride, e, dim, x[q]);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (r + q * groups < rows) use(r + q * groups, e, x[q]);
        }
}

// (Bound by memory: 84 284 rows of 452, 152 MB: 29 us, 5.2 TB/s.  A small table's 5 us are a launch.)
__global__ void __launch_bounds__(kThreads) amax_kernel(AmaxArgs a)
{
    __shared__ float lds[4];
    float w = 0.0f, h = 0.0f, ch = 0.0f;
    for_eights(a.w, a.w_stride, a.num_rows, a.dim, a.dim, blockIdx.x, gridDim.x, [&](int64_t, int, const float (&x)[8]) {
#pragma unroll
        for (int q = 0; q < 8; ++q) w = fmaxf(w, finite_abs(x[q]));
    });
    for_eights(a.h, a.h_stride, a.n, a.dim, a.dim, blockIdx.x, gridDim.x, [&](int64_t i, int, const float (&x)[8]) {
        if (a.targets && static_cast<uint32_t>(a.targets[i]) >= static_cast<uint32_t>(a.num_rows)) return;
        const float c = a.c ? a.c[i] : 1.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            h = fmaxf(h, finite_abs(x[q]));
            ch = fmaxf(ch, finite_abs(c * x[q]));
        }
    });
    w = block_max(w, lds);
    h = block_max(h, lds);
    ch = block_max(ch, lds);
    if (threadIdx.x == 0) {
        a.amax[blockIdx.x] = w;
        a.amax[kAmaxBlocks + blockIdx.x] = h;
        a.amax[2 * kAmaxBlocks + blockIdx.x] = ch;
    }
}

// The power of two that brings a matrix's largest magnitude into [2^13, 2^14).
__device__ __forceinline__ int shift_of(float amax)
{
    if (amax == 0.0f) return 0;
    const int e = static_cast<int>(__float_as_uint(amax) >> 23);
    return 13 - (max(e, 1) - 127);
}

// (Bound by memory: 84 284 rows of 452 fp32, 312 MB read and written: 57 us, 5.5 TB/s.)
struct PackArgs {
    const void* in;
    int64_t in_stride, rows, padded_rows;
    const int32_t* targets;        // rows without a target become zeros; NULL: all rows count
    uint32_t num_targets;
    const float* c;                // NULL, or factors of the rows
    int32_t dim, padded;
    uint16_t* out[2];              // P == 1: NULL where only the largest magnitude is wanted
    const float* amax;             // NULL: bf16 as it is (factors aside); otherwise `maxima` largest magnitudes, for fp16 parts
    int32_t* shift;                // receives their power of two
    int32_t maxima;
    float* amax_out;               // NULL, or where every workgroup leaves the largest magnitude of its rows times their factors
};

struct PackJobs {
    PackArgs job[3];
};

// look(e, x): sees every eight elements that are packed, from column e on.
template <int P, int THREADS, class Look>
__device__ __forceinline__ void pack_rows(const PackArgs& a, uint32_t block, uint32_t blocks, float* lds, Look look)
{
    typedef typename std::conditional<P == 2, float, bf16_t>::type T;
    int k = 0;
    if (a.amax) {
        float top = 0.0f;
#pragma unroll 4
        for (int i = threadIdx.x; i < a.maxima; i += THREADS) top = fmaxf(top, a.amax[i]);
        k = shift_of(block_max<THREADS>(top, lds));
        if (block == 0 && threadIdx.x == 0) *a.shift = k;
    }
    float largest = 0.0f;
    auto write = [&](int64_t r, int e0, const T (&x)[8]) {
        s16x8 out[P] = {};
        look(e0, x);
        const bool counts = !a.targets || static_cast<uint32_t>(a.targets[r]) < a.num_targets;
        const float c = a.c ? a.c[r] : 1.0f;
        if (P == 2 || a.amax) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = counts ? ldexpf(c * static_cast<float>(x[e]), k) : 0.0f;
                const f16_t hi = static_cast<f16_t>(y);
                out[0][e] = __builtin_bit_cast(short, hi);
                if constexpr (P == 2) out[1][e] = __builtin_bit_cast(short, static_cast<f16_t>(y - static_cast<float>(hi)));
            }
        } else if (counts) {
            __builtin_memcpy(&out[0], x, 16);
            if (a.amax_out)
#pragma unroll
                for (int e = 0; e < 8; ++e) largest = fmaxf(largest, finite_abs(c * static_cast<float>(x[e])));
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (P == 2 || a.out[p]) *reinterpret_cast<s16x8*>(a.out[p] + r * a.padded + e0) = out[p];
    };
    for_eights<THREADS>(static_cast<const T*>(a.in), a.in_stride, a.rows, a.dim, a.padded, block, blocks, write);
    // rows beyond the last one: zeros
    const int64_t zeros = (a.padded_rows - a.rows) * a.padded / 8;
    for (int64_t i = static_cast<int64_t>(block) * THREADS + threadIdx.x; i < zeros; i += static_cast<int64_t>(blocks) * THREADS)
#pragma unroll
        for (int p = 0; p < P; ++p) *reinterpret_cast<s16x8*>(a.out[p] + a.rows * a.padded + i * 8) = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (P == 1 && a.amax_out) {
        largest = block_max<THREADS>(largest, lds);
        if (threadIdx.x == 0) a.amax_out[block] = largest;
    }
}

template <int P, int THREADS>
__device__ __forceinline__ void pack_rows(const PackArgs& a, uint32_t block, uint32_t blocks, float* lds)
{
    pack_rows<P, THREADS>(a, block, blocks, lds, [](int, const auto&) {});
}

template <int P>
__global__ void __launch_bounds__(kThreads) pack_kernel(PackJobs jobs)
{
    __shared__ float lds[kThreads / 64];
    pack_rows<P, kThreads>(jobs.job[blockIdx.y], blockIdx.x, gridDim.x, lds);
}

// ---------------------------------------------------------------------------------------------
// scores of a tile of table rows against one of H
// ---------------------------------------------------------------------------------------------
// A softmax's maximum and sum, in powers of two, joined with those of other scores.
__device__ __forceinline__ void join_stat(float& top, float& sum, float2 other)
{
    const float now = fmaxf(top, other.x), by = now == -INFINITY ? 0.0f : now;      // (nothing seen yet but scores of minus infinity)
    sum = sum * __builtin_amdgcn_exp2f(top - by) + other.y * __builtin_amdgcn_exp2f(other.x - by);
    top = now;
}

template <int P>
__device__ __forceinline__ float score_factor(const int32_t* shift)
{
    if (P == 1) return 1.0f;
    return ldexpf(1.0f, max(min(-(shift[0] + shift[1]), 127), -126));
}

// Scores of tiles tile0 .. tile1 - 1 of the table's rows against one tile of H's, epilogue(row0, acc) for each; the next tile's first
// stage travels meanwhile.
template <int P, int W, class Epilogue>
__device__ __forceinline__ void score_tiles(const Operand& w, const Operand& h, uint32_t token_tile, uint32_t first, uint32_t tile0, uint32_t tile1, int steps,
                                            unsigned char* lds, Epilogue epilogue)
{
    constexpr int R = rows_of<W>();
    f32x16 acc[W / 2][2];
    clear(acc);
    Loader<P, W, true> load_w, load_h;
    uint32_t row0 = first + tile0 * R, next_row0 = row0;
    int step = 0, next_step = 0;
    run_stages<W>(
        tile1 > tile0 ? (tile1 - tile0) * steps : 0, lds,
        [&](uint32_t to) {
            if (next_step == 0) {
                load_w.start(w, next_row0, 0);
                load_h.start(h, token_tile * R, 0);
            }
            load_w.fetch(to);
            load_h.fetch(to + operand_bytes<W>());
            if (++next_step == steps) { next_step = 0; next_row0 += R; }
        },
        [&](const unsigned char* stage) {
            multiply<P, W, true, true>(stage, acc);
            if (++step == steps) {
                epilogue(row0, acc);
                clear(acc);
                step = 0;
                row0 += R;
            }
        });
}

// The same with small tiles where H's rows have at most KS stages: a wavefront holds its 64 rows of H in registers, as the operands that they
// are, and only the table travels, in a ring of four stages, three of them ahead.  (Loads from L2 are what bounds these shapes: 10 007 rows
// against 10 000 of 100, fp32: 94 us, 5 more with H through LDS; a copy without the exponentials took 73, without loads 87.)
template <int P, int KS, class Epilogue>
__device__ __forceinline__ void score_tiles_held(const Operand& w, const Operand& h, uint32_t token_tile, uint32_t first, uint32_t tile0, uint32_t tile1, int steps,
                                                 unsigned char* lds, Epilogue epilogue)
{
    constexpr int BYTES = operand_bytes<4>(), KK = step_of<P>() / 16, LOADS = 4;
    const int m0 = first_row<4>(), n0 = first_col<4>();
    const uint32_t lds0 = lds_address(lds);
    s16x8 held[KS][KK][P][2];
    {
        Loader<P, 4, true> load_h;
        load_h.start(h, token_tile * rows_of<4>(), 0);
        for (int s = 0; s < steps; ++s) load_h.fetch(lds0 + s * BYTES);
        stage_done();
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        held[s][kk][p][i] = s < steps ? fragment<P, 4, true>(lds + s * BYTES, p, n0 + 32 * i, kk) : s16x8{0, 0, 0, 0, 0, 0, 0, 0};
        stage_done();
    }
    f32x16 acc[2][2];
    clear(acc);
    const uint32_t total = tile1 > tile0 ? (tile1 - tile0) * steps : 0;
    Loader<P, 4, true> load_w;
    uint32_t row0 = first + tile0 * rows_of<4>(), next_row0 = row0, issued = 0, used = 0;
    int next_step = 0;
    auto issue = [&]() {
        if (issued == total) return;
        if (next_step == 0) load_w.start(w, next_row0, 0);
        load_w.fetch(lds0 + (issued & 3) * BYTES);
        ++issued;
        if (++next_step == steps) { next_step = 0; next_row0 += rows_of<4>(); }
    };
    // (writes may overtake loads: after some, all loads are waited for)
    auto wait = [&](bool wrote) {
        if (issued - used == 3 && !wrote) stage_done<2 * LOADS>();
        else stage_done();
    };
    issue();
    issue();
    issue();
    wait(false);
    while (used < total) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s >= steps) break;
            issue();
            const unsigned char* stage = lds + (used & 3) * BYTES;
            s16x8 a[2][P][2];
            auto read = [&](int kk) {
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < 2; ++i) a[kk & 1][p][i] = fragment<P, 4, true>(stage, p, m0 + 32 * i, kk);
            };
            read(0);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if (kk + 1 < KK) read(kk + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int im = 0; im < 2; ++im)
#pragma unroll
                    for (int in = 0; in < 2; ++in) {
                        acc[im][in] = mfma<P>(a[kk & 1][0][im], held[s][kk][0][in], acc[im][in]);
                        if (P == 2) {
                            acc[im][in] = mfma<P>(a[kk & 1][0][im], held[s][kk][P - 1][in], acc[im][in]);
                            acc[im][in] = mfma<P>(a[kk & 1][P - 1][im], held[s][kk][0][in], acc[im][in]);
                        }
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (s == steps - 1) {
                epilogue(row0, acc);
                clear(acc);
                row0 += rows_of<4>();
            }
            ++used;
            wait(s == steps - 1);
        }
    }
}

// Either: KS stages of H at most in registers, or none.
template <int P, int W, int KS, class Epilogue>
__device__ __forceinline__ void all_scores(const Operand& w, const Operand& h, uint32_t token_tile, uint32_t first, uint32_t tile0, uint32_t tile1, int steps,
                                           unsigned char* lds, Epilogue epilogue)
{
    if constexpr (KS > 0) score_tiles_held<P, KS>(w, h, token_tile, first, tile0, tile1, steps, lds, epilogue);
    else score_tiles<P, W>(w, h, token_tile, first, tile0, tile1, steps, lds, epilogue);
}

template <int PARTS>
__device__ __forceinline__ void split_bf16(const bf16_t (&x)[8], bf16x8 (&out)[PARTS])
{
#pragma unroll
    for (int q = 0; q < 8; ++q) out[0][q] = x[q];
}

template <int PARTS>
__device__ __forceinline__ void split_bf16(const float (&x)[8], bf16x8 (&out)[PARTS])
{
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        float rest = x[q];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            out[p][q] = static_cast<bf16_t>(rest);
            rest -= static_cast<float>(out[p][q]);
        }
    }
}

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// A lane has 4 values of 16 bits of rows 8 q + 4 (lane / 32) .. + 3 (a: of q, b: of q + 1): lanes l and l + 32 swap halves, so that
// l has the 8 of q and l + 32 the 8 of q + 1, side by side.
__device__ __forceinline__ u32x4 eight_of(u32x2 a, u32x2 b)
{
    const auto x = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false), y = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
    return u32x4{x[0], y[0], x[1], y[1]};
}

template <int P, int W, bool GROWS, Kind K>
__device__ __forceinline__ void product_tile(const Operand& cols, const Operand& g, uint32_t col0, uint32_t row0, uint32_t s0, uint32_t s1,
                                             unsigned char* lds, f32x16 (&acc)[W / 2][2])
{
    clear(acc);
    if (s0 >= s1) return;
    Loader<P, W, false> load_c;
    Loader<P, W, GROWS> load_g;
    load_c.start(cols, col0, s0);
    load_g.start(g, row0, s0);
    run_stages<W>(
        s1 - s0, lds,
        [&](uint32_t to) {
            load_c.fetch(to);
            load_g.fetch(to + operand_bytes<W>());
        },
        [&](const unsigned char* stage) { multiply<P, W, false, GROWS, K>(stage, acc); });
}

// Writes up to V values, the first `have` of them.
template <class T, int V>
__device__ __forceinline__ void store_some(T* to, int have, const float (&x)[V])
{
    if (have >= V) {
        store_vec<T, V>(to, x);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < have) to[e] = from_float<T>(x[e]);
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// Workgroups over table tiles for one tile of H, all with about as many tiles: as many as fill the machine once, or up to four times over where
// that ends sooner, and a workgroup's beginning counts as half a tile (bf16 losses of 38 400 rows against 20 000 of 128, 300 tiles of H for 512
// places: 460 us with one workgroup each, 298 with five).
uint32_t splits_of(int64_t row_tiles, int64_t token_tiles, bool large)
{
    const int64_t slots = slots_of(large);
    int64_t best = INT64_MAX, splits = 1;
    for (int64_t rounds = 1; rounds <= 4; ++rounds) {
        const int64_t most = std::max<int64_t>(1, std::min(row_tiles, rounds * slots / token_tiles)), per = ceil_div(row_tiles, most), s = ceil_div(row_tiles, per);
        const int64_t time = ceil_div(s * token_tiles, slots) * (2 * per + 1);
        if (time >= best) continue;
        best = time;
        splits = s;
    }
    return static_cast<uint32_t>(splits);
}

// Large tiles of scores: where a tile's products take longer than its exponentials, which nothing else runs beside there, and where there are
// enough of them to fill the machine several times over (bf16, 2048 rows against 100 000 of 512: 218 us, 231 with small tiles; of 256: 122 and
// 117).  Halves take three products per fetch, which small tiles keep up with (4096 x 50 000 x 512: 657 us, large tiles 674).
bool large_scores(int64_t n, int64_t num_rows, int32_t dim, int parts)
{
    return parts == 1 && dim >= 384 && ceil_div(n, 256) * ceil_div(num_rows, 256) >= 1024;
}

// LDS of the rows of H that a launch of the few-rows kernels has, as second operands.
int64_t few_bytes_of(int blocks, int32_t dim, int parts) { return blocks * ceil_div(dim, 32) * (parts == 2 ? 3 : 1) * 1024; }

// Whether the table streams through registers for scores (blocks of 16 rows of H of a launch, or 0): up to 64 rows, or in fp32, where the other way
// makes halves of the table first, two launches of as many rows as LDS has place for, three where the table is no small part of the last-level cache
// (us of the loss at 200 003 x 256 fp32: 64 rows 55, 128 rows 107, 192 rows 169, the other way 178, 182 and 212; 192 rows against 100 000 x 100: 76 and 63).
int few_blocks_of(int64_t n, int64_t num_rows, int32_t dim, int parts)
{
    const int64_t launches = parts == 1 ? 1 : num_rows * dim < (1 << 25) ? 2 : 3;
    int blocks = n <= 16 ? 1 : n <= 32 ? 2 : 4;
    while (blocks > 1 && few_bytes_of(blocks, dim, parts) > kFewBytesAlone) blocks /= 2;
    return few_bytes_of(blocks, dim, parts) <= kFewBytesAlone && ceil_div(n, 16 * blocks) <= launches ? blocks : 0;
}

// Packed operands in a workspace.
struct Packs {
    int32_t parts, padded, cols;
    int64_t tokens;                    // padded n
    bool large_scores;                 // tiles of 256 x 256
    float* amax;
    int32_t* shift;                    // of W, H, c H
    uint16_t *h[2], *hc[2], *w[2];
};

// Stages of H that the scores' wavefronts hold in registers: 2, 4, or 0 for H through LDS like the table: where there are more, with large
// tiles, and where a workgroup has so few tiles that fetching H ahead of them does not pay.
int held_stages(const Packs& w, uint32_t row_tiles, uint32_t splits, int steps)
{
    if (w.large_scores || steps > 4 || ceil_div(row_tiles, splits) < 3) return 0;
    return steps > 2 ? 4 : 2;
}

struct SoftmaxCall {
    const void *h, *w;
    int64_t h_stride, w_stride, n, num_rows;
    int32_t dim, type;
    const int32_t* targets;
    const float* c;
};

// Whether a bf16 table is read as it lies, or has to be packed first.
bool usable_as_it_lies(const SoftmaxCall& x)
{
    return x.type == NE_BF16 && x.dim % 8 == 0 && x.w_stride % 8 == 0 && x.w_stride < kMostStride && aligned(x.w, 16);
}

Operand packed_operand(uint16_t* const* part, int64_t rows, int32_t padded)
{
    return Operand{{part[0], part[1]}, padded, static_cast<uint32_t>(rows - 1), static_cast<uint32_t>(padded)};
}

// Workgroups of `threads` that pack `rows` rows: of a row's lanes, as in the kernel, four rows of a lane group in flight.
uint32_t pack_blocks(const Packs& w, int64_t rows, int threads, int64_t most)
{
    int lanes = 1;
    while (lanes < 64 && 8 * lanes < w.padded) lanes *= 2;
    return static_cast<uint32_t>(std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, 4 * (threads / lanes)), most)));
}

// Packs H and, where it cannot be used as it is, W.  With dw, c H for its product, too: in fp32 its halves, if there are factors; in bf16 it is to be
// fp16, which `later` says how, as its largest magnitude is found here.  table_max (bf16; NULL, or kMostPack numbers) receives `maxima` largest magnitudes of W.
hipError_t pack(const SoftmaxCall& x, const Packs& w, bool dw, Operand* h, Operand* hc, Operand* wo, PackArgs* later, float* table_max, int32_t* maxima, hipStream_t st)
{
    const bool direct = usable_as_it_lies(x);
    const bool f32 = x.type == NE_F32;
    if (f32) {
        AmaxArgs a{static_cast<const float*>(x.h), static_cast<const float*>(x.w), x.targets, x.c, x.h_stride, x.w_stride, x.n, x.num_rows, x.dim, w.amax};
        hipLaunchKernelGGL(amax_kernel, dim3(kAmaxBlocks), dim3(kThreads), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    PackJobs jobs{};
    int count = 0;
    int64_t most = 0;
    auto add = [&](const void* in, int64_t stride, int64_t rows, int64_t padded_rows, const int32_t* targets, const float* c, uint16_t* const* out, int which) {
        PackArgs& a = jobs.job[count++];
        a.in = in; a.in_stride = stride; a.rows = rows; a.padded_rows = padded_rows; a.targets = targets;
        a.num_targets = static_cast<uint32_t>(x.num_rows); a.c = c; a.dim = x.dim; a.padded = w.padded;
        a.out[0] = out[0]; a.out[1] = out[1]; a.shift = w.shift + which;
        if (f32) { a.amax = w.amax + which * kAmaxBlocks; a.maxima = kAmaxBlocks; }
        most = std::max(most, padded_rows);
    };
    auto operand = [&](uint16_t* const* part, int64_t rows) { return packed_operand(part, rows, w.padded); };
    add(x.h, x.h_stride, x.n, w.tokens, x.targets, nullptr, w.h, 1);
    *h = operand(w.h, w.tokens);
    *hc = *h;
    if (dw && f32 && x.c) add(x.h, x.h_stride, x.n, w.tokens, x.targets, x.c, w.hc, 2);
    if (dw && (!f32 || x.c)) *hc = operand(w.hc, w.tokens);
    *wo = operand(w.w, x.num_rows);
    if (direct) {
        wo->part[0] = static_cast<const uint16_t*>(x.w);
        wo->stride = x.w_stride;
        wo->width = static_cast<uint32_t>(x.dim);
    } else {
        add(x.w, x.w_stride, x.num_rows, x.num_rows, nullptr, nullptr, w.w, 0);
    }
    if (table_max) {
        uint16_t* const none[2] = {};
        if (direct) add(x.w, x.w_stride, x.num_rows, x.num_rows, nullptr, nullptr, none, 0);
        jobs.job[count - 1].amax_out = table_max;
    }
    const dim3 grid(pack_blocks(w, most, kThreads, kMostPack), static_cast<unsigned>(count));
    if (table_max) *maxima = static_cast<int32_t>(grid.x);
    if (dw && !f32) {
        *later = jobs.job[0];
        later->c = jobs.job[0].c = x.c;
        jobs.job[0].amax_out = w.amax;
        later->amax = w.amax; later->maxima = static_cast<int32_t>(grid.x);
        later->out[0] = w.hc[0]; later->shift = w.shift + (x.c ? 2 : 1);
    }
    if (w.parts == 1) hipLaunchKernelGGL(pack_kernel<1>, grid, dim3(kThreads), 0, st, jobs);
    else hipLaunchKernelGGL(pack_kernel<2>, grid, dim3(kThreads), 0, st, jobs);
    return hipGetLastError();
}

}  // namespace
