// AdamW over many tensors at once, states in 32 or in 8 bits: ne_create_adamw, ne_adamw_step.
//
// One launch per step.  Work is cut into units of 16 blocks of 256 elements that never straddle two tensors; a map
// {tensor, unit of the tensor} in the workspace, made when the handle is created, tells a workgroup its unit, so that
// thousands of small tensors cost no more than their elements.  A wavefront has one block of 256 at a time (four
// consecutive elements per lane), which is also the block that shares a scale with 8-bit states: its largest
// magnitude is a reduction inside the wavefront, and the new states are quantised from registers.
//
// Bound by memory: 28 bytes an element with 32-bit states and fp32 gradients (two tensors of 128 million: 1.34 ms, 5.35 TB/s,
// where a copy makes 4.75); with 8-bit states 16 bytes, or 14 and 2 for the copy with gradients and a copy in bf16 (64 tensors
// of 18.8 million elements in all: 68 us, 4.4 TB/s).  16 blocks a workgroup: one wavefront's four keep loads of a block ahead of
// another's arithmetic without many workgroups that only read their unit.
// Every operation is rounded by itself (no fused multiply-adds): the result is that of the formula taken step by step
// in fp32, and 8-bit states are the same bit for bit whoever computes them.
#include <memory>

#include "ne_internal.h"
#include "ne_ops.h"

#pragma clang fp contract(off)

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;                    // elements that share a scale
constexpr int kUnitBlocks = 16;                // blocks of a workgroup
constexpr int kUnit = kBlock * kUnitBlocks;
constexpr int kMostTensors = 65536;
enum : uint32_t { kStreamRound = 3 };
constexpr float kTopE4m3 = 448.0f;             // the largest value of e4m3

struct StepArgs {
    const ne_adamw_tensor* tensors;
    const uint2* units;
    uint64_t step;
    uint32_t k0, k1;
    float lr, b1, b2, c1, c2, size, root, eps, grad_scale;
};

// a >= 0, at most 448, as the e4m3 value below or above it: the upper one with probability (r16 + its fraction's bits) as
// if r16 / 65536 of a last place were added before the excess bits are cut.  Below 2^-6 the values are multiples of 2^-9.
__device__ __forceinline__ float e4m3_at_random(float a, uint32_t r16, bool keep)
{
    const float big = __uint_as_float((__float_as_uint(a) + (r16 << 4)) & 0xFFF00000u);
    float small = floorf(a * 512.0f + static_cast<float>(r16) * 0x1p-16f);
    if (keep && a > 0.0f) small = fmaxf(small, 1.0f);
    return a < 0x1p-6f ? small * 0x1p-9f : big;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o, 64)));
    return v;
}

// The block's new states from x (m or sqrt(v)): packed e4m3, and the block's scale.  A NaN is the largest of all bit
// patterns of magnitudes: it becomes the scale, and the whole block NaN.
__device__ __forceinline__ uint32_t quantise(const float (&x)[4], const uint32_t (&r16)[4], bool keep, float* scale)
{
    uint32_t top_bits = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top_bits = max(top_bits, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    top_bits = max(wave_max(top_bits), __float_as_uint(0x1p-100f));
    const float top = __uint_as_float(top_bits);
    const float to = (1.0f / top) * kTopE4m3;
    *scale = top * (1.0f / kTopE4m3);
    float q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float y = x[e] * to;
        q[e] = copysignf(e4m3_at_random(fminf(fabsf(y), kTopE4m3), r16[e], keep), y);
    }
    int packed = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);      // (exact: the values are e4m3 values)
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], packed, true));
}

__device__ __forceinline__ void dequantise(uint32_t packed, float scale, float (&x)[4])
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(packed), false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(packed), true);
    x[0] = lo[0] * scale; x[1] = lo[1] * scale; x[2] = hi[0] * scale; x[3] = hi[1] * scale;
}

template <class T>
__device__ __forceinline__ void load4(const T* p, int have, float (&x)[4])
{
    if (have == 4) {
        load_vec<T, 4>(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = e < have ? static_cast<float>(p[e]) : 0.0f;
    }
}

template <class T>
__device__ __forceinline__ void store4(T* p, int have, const float (&x)[4])
{
    if (have == 4) {
        store_vec<T, 4>(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) p[e] = from_float<T>(x[e]);
    }
}

__device__ __forceinline__ uint32_t load4_bytes(const uint8_t* p, int have)
{
    uint32_t v = 0;
    if (have == 4) {
        __builtin_memcpy(&v, p, 4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) v |= static_cast<uint32_t>(p[e]) << (8 * e);
    }
    return v;
}

__device__ __forceinline__ void store4_bytes(uint8_t* p, int have, uint32_t v)
{
    if (have == 4) {
        __builtin_memcpy(p, &v, 4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) p[e] = static_cast<uint8_t>(v >> (8 * e));
    }
}

template <bool EIGHT>
__global__ void __launch_bounds__(kThreads) adamw_kernel(StepArgs a)
{
    const uint2 unit = a.units[blockIdx.x];
    const ne_adamw_tensor t = a.tensors[unit.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float kept = 1.0f - t.weight_decay * a.lr;
    for (int b = wave; b < kUnitBlocks; b += kThreads / 64) {
        const int64_t block = static_cast<int64_t>(unit.y) * kUnitBlocks + b;
        const int64_t at = block * kBlock + lane * 4;
        if (block * kBlock >= t.n) break;
        const int have = static_cast<int>(min(max(t.n - at, static_cast<int64_t>(0)), static_cast<int64_t>(4)));
        float p[4], g[4], m[4], v[4];
        load4(t.param + at, have, p);
        if (t.grad_type == NE_F32) load4(static_cast<const float*>(t.grad) + at, have, g);
        else load4(static_cast<const bf16_t*>(t.grad) + at, have, g);
        if (EIGHT) {
            dequantise(load4_bytes(static_cast<const uint8_t*>(t.m) + at, have), t.m_scale[block], m);
            dequantise(load4_bytes(static_cast<const uint8_t*>(t.v) + at, have), t.v_scale[block], v);
        } else {
            load4(static_cast<const float*>(t.m) + at, have, m);
            load4(static_cast<const float*>(t.v) + at, have, v);
        }
        float r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ge = g[e] * a.grad_scale;
            if (EIGHT) v[e] = v[e] * v[e];
            m[e] = m[e] * a.b1 + ge * a.c1;
            v[e] = v[e] * a.b2 + (ge * ge) * a.c2;
            r[e] = sqrtf(v[e]);
            p[e] = p[e] * kept - (m[e] / (r[e] * a.root + a.eps)) * a.size;
        }
        store4(t.param + at, have, p);
        if (t.param_bf16) store4(static_cast<bf16_t*>(t.param_bf16) + at, have, p);
        if (EIGHT) {
            const uint4 w = philox4x32_10(make_uint4(static_cast<uint32_t>(at >> 2), unit.x, static_cast<uint32_t>(a.step), kStreamRound), a.k0, a.k1);
            const uint32_t lo[4] = {w.x & 0xFFFFu, w.y & 0xFFFFu, w.z & 0xFFFFu, w.w & 0xFFFFu};
            const uint32_t hi[4] = {w.x >> 16, w.y >> 16, w.z >> 16, w.w >> 16};
            float ms, vs;
            const uint32_t mq = quantise(m, lo, false, &ms), vq = quantise(r, hi, true, &vs);
            store4_bytes(static_cast<uint8_t*>(t.m) + at, have, mq);
            store4_bytes(static_cast<uint8_t*>(t.v) + at, have, vq);
            if (lane == 0) {
                t.m_scale[block] = ms;
                t.v_scale[block] = vs;
            }
        } else {
            store4(static_cast<float*>(t.m) + at, have, m);
            store4(static_cast<float*>(t.v) + at, have, v);
        }
    }
}

struct AdamwWs {
    ne_adamw_tensor* tensors;
    uint2* units;
    size_t total;
};

// Units of all tensors, or -1 where a tensor has no sensible size.
int64_t count_units(const ne_adamw_tensor* t, int64_t n)
{
    int64_t units = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (t[i].n <= 0 || t[i].n >= (1ll << 33)) return -1;
        units += (t[i].n + kUnit - 1) / kUnit;
    }
    return units < (1ll << 31) ? units : -1;
}

AdamwWs adamw_layout(int64_t tensors, int64_t units, char* base)
{
    Carver take{base};
    AdamwWs w{};
    w.tensors = take.get<ne_adamw_tensor>(static_cast<size_t>(tensors));
    w.units = take.get<uint2>(static_cast<size_t>(units));
    w.total = take.total();
    return w;
}

}  // namespace

struct ne_adamw {
    AdamwWs ws;
    int64_t units;
    int32_t state_bits;
    uint64_t seed;
};

extern "C" {

size_t ne_adamw_workspace_bytes(const ne_adamw_tensor* tensors_host, int64_t n_tensors)
{
    if (!tensors_host || n_tensors < 1 || n_tensors > kMostTensors) return 0;
    const int64_t units = count_units(tensors_host, n_tensors);
    return units < 0 ? 0 : adamw_layout(n_tensors, units, nullptr).total;
}

ne_status ne_create_adamw(ne_adamw** out, const ne_adamw_tensor* tensors_host, int64_t n_tensors, int32_t state_bits,
                          uint64_t seed, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    if (!out) return fail(NE_ERR_ARG, "ne_create_adamw: out is NULL");
    *out = nullptr;
    if (!tensors_host || n_tensors < 1 || n_tensors > kMostTensors) return fail(NE_ERR_ARG, "ne_create_adamw: tensors_host is NULL or n_tensors outside [1, 65536]");
    if (state_bits != 8 && state_bits != 32) return fail(NE_ERR_ARG, "ne_create_adamw: state_bits is neither 8 nor 32");
    const size_t state = state_bits == 32 ? 4 : 1;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const ne_adamw_tensor& t = tensors_host[i];
        const char* why = nullptr;
        if (t.n <= 0 || t.n >= (1ll << 33)) why = "n outside [1, 2^33)";
        else if (!type_ok(t.grad_type)) why = "grad_type is neither NE_F32 nor NE_BF16";
        else if (!t.param || !aligned(t.param, 4)) why = "param is NULL or misaligned";
        else if (!t.grad || !aligned(t.grad, type_bytes(t.grad_type))) why = "grad is NULL or misaligned";
        else if (!t.m || !t.v || !aligned(t.m, state) || !aligned(t.v, state)) why = "m or v is NULL or misaligned";
        else if (state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))) why = "a scale is NULL or misaligned";
        else if (t.param_bf16 && !aligned(t.param_bf16, 2)) why = "param_bf16 is misaligned";
        else if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.0f) why = "weight_decay is negative or not finite";
        if (why) return fail(NE_ERR_ARG, "ne_create_adamw: tensor " + std::to_string(i) + ": " + why);
    }
    const int64_t units = count_units(tensors_host, n_tensors);
    if (units < 0) return fail(NE_ERR_ARG, "ne_create_adamw: too many elements");
    const AdamwWs w = adamw_layout(n_tensors, units, static_cast<char*>(workspace_dev));
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < w.total)
        return fail(NE_ERR_ARG, "ne_create_adamw: workspace_dev is NULL, not 256-byte aligned, or smaller than ne_adamw_workspace_bytes()");
    std::unique_ptr<uint2[]> map(new (std::nothrow) uint2[static_cast<size_t>(units)]);
    std::unique_ptr<ne_adamw> opt(new (std::nothrow) ne_adamw);
    if (!map || !opt) return fail(NE_ERR_NOMEM, "ne_create_adamw: host allocation failed");
    int64_t k = 0;
    for (int64_t i = 0; i < n_tensors; ++i)
        for (int64_t u = 0; u * kUnit < tensors_host[i].n; ++u) map[k++] = make_uint2(static_cast<uint32_t>(i), static_cast<uint32_t>(u));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    NE_HIP_CHECK(hipMemcpyAsync(w.tensors, tensors_host, sizeof(ne_adamw_tensor) * static_cast<size_t>(n_tensors), hipMemcpyHostToDevice, st));
    NE_HIP_CHECK(hipMemcpyAsync(w.units, map.get(), sizeof(uint2) * static_cast<size_t>(units), hipMemcpyHostToDevice, st));
    NE_HIP_CHECK(hipStreamSynchronize(st));
    *opt = ne_adamw{w, units, state_bits, seed};
    *out = opt.release();
    return NE_OK;
}

ne_status ne_adamw_step(ne_adamw* opt, int64_t step, float lr, float beta1, float beta2, float eps, float grad_scale, void* hip_stream)
{
    if (!opt) return fail(NE_ERR_ARG, "ne_adamw_step: handle is NULL");
    if (step < 1 || step >= (1ll << 32)) return fail(NE_ERR_ARG, "ne_adamw_step: step outside [1, 2^32)");
    if (!std::isfinite(lr) || lr < 0.0f || !std::isfinite(grad_scale) || !std::isfinite(eps) || eps < 0.0f)
        return fail(NE_ERR_ARG, "ne_adamw_step: lr, eps or grad_scale is not finite, or lr or eps negative");
    if (!(beta1 >= 0.0f && beta1 < 1.0f && beta2 >= 0.0f && beta2 < 1.0f)) return fail(NE_ERR_ARG, "ne_adamw_step: a beta is outside [0, 1)");
    StepArgs a{};
    a.tensors = opt->ws.tensors; a.units = opt->ws.units; a.step = static_cast<uint64_t>(step);
    a.k0 = static_cast<uint32_t>(opt->seed); a.k1 = static_cast<uint32_t>(opt->seed >> 32);
    const double t = static_cast<double>(step), b1 = beta1, b2 = beta2;
    a.lr = lr; a.b1 = beta1; a.b2 = beta2; a.c1 = static_cast<float>(1.0 - b1); a.c2 = static_cast<float>(1.0 - b2);
    a.size = static_cast<float>(static_cast<double>(lr) / (1.0 - std::pow(b1, t)));
    a.root = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(b2, t)));
    a.eps = eps; a.grad_scale = grad_scale;
    const dim3 grid(static_cast<unsigned>(opt->units));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (opt->state_bits == 8) hipLaunchKernelGGL(adamw_kernel<true>, grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(adamw_kernel<false>, grid, dim3(kThreads), 0, st, a);
    NE_HIP_CHECK(hipGetLastError());
    return NE_OK;
}

void ne_destroy_adamw(ne_adamw* opt) { delete opt; }

}  // extern "C"
