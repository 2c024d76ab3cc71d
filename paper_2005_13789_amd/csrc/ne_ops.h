// What the operators of full-softmax training share: their types, wide loads and stores, workspace carving.
#pragma once
#include "ne_internal.h"

namespace {

typedef __bf16 bf16_t;

inline bool type_ok(int32_t t) { return t == NE_F32 || t == NE_BF16; }
inline size_t type_bytes(int32_t t) { return t == NE_F32 ? 4 : 2; }

// Places of a workspace's parts, each at a multiple of 256 bytes; with base == nullptr only their total size.
struct Carver {
    char* base;
    size_t off = 0;
    template <class T>
    T* get(size_t count)
    {
        char* p = base ? base + off : nullptr;
        off += (count * sizeof(T) + 255) & ~static_cast<size_t>(255);
        return reinterpret_cast<T*>(p);
    }
    size_t total() const { return off; }
};

template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t from_float<bf16_t>(float x) { return static_cast<bf16_t>(x); }

// Elements of the widest access that both types make in 16 bytes at most.
template <class A, class B> constexpr int vec_of() { return sizeof(A) == 2 && sizeof(B) == 2 ? 8 : 4; }

// V elements as floats, from and to an address that is aligned to one element: one wide access (the hardware takes any
// alignment of dwords and of halves; rows of odd length are not aligned to more).
template <class T, int V>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[V])
{
    typedef T vec __attribute__((ext_vector_type(V)));
    vec v;
    __builtin_memcpy(&v, p, sizeof(T) * V);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = static_cast<float>(v[e]);
}

template <class T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[V])
{
    typedef T vec __attribute__((ext_vector_type(V)));
    vec v;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = from_float<T>(x[e]);
    __builtin_memcpy(p, &v, sizeof(T) * V);
}

}  // namespace
