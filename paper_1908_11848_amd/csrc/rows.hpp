// Vectors of a row of fp32 or bf16 numbers, as fp32 (internal).  16 bytes a lane and access; rows need not be aligned for it (gfx950 takes 16-byte
// accesses at any address of the element's own alignment), and the last, partial vector of a row is moved element by element.
#pragma once
#include "common.hpp"

// The most workgroups of so many threads that a launch takes: one of 2^32 threads or more in a dimension is cut short without an error.
inline long most_blocks(int threads) { return (1L << 31) / threads; }

namespace rows {

typedef __bf16 bf16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));

template <class T> constexpr int VEC = 16 / sizeof(T);

template <class T> __device__ __forceinline__ void load(const T* p, float* v) {
    if constexpr (sizeof(T) == 4) {
        const floatx4 u = *reinterpret_cast<const float4u*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = u[e];
    } else {
        const bf16x8 u = *reinterpret_cast<const bf16x8u*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)u[e];
    }
}
// n of a vector's elements are in the row; the others read as zero
template <class T> __device__ __forceinline__ void load(const T* p, int n, float* v) {
    if (n >= VEC<T>) { load(p, v); return; }
#pragma unroll
    for (int e = 0; e < VEC<T>; ++e) v[e] = e < n ? (float)p[e] : 0.f;
}
// Results of more than half of the last cache are written past the caches: what is next to read them finds nothing of them there anyway, and what the kernel reads
// stays.  A block's forward pass (layer norm, product with GELU, product with residual; bf16, the hidden layer's results of 128 to 224 MB read by the next product) takes 295, 432, 501 and 561 us so and
// 338, 449, 518 and 585 with the caches up to 256 MB, its backward pass 646, 808, 930 and 1068 and 658, 819, 945 and 1078; of eight such blocks none was slower.  Smaller results are read again
// from there (a step of a network of width 512, 8192 rows, fp32: 1450 us, 1535 past the caches).
inline bool past_the_caches(int64_t bytes) { return bytes >= 128LL << 20; }
// (The empty statements keep the compiler from making one store of the two branches, which would then be an ordinary one.)
// Not a template over the vector: that would drop the alignment of its elements from the type.
__device__ __forceinline__ void store_past(float4u* p, const floatx4& v) {
    asm volatile("");
    __builtin_nontemporal_store(v, p);
    asm volatile("");
}
__device__ __forceinline__ void store_past(bf16x8u* p, const bf16x8& v) {
    asm volatile("");
    __builtin_nontemporal_store(v, p);
    asm volatile("");
}
template <class T> __device__ __forceinline__ void store(T* p, int n, const float* v, bool past = false) {
    if (n >= VEC<T>) {
        if constexpr (sizeof(T) == 4) {
            floatx4 u;
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = v[e];
            if (past) store_past(reinterpret_cast<float4u*>(p), u);
            else *reinterpret_cast<float4u*>(p) = u;
        } else {
            bf16x8 u;
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = (bf16)v[e];
            if (past) store_past(reinterpret_cast<bf16x8u*>(p), u);
            else *reinterpret_cast<bf16x8u*>(p) = u;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < VEC<T>; ++e)
        if (e < n) p[e] = (T)v[e];
}

// a vector as it is in memory, and its elements
template <class T> __device__ __forceinline__ uint4 fetch(const T* p, int n) {
    uint4 r;
    if (n >= VEC<T>) {
        __builtin_memcpy(&r, __builtin_assume_aligned(p, sizeof(T)), sizeof r);
        return r;
    }
    T v[VEC<T>];
#pragma unroll
    for (int e = 0; e < VEC<T>; ++e) v[e] = e < n ? p[e] : (T)0.f;
    return __builtin_bit_cast(uint4, v);
}
template <class T> __device__ __forceinline__ void convert(const uint4& r, float* v) {
    struct V { T e[VEC<T>]; };
    const V u = __builtin_bit_cast(V, r);
#pragma unroll
    for (int e = 0; e < VEC<T>; ++e) v[e] = (float)u.e[e];
}

// eight elements, n of them in the row
template <class T> __device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
    load(p, n, v);
    if constexpr (VEC<T> == 4) load(p + 4, n - 4, v + 4);
}
template <class T> __device__ __forceinline__ void store8(T* p, int n, const float (&v)[8], bool past = false) {
    store(p, n, v, past);
    if constexpr (VEC<T> == 4) store(p + 4, n - 4, v + 4, past);
}

// eight elements as they are in memory
template <class T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
template <class T> __device__ __forceinline__ Raw8<T> fetch8(const T* p, int n) {
    Raw8<T> r;
    if (n >= 8) {
        __builtin_memcpy(&r, __builtin_assume_aligned(p, sizeof(T)), sizeof r);
    } else {
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : (T)0.f;
        r = __builtin_bit_cast(Raw8<T>, v);
    }
    return r;
}
template <class T> __device__ __forceinline__ void convert8(const Raw8<T>& r, float (&v)[8]) {
    struct E { T e[8]; };
    const E u = __builtin_bit_cast(E, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)u.e[e];
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

}  // namespace rows
