// Rows of bf16 or fp32 values in 16-byte vectors, for the kernels that are bound by memory (norms, embedding, optimizer).
//
// A row may begin at any multiple of its value's size: an odd row length puts most rows off the 16-byte grid.  The vector loads and
// stores below promise the compiler no more than a value's alignment; gfx950 serves them as one 16-byte access all the same, so rows of
// any length take the same code, and only the last vector of a row is done value by value.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sbn.h"

namespace sbn {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_by2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));

// two fp32 values rounded to the nearest bf16, ties to even; the first in the low half
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}
__device__ __forceinline__ float bf16_low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float bf16_high(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

template <sbn_dtype DT> struct Row;

template <> struct Row<SBN_BF16> {
    static constexpr int E = 8;   // values of a vector
    typedef uint16_t value;
    static __device__ __forceinline__ float number(value x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ value rounded(float f) { return (value)bf16_pair(f, 0.0f); }
    static __device__ __forceinline__ value get(u32x4 v, int k) { return (value)(v[k / 2] >> (16 * (k % 2))); }
    static __device__ __forceinline__ void set(u32x4 &v, int k, value x) { v[k / 2] |= (uint32_t)x << (16 * (k % 2)); }   // of a value that is zero
    static __device__ __forceinline__ void clear(u32x4 &v, int k) { v[k / 2] &= k % 2 ? 0xffffu : 0xffff0000u; }
    template <bool ONCE = false> static __device__ __forceinline__ u32x4 load(const void *row, int64_t vec)
    {
        const u32x4_by2 *p = reinterpret_cast<const u32x4_by2 *>(static_cast<const value *>(row) + vec * E);
        return ONCE ? __builtin_nontemporal_load(p) : *p;
    }
    template <bool ONCE = false> static __device__ __forceinline__ void store(void *row, int64_t vec, u32x4 v)
    {
        u32x4_by2 *p = reinterpret_cast<u32x4_by2 *>(static_cast<value *>(row) + vec * E);
        if (ONCE)
            __builtin_nontemporal_store(v, p);
        else
            *p = v;
    }
    // the last vector, of which `n` values are the row's; the others come as zeros and are not written
    static __device__ __forceinline__ u32x4 load_part(const void *row, int64_t vec, int n)
    {
        u32x4 v = {0, 0, 0, 0};
        const value *p = static_cast<const value *>(row) + vec * E;
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) set(v, k, p[k]);
        return v;
    }
    static __device__ __forceinline__ void store_part(void *row, int64_t vec, int n, u32x4 v)
    {
        value *p = static_cast<value *>(row) + vec * E;
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) p[k] = get(v, k);
    }
    static __device__ __forceinline__ void unpack(u32x4 v, float (&f)[E])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = bf16_low(v[k]);
            f[2 * k + 1] = bf16_high(v[k]);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[E])
    {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = bf16_pair(f[2 * k], f[2 * k + 1]);
        return v;
    }
};

template <> struct Row<SBN_F32> {
    static constexpr int E = 4;
    typedef float value;
    static __device__ __forceinline__ float number(value x) { return x; }
    static __device__ __forceinline__ value rounded(float f) { return f; }
    static __device__ __forceinline__ value get(u32x4 v, int k) { return __uint_as_float(v[k]); }
    static __device__ __forceinline__ void set(u32x4 &v, int k, value x) { v[k] = __float_as_uint(x); }
    static __device__ __forceinline__ void clear(u32x4 &v, int k) { v[k] = 0; }
    template <bool ONCE = false> static __device__ __forceinline__ u32x4 load(const void *row, int64_t vec)
    {
        const u32x4_by4 *p = reinterpret_cast<const u32x4_by4 *>(static_cast<const value *>(row) + vec * E);
        return ONCE ? __builtin_nontemporal_load(p) : *p;
    }
    template <bool ONCE = false> static __device__ __forceinline__ void store(void *row, int64_t vec, u32x4 v)
    {
        u32x4_by4 *p = reinterpret_cast<u32x4_by4 *>(static_cast<value *>(row) + vec * E);
        if (ONCE)
            __builtin_nontemporal_store(v, p);
        else
            *p = v;
    }
    static __device__ __forceinline__ u32x4 load_part(const void *row, int64_t vec, int n)
    {
        u32x4 v = {0, 0, 0, 0};
        const value *p = static_cast<const value *>(row) + vec * E;
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) set(v, k, p[k]);
        return v;
    }
    static __device__ __forceinline__ void store_part(void *row, int64_t vec, int n, u32x4 v)
    {
        value *p = static_cast<value *>(row) + vec * E;
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) p[k] = get(v, k);
    }
    static __device__ __forceinline__ void unpack(u32x4 v, float (&f)[E])
    {
#pragma unroll
        for (int k = 0; k < E; ++k) f[k] = __uint_as_float(v[k]);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[E])
    {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = __float_as_uint(f[k]);
        return v;
    }
};

// vector `vec` of a row of d values; zeros behind its end.  ONCE: nobody will read it again soon (a nontemporal load)
template <sbn_dtype DT, bool ONCE = false> __device__ __forceinline__ u32x4 load_vec(const void *row, int64_t vec, int64_t d)
{
    const int64_t left = d - vec * Row<DT>::E;
    if (left >= Row<DT>::E) return Row<DT>::template load<ONCE>(row, vec);
    if (left > 0) return Row<DT>::load_part(row, vec, (int)left);
    return (u32x4){0, 0, 0, 0};
}
template <sbn_dtype DT> __device__ __forceinline__ void store_vec(void *row, int64_t vec, int64_t d, u32x4 v)
{
    const int64_t left = d - vec * Row<DT>::E;
    if (left >= Row<DT>::E)
        Row<DT>::store(row, vec, v);
    else if (left > 0)
        Row<DT>::store_part(row, vec, (int)left, v);
}

// U values at U * unit of a row, a whole number of vectors: what one thread has of rows of two types
template <sbn_dtype DT, int U> __device__ __forceinline__ void load_unit(const void *row, int64_t unit, int64_t d, float (&f)[U])
{
    constexpr int E = Row<DT>::E;
#pragma unroll
    for (int j = 0; j < U / E; ++j) {
        float part[E];
        Row<DT>::unpack(load_vec<DT>(row, unit * (U / E) + j, d), part);
#pragma unroll
        for (int k = 0; k < E; ++k) f[j * E + k] = part[k];
    }
}
template <sbn_dtype DT, int U> __device__ __forceinline__ void store_unit(void *row, int64_t unit, int64_t d, const float (&f)[U])
{
    constexpr int E = Row<DT>::E;
#pragma unroll
    for (int j = 0; j < U / E; ++j) {
        float part[E];
#pragma unroll
        for (int k = 0; k < E; ++k) part[k] = f[j * E + k];
        store_vec<DT>(row, unit * (U / E) + j, d, Row<DT>::pack(part));
    }
}
constexpr int unit_of(sbn_dtype a, sbn_dtype b) { return a == SBN_F32 && b == SBN_F32 ? 4 : 8; }

// fp32 values at `first`, those behind d as `none`
template <int E> __device__ __forceinline__ void load_floats(const float *p, int64_t first, int64_t d, float none, float (&f)[E])
{
    if (first + E <= d) {
#pragma unroll
        for (int k = 0; k < E; k += 4) {
            const f32x4_by4 v = *reinterpret_cast<const f32x4_by4 *>(p + first + k);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[k + j] = v[j];
        }
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k) f[k] = first + k < d ? p[first + k] : none;
    }
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

}  // namespace sbn
