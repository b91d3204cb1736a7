// Elements of rows of vectors (fp32, bf16, f16) as vectors of a few bytes, and the widths that rows allow.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "avq_internal.h"

namespace avq {

struct bf16_t { uint16_t bits; };
struct f16_t { uint16_t bits; };

template <class T> struct TypeOf;
template <> struct TypeOf<float> { static constexpr int id = AVQ_F32; };
template <> struct TypeOf<bf16_t> { static constexpr int id = AVQ_BF16; };
template <> struct TypeOf<f16_t> { static constexpr int id = AVQ_F16; };

__host__ inline int type_bytes(int type) { return type == AVQ_F32 ? 4 : 2; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __uint_as_float((uint32_t)v.bits << 16); }
__device__ __forceinline__ float to_f32(f16_t v) { return (float)__builtin_bit_cast(_Float16, v.bits); }

// to nearest, ties to even; NaN stays NaN
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v)
{
    return bf16_t{__builtin_bit_cast(uint16_t, (__bf16)v)};
}
template <> __device__ __forceinline__ f16_t from_f32<f16_t>(float v) { return f16_t{__builtin_bit_cast(uint16_t, (_Float16)v)}; }

// V elements that are loaded and stored at once (V * sizeof(T) = 16, 8, 4 or 2 bytes).
template <class T, int V> struct alignas(sizeof(T) * V) Pack { T e[V]; };

// Bytes that every row of rows at `p`, `ld` elements apart and `d` long, can be read in at once: 16, 8 or one element.
inline int row_width(const void *p, int64_t ld, int64_t d, int size)
{
    for (int w = 16; w > 4; w /= 2)
        if (((uintptr_t)p % w) == 0 && (ld * size) % w == 0 && (d * size) % w == 0) return w;
    return size;
}

// sum over the L lanes (a power of two, at most 64) of an aligned group, in a fixed order; every lane gets it
template <int L> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int m = 1; m < L; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

// q = i / by for i * by < 2^32: q = (i * magic) >> 32
__host__ __device__ inline uint32_t magic_of(uint32_t by) { return by <= 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + by - 1) / by); }
__device__ __forceinline__ uint32_t magic_div(uint32_t i, uint32_t magic) { return magic == 0 ? i : __umulhi(i, magic); }

} // namespace avq
