// Elements of rows of vectors (fp32, bf16, f16) as vectors of a few bytes, and the widths that rows allow.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// 16 bytes of a row: what a lane loads and stores at once.
template <class T> constexpr int kUnit = 16 / (int)sizeof(T);
template <class T> using Unit = Pack<T, kUnit<T>>;
template <class T> __host__ __device__ inline int units_of(int d) { return (d + kUnit<T> - 1) / kUnit<T>; }

// Whether every row of rows at `p`, `ld` elements apart and `d` long, is whole units on 16 bytes; others are RAGGED: their units lie
// anywhere, and the last is part of one.
inline bool whole_units(const void *p, int64_t ld, int64_t d, int size) { return (uintptr_t)p % 16 == 0 && (ld * size) % 16 == 0 && (d * size) % 16 == 0; }

// Unit k / kUnit of a row, zeros past the row's end. The last one of a ragged row is read from the row's last 16 bytes and moved down:
// no load past the row, and none that waits for a branch.
template <class T, bool RAGGED> __device__ __forceinline__ Unit<T> load_unit(const T *__restrict__ row, int k, int d)
{
    constexpr int V = kUnit<T>;
    Unit<T> v;
    if (!RAGGED) return *(const Unit<T> *)(row + k);
    if (d < V) {
#pragma unroll
        for (int e = 0; e < V; ++e) v.e[e] = k + e < d ? row[k + e] : T{};
        return v;
    }
    const int past = k + V - d; // elements past the end
    __builtin_memcpy(&v, row + (past > 0 ? d - V : k), 16);
    unsigned long long lo, hi;
    __builtin_memcpy(&lo, &v.e[0], 8);
    __builtin_memcpy(&hi, &v.e[V / 2], 8);
    const int bits = d % V == 0 ? 0 : (V - d % V) * 8 * (int)sizeof(T); // (the same for all lanes: scalar shifts)
    const unsigned long long low = bits >= 64 ? hi >> (bits - 64) : bits == 0 ? lo : (lo >> bits) | (hi << (64 - bits)), high = bits >= 64 ? 0ull : hi >> bits;
    lo = past > 0 ? low : lo;
    hi = past > 0 ? high : hi;
    __builtin_memcpy(&v.e[0], &lo, 8);
    __builtin_memcpy(&v.e[V / 2], &hi, 8);
    return v;
}

template <class T, bool RAGGED> __device__ __forceinline__ void store_unit(T *__restrict__ row, int k, int d, const Unit<T> &v)
{
    constexpr int V = kUnit<T>;
    if (!RAGGED) {
        *(Unit<T> *)(row + k) = v;
    } else if (k + V <= d) {
        __builtin_memcpy(row + k, &v, 16);
    } else {
#pragma unroll
        for (int e = 0; e < V - 1; ++e)
            if (k + e < d) row[k + e] = v.e[e];
    }
}

// Bytes that every row of rows at `p`, `ld` elements apart and `d` long, can be read in at once: 16, 8 or one element.
inline int row_width(const void *p, int64_t ld, int64_t d, int size)
{
    for (int w = 16; w > 4; w /= 2)
        if (((uintptr_t)p % w) == 0 && (ld * size) % w == 0 && (d * size) % w == 0) return w;
    return size;
}

// sum over the L lanes (a power of two, at most 64) of an aligned group, in a fixed order; every lane gets it. Lanes are reached by the
// adders' own operand paths, not through LDS (eight sums over 32 lanes a row, 1,183,514 x 100 fp32: the gradient took 405 against 451 us).
template <int L> __device__ __forceinline__ float group_sum(float v)
{
    auto moved = [](float x, auto ctrl) __attribute__((always_inline)) { return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    if constexpr (L > 1) v += moved(v, std::integral_constant<int, 0xB1>{});  // the lane beside: quad_perm [1, 0, 3, 2]
    if constexpr (L > 2) v += moved(v, std::integral_constant<int, 0x4E>{});  // the other pair: quad_perm [2, 3, 0, 1]
    if constexpr (L > 4) v += moved(v, std::integral_constant<int, 0x141>{}); // the other four of eight: row_half_mirror
    if constexpr (L > 8) v += moved(v, std::integral_constant<int, 0x140>{}); // the other eight of sixteen: row_mirror
    if constexpr (L > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (L > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// q = i / by for i * by < 2^32: q = (i * magic) >> 32
__host__ __device__ inline uint32_t magic_of(uint32_t by) { return by <= 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + by - 1) / by); }
__device__ __forceinline__ uint32_t magic_div(uint32_t i, uint32_t magic) { return magic == 0 ? i : __umulhi(i, magic); }

} // namespace avq
