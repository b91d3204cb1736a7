// Inner products of single rows with a query, by the arithmetic of the pass that formed the query's statistics, so that what is
// taken from those is what went into them: log p of a row with nearly all of the probability is the difference of two logits
// near the maximum, and two orders of additions would leave their rounding there.
#pragma once
#include "mma_tiles.h"
#include "probs.h"
#include "row_types.h"

namespace avq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// ---- operands: 16 bytes a lane -------------------------------------------------------------

struct alignas(16) Frag { uint32_t w[4]; };
template <class T> constexpr int kFragElems = 16 / sizeof(T);
template <class T> constexpr int kStepElems = 4 * kFragElems<T>; // coordinates that a step of 64 lanes covers (16 rows by 4 lanes)

template <class T, bool ALIGNED>
__device__ __forceinline__ Frag load_whole(const T *__restrict__ p)
{
    Frag f;
    if (ALIGNED) f = *(const Frag *)p;
    else __builtin_memcpy(&f, p, 16);
    return f;
}

// of what is not read again, and had better not displace what the caches hold
template <class T>
__device__ __forceinline__ Frag load_once(const T *__restrict__ p)
{
    typedef uint32_t on4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint32_t on2 __attribute__((ext_vector_type(4), aligned(2)));
    return __builtin_bit_cast(Frag, sizeof(T) == 4 ? __builtin_nontemporal_load((const on4 *)p) : __builtin_nontemporal_load((const on2 *)p));
}

// The coordinates k .. k + kFragElems - 1 of a row of d, zeros past its end. ALIGNED: the row starts on 16 bytes.
template <class T, bool ALIGNED>
__device__ __forceinline__ Frag load_frag(const T *__restrict__ row, int k, int d)
{
    constexpr int E = kFragElems<T>;
    Frag f{};
    if (k + E <= d) {
        f = load_whole<T, ALIGNED>(row + k);
    } else {
        T e[E];
#pragma unroll
        for (int j = 0; j < E; ++j) e[j] = k + j < d ? row[k + j] : T{};
        __builtin_memcpy(&f, e, 16);
    }
    return f;
}

// acc += A B^T over the step's coordinates; both operands: lane l has row l & 15, coordinates kFragElems (l >> 4) onwards.
// (fp32: which four coordinates share an instruction does not matter as long as both operands agree.)
__device__ __forceinline__ f32x4 mma16(const Frag &a, const Frag &b, f32x4 acc, float)
{
#pragma unroll
    for (int c = 0; c < 4; ++c) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[c]), __uint_as_float(b.w[c]), acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ f32x4 mma16(const Frag &a, const Frag &b, f32x4 acc, bf16_t)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(const Frag &a, const Frag &b, f32x4 acc, f16_t)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}

template <class T> __device__ __forceinline__ Frag negated(Frag f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f.w[i] ^= sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
    return f;
}

// ---- rows of one query ------------------------------------------------------------------------

// The query in LDS, as the pass multiplies with it: of its type, negated where the scale is, zeros from d to a multiple of 32.
template <class T>
__device__ __forceinline__ void stage_query(T *qs, const T *__restrict__ q, int d, bool negate, int threads)
{
    for (int k = threadIdx.x; k < (d + 31) / 32 * 32; k += threads) {
        float v = k < d ? to_f32(q[k]) : 0.0f;
        qs[k] = from_f32<T>(negate ? -v : v);
    }
}
inline size_t staged_query_bytes(int d) { return (size_t)(d + 31) / 32 * 32 * 4; }

// 16 bytes of a row that are read whatever lies there (at k, or at the row's start), and then only count where they are the row's:
// no load waits for a branch. Rows of at least 16 bytes.
template <class T> __device__ __forceinline__ Frag load_or_start(const T *__restrict__ row, int k, int d) { return load_whole<T, false>(row + (k + kFragElems<T> <= d ? k : 0)); }
template <class T>
__device__ __forceinline__ Frag checked(const Frag &f, const T *__restrict__ row, int k, int d)
{
    if (k + kFragElems<T> <= d) return f;
    return k < d ? load_frag<T, false>(row, k, d) : Frag{};
}

// What the pass of a query's statistics is described by. lanes: of a row (kByRow); q_scale: of the query's fp32 pairs (kByTiles).
struct Scoring { int lanes; float q_scale; };

// Rows that a wave scores at once.
template <int PATH> __device__ __forceinline__ int scored_at_once(const Scoring &how) { return PATH == kByTiles ? 32 : PATH == kByStream ? 16 : 4 * (64 / how.lanes); }

// row(i): the i-th of those rows (a valid one always); inverse(i): that of its scale (fp32 pairs); emit(i, product): once for each, on
// some lane.
// AHEAD: 16 coordinates' loads in flight (kByTiles), STEPS: steps' (kByStream).
template <int PATH, int AHEAD, int STEPS = 16, class T, class RowOf, class InverseOf, class Emit>
__device__ __forceinline__ void score_rows(const T *__restrict__ qs, int d, const Scoring &how, RowOf row, InverseOf inverse, Emit emit)
{
    constexpr int E = kFragElems<T>;
    const int lane = threadIdx.x & 63;
    if constexpr (PATH == kByRow) {
        const int L = how.lanes, in_row = lane % L, per = 64 / L, loads = (d + E * L - 1) / (E * L); // (at most four)
        const T *p[4];
        float s[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) { p[b] = row(b * per + lane / L); s[b] = 0.0f; }
        for (int f = 0; f < loads; ++f) {
            const int k = (f * L + in_row) * E;
            Frag v[4];
            if (d >= E) {
#pragma unroll
                for (int b = 0; b < 4; ++b) v[b] = load_or_start(p[b], k, d);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                T e[E];
                const Frag w = d >= E ? checked(v[b], p[b], k, d) : load_frag<T, false>(p[b], k, d);
                __builtin_memcpy(e, &w, 16);
#pragma unroll
                for (int j = 0; j < E; ++j) s[b] = __fmaf_rn(k + j < d ? to_f32(qs[k + j]) : 0.0f, to_f32(e[j]), s[b]);
            }
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            for (int w = 1; w < L; w <<= 1) s[b] += __shfl_xor(s[b], w, 64);
            if (in_row == 0) emit(b * per + lane / L, s[b]);
        }
    } else if constexpr (PATH == kByStream) {
        // whole steps, NB of them asked for at once (some again past the last), and what is left
        constexpr int S = kStepElems<T>, NB = STEPS;
        const int r16 = lane & 15, kg = lane >> 4, whole = d / S;
        const T *p = row(r16);
        f32x4 acc{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
        for (int s0 = 0; s0 < whole; s0 += NB) {
            Frag v[NB];
#pragma unroll
            for (int u = 0; u < NB; ++u) v[u] = load_whole<T, false>(p + min(s0 + u, whole - 1) * S + kg * E);
#pragma unroll
            for (int u = 0; u < NB; ++u)
                if (s0 + u < whole) acc = mma16(v[u], *(const Frag *)(qs + (s0 + u) * S + kg * E), acc, T{});
        }
        if (whole * S < d) acc = mma16(load_frag<T, false>(p, whole * S + kg * E, d), *(const Frag *)(qs + whole * S + kg * E), acc, T{});
        if (r16 == 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r) emit(4 * kg + r, acc[r]);
        }
    } else {
        constexpr bool SPLIT = sizeof(T) == 4;
        constexpr int NB = AHEAD, V = SPLIT ? 2 : 1; // loads of a lane's eight
        const int half = lane >> 5, whole = d / 16;
        const T *p = row(lane & 31);
        const float inv = SPLIT ? inverse(lane & 31) : 1.0f, x_scale = SPLIT ? scale_of_inverse(inv) : 1.0f;
        f32x16 acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
        auto add = [&](const Frag (&a)[V], int k) __attribute__((always_inline)) {
            if constexpr (SPLIT) {
                float xs[8];
                __builtin_memcpy(xs, a, 32);
                uint16_t xh[8], xl[8], qh[8], ql[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    split_f16(x_scale == 0.0f ? 0.0f : xs[e] * x_scale, &xh[e], &xl[e]);
                    split_f16(qs[k + e] * how.q_scale, &qh[e], &ql[e]);
                }
                Quad hi, lo, q_hi, q_lo;
                __builtin_memcpy(&hi, xh, 16);
                __builtin_memcpy(&lo, xl, 16);
                __builtin_memcpy(&q_hi, qh, 16);
                __builtin_memcpy(&q_lo, ql, 16);
                acc = mma32(hi, q_hi, acc, f16_t{});
                acc = mma32(hi, q_lo, acc, f16_t{});
                acc = mma32(lo, q_hi, acc, f16_t{});
            } else {
                acc = mma32(__builtin_bit_cast(Quad, a[0]), *(const Quad *)(qs + k), acc, T{});
            }
        };
#pragma unroll 1
        for (int b0 = 0; b0 < whole; b0 += NB) {
            Frag v[NB][V];
#pragma unroll
            for (int u = 0; u < NB; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) v[u][i] = load_whole<T, false>(p + min(b0 + u, whole - 1) * 16 + half * 8 + i * E);
#pragma unroll
            for (int u = 0; u < NB; ++u)
                if (b0 + u < whole) add(v[u], (b0 + u) * 16 + half * 8);
        }
        if (whole * 16 < d) {
            const int k = whole * 16 + half * 8;
            Frag v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = load_frag<T, false>(p, k + i * E, d);
            add(v, k);
        }
        // (every column is the same: of two lanes that loaded a row one has its product, at acc_row's place)
        const int mine = lane & 31, at = (mine >> 3) * 4 + (mine & 3);
        float product = acc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) product = at == r ? acc[r] : product;
        if ((mine >> 2 & 1) == half) emit(mine, SPLIT ? fmaxf(product * inv, -INFINITY) : product); // (an odd row's 0 times infinity: -infinity)
    }
}

} // namespace avq
