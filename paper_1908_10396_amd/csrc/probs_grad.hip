// The gradient of log probabilities, entropy and log-sum-exp with respect to queries and rows. With s_ti = c <q_t, x_i> and
// upstream g_tj (of log p of id_tj), h_t (of H_t), l_t (of lse_t):
//   G_ti = sum_j g_tj [id_tj = i] - p_ti (a_t + h_t log p_ti),  a_t = sum_j g_tj - l_t + h_t H_t,
//   dq_t = c sum_i G_ti x_i,  dx_i = c sum_t G_ti q_t.
// Three products of 2 n nq d operations each, on the matrix instructions, a part of the rows at a time: the part's logits once
// more, whose epilogue leaves G transposed, a row's queries side by side, in 16 bits (fp32: pairs of f16); dx = G^T Q, whose inner dimension
// both operands hold side by side (Q transposed once); dq += G X by operands that are turned as they are read from LDS. G is kept
// relative to a bound of its query's, so that f16 holds it down to 2^-39 of that; its rounding to 16 bits (bf16: 2^-9) is that of
// the operands' own type. The entries of the given ids, where p is taken from g, are formed by themselves in fp32 before rounding; p there
// has lse's rounding, 2^-24 |lse| of it, which 1 - p keeps as it is however small it is.
// Bound: the matrix instructions and G's bytes. 1,024 queries, 670,091 x 1,024 bf16, in ms: G 1.50 (0.94 PFLOP/s), dx 1.71 (0.82), dq 1.46 (0.96);
// 1,001 queries, 1,183,514 x 100 fp32: 1.10, 1.18, 1.26, where G is 4.8 GB, written once and read twice.
#include "mma_tiles.h"
#include "prob_score.h"
#include "probs.h"
#include "row_types.h"

#include <type_traits>

namespace avq {

// G of a query is kept times a power of two of its own that brings a bound of its magnitude to 2^14 .. 2^15 (bf16 needs none), so that the
// weight of other queries costs it nothing; the inverse goes to dq, and with the transposed queries into dx. What dx adds up has one scale
// all the same: where queries over their factors are apart by more than kWeightSpread, pairs (and f16) would lose the least of them, and
// dx goes by the fp32 matrix instruction.
// On top of it all queries have a constant in (1/2, 1] that brings the largest bound to a power of two: where the queries weigh the same, as
// in a mean, g of a given row is then kept as it is, and not rounded alike in every query.
struct GradCoef { float a, h, factor, inverse; }; // (inverse 0: nothing comes from this query)
constexpr float kWeightSpread = 0x1p16f;
template <class T> constexpr bool kHasFactor = std::is_same<T, float>::value || std::is_same<T, f16_t>::value;

__device__ __forceinline__ float grad_constant(const Ranges *ranges)
{
    return ranges->upstream == 0 ? 1.0f : 0x1p14f / (__uint_as_float(ranges->upstream) * range_scale(ranges->upstream));
}

template <class T> __device__ __forceinline__ bool weights_apart(const Ranges *ranges)
{
    return kHasFactor<T> && __uint_as_float(ranges->weighted) > kWeightSpread * __uint_as_float(ranges->least_weighted);
}

// A wave a query: a_t, h_t, the factor, and the range of what dx adds up.
template <class T>
__global__ __launch_bounds__(256) void grad_coef_kernel(const T *__restrict__ q, int64_t ld_q, int d, const int32_t *__restrict__ ids, int64_t n, int nq, int given,
                                                        const float *__restrict__ g, const float *__restrict__ h, const float *__restrict__ entropy, const float *__restrict__ gl,
                                                        GradCoef *__restrict__ coef, Ranges *__restrict__ ranges)
{
    __shared__ uint32_t shared_most[4], shared_least[4], shared_bound[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, t = blockIdx.x * 4 + wave;
    uint32_t most = 0, least = 0x7f800000u, bound_bits = 0; // of the query's largest magnitude over its factor; of its bound
    if (t < nq) {
        float a = 0.0f, mag = 0.0f;
        for (int j = lane; j < given; j += 64) {
            const int32_t id = ids[(int64_t)t * given + j];
            if (id >= 0 && (int64_t)id < n) {
                const float v = g[(int64_t)t * given + j];
                a += v;
                mag += fabsf(v);
            }
        }
        a = group_sum<64>(a);
        mag = group_sum<64>(mag);
        uint32_t top = 0;
        if (kHasFactor<T>) {
            for (int c = lane; c < d; c += 64) {
                const uint32_t bits = __float_as_uint(to_f32(q[t * ld_q + c])) & 0x7fffffffu;
                top = max(top, bits < 0x7f800000u ? bits : 0u);
            }
#pragma unroll
            for (int w = 1; w < 64; w <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, w, 64));
        }
        const float ht = h ? h[t] : 0.0f;
        if (gl) a -= gl[t];
        if (h) a += ht * entropy[t];
        const float bound = mag + fabsf(a) + fabsf(ht); // of |G| (p |log p| < 0.37)
        const bool some = !(bound == 0.0f);
        bound_bits = bound < INFINITY ? __float_as_uint(bound) : 0u;
        const float factor = kHasFactor<T> && bound < INFINITY ? range_scale(__float_as_uint(bound)) : 1.0f;
        if (lane == 0) coef[t] = GradCoef{a, ht, factor, some ? 1.0f / factor : 0.0f};
        const uint32_t weighted = __float_as_uint(__uint_as_float(top) / factor);
        if (kHasFactor<T> && some && bound < INFINITY && top != 0 && weighted < 0x7f800000u) most = least = weighted;
    }
    if (lane == 0) { shared_most[wave] = most; shared_least[wave] = least; shared_bound[wave] = bound_bits; }
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) { most = max(most, shared_most[w]); least = min(least, shared_least[w]); bound_bits = max(bound_bits, shared_bound[w]); }
    // (maxima and minima: no order matters; asked for first, since most change nothing)
    if (bound_bits > __hip_atomic_load(&ranges->upstream, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(&ranges->upstream, bound_bits);
    if (most > __hip_atomic_load(&ranges->weighted, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(&ranges->weighted, most);
    if (least < __hip_atomic_load(&ranges->least_weighted, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMin(&ranges->least_weighted, least);
}

// what the transposed queries are multiplied by
__global__ __launch_bounds__(256) void grad_factor_kernel(const GradCoef *__restrict__ coef, int nq, const Ranges *__restrict__ ranges, float *__restrict__ factor)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t < nq) factor[t] = coef[t].inverse == 0.0f ? 0.0f : range_scale(ranges->weighted) * coef[t].inverse;
}

// eight values as operands: rounded to the type, or (fp32) hi and lo
typedef float f32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ void put16(const f32x8 &v, Quad *hi, Quad *, bf16_t) { *hi = __builtin_bit_cast(Quad, __builtin_convertvector(v, bf16v8)); }
__device__ __forceinline__ void put16(const f32x8 &v, Quad *hi, Quad *, f16_t) { *hi = __builtin_bit_cast(Quad, __builtin_convertvector(v, f16v8)); }
__device__ __forceinline__ void put16(const f32x8 &v, Quad *hi, Quad *lo, float)
{
    const f16v8 h = __builtin_convertvector(v, f16v8);
    *hi = __builtin_bit_cast(Quad, h);
    *lo = __builtin_bit_cast(Quad, __builtin_convertvector(v - __builtin_convertvector(h, f32x8), f16v8));
}

// G is a gigabyte that is read again when all of it is written: stored past the caches, it leaves the operands there (262,144 rows,
// 1,001 queries, fp32: 225 against 320 us, and the products after it 2 to 8 % faster)
__device__ __forceinline__ void put_once(uint16_t *to, const Quad &v)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4 *)to);
}

// G^T of the part's rows: 256 queries of a workgroup by 128 rows at a time. T: the caller's type, H: the instructions'.
template <class T, class H, bool SPLIT, bool ENTROPY>
__global__ __launch_bounds__(kTileThreads, 2) void grad_tile_kernel(Rows16 Q, Rows16 X, int steps, float c2, const float *__restrict__ x_inv, const float *__restrict__ q_inv, const float *__restrict__ lse, const GradCoef *__restrict__ coef,
                                                                    const Ranges *__restrict__ ranges, int parts, int others, Rows16 G, int width)
{
    extern __shared__ char lds[];
    __shared__ float4 shift[kTileM / 4], up[kTileM / 4], up_h[kTileM / 4]; // -lse / log 2; a and h, times the factor
    __shared__ float4 to_logit[SPLIT ? kTileM / 4 : 1];
    const Place place = place_of(blockIdx.x, others);
    const int wave = threadIdx.x >> 6, half = (threadIdx.x & 63) >> 5;
    const int64_t tiles = (X.rows + kTileN - 1) / kTileN, q0 = (int64_t)place.other * kTileM;
    int64_t first;
    int count;
    part_tiles(tiles, parts, place.part, &first, &count);
    const bool apart = SPLIT && rows_apart(ranges), odd = SPLIT && ranges->odd > 0;
    {
        const int64_t t = q0 + threadIdx.x;
        const bool real = t < Q.rows; // (queries past the last have the last one's products: a probability of 0 all the same)
        const GradCoef c = real ? coef[t] : GradCoef{0.0f, 0.0f, 1.0f, 0.0f};
        ((float *)shift)[threadIdx.x] = real ? -lse[t] * 1.44269504088896341f : -INFINITY;
        if (SPLIT) ((float *)to_logit)[threadIdx.x] = real ? c2 * q_inv[t] * (apart ? 1.0f : __uint_as_float(ranges->inverse)) : 0.0f;
        const float f = c.factor * grad_constant(ranges);
        ((float *)up)[threadIdx.x] = -c.a * f;
        if (ENTROPY) ((float *)up_h)[threadIdx.x] = -c.h * f * 0.693147180559945309f;
    }
    __syncthreads();
    typedef RowCopies<true, SPLIT> Copies;
    run_tiles<H, SPLIT, true, Copies>(Q, X, steps, count, lds, [&](int i, Copies &c) { c.seek(Q, q0, X, (first + i) * kTileN); },
        [&](int i, f32x16 (&acc)[4][2]) {
            const int64_t row0 = (first + i) * kTileN;
            bool none[2] = {false, false}; // odd rows: no gradient
            if (SPLIT && (apart || odd)) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float inv = x_inv[min(row0 + acc_col(j), X.rows - 1)];
                    none[j] = inv == INFINITY;
#pragma unroll
                    for (int a = 0; a < 4; ++a)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[a][j][r] *= apart && !none[j] ? inv : 1.0f;
                }
            }
            auto take = [&](auto tail) __attribute__((always_inline)) {
                constexpr bool TAIL = decltype(tail)::value; // some rows are past the last, or odd: no gradient
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int64_t row = row0 + acc_col(j);
                    const bool real = !TAIL || (row < X.rows && !none[j]);
#pragma unroll
                    for (int a = 0; a < 4; ++a)
#pragma unroll
                        for (int block = 0; block < 2; ++block) {
                            // queries 16 block + 8 b + 4 half + e of the 32: stored side by side, two lanes' 32 bytes
                            f32x8 v;
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                const int t = (wave >> 1) * 128 + a * 32 + block * 16 + 8 * b + 4 * half;
                                const float4 s4 = shift[t / 4], u4 = up[t / 4];
                                const float sh[4] = {s4.x, s4.y, s4.z, s4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w};
                                float hh[4] = {};
                                float cq[4] = {c2, c2, c2, c2};
                                if (SPLIT) { const float4 w = to_logit[t / 4]; cq[0] = w.x; cq[1] = w.y; cq[2] = w.z; cq[3] = w.w; }
                                if (ENTROPY) { const float4 w = up_h[t / 4]; hh[0] = w.x; hh[1] = w.y; hh[2] = w.z; hh[3] = w.w; }
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float s2 = __fmaf_rn(acc[a][j][8 * block + 4 * b + e], cq[e], sh[e]), p = __builtin_amdgcn_exp2f(s2);
                                    float g = p * (ENTROPY ? __fmaf_rn(hh[e], s2, u[e]) : u[e]);
                                    if (ENTROPY && p == 0.0f) g = 0.0f; // (p log p)
                                    v[4 * b + e] = real ? g : 0.0f;
                                }
                            }
                            const int64_t t0 = q0 + (wave >> 1) * 128 + a * 32 + block * 16;
                            if (t0 < width) {
                                Quad hi, lo;
                                put16(v, &hi, &lo, T{});
                                uint16_t *to = (uint16_t *)G.p + block16<SPLIT>(t0) * G.block + row * G.row + half * 8;
                                put_once(to, hi);
                                if (SPLIT) put_once(to + G.block, lo);
                            }
                        }
                }
            };
            if (row0 + kTileN <= X.rows && !(SPLIT && __any(none[0] || none[1]))) take(std::false_type{});
            else take(std::true_type{});
        });
}

// The entries of the given ids among the part's rows, a wave each (with more ids than a launch has workgroups, one after the other); the
// first of a query's equal ids has the sum of their g. Their logits as the pass formed them that lse is of.
constexpr int64_t kGivenGroups = 1 << 22; // a launch has fewer than 2^32 threads

template <int PATH, class T>
__global__ __launch_bounds__(64) void grad_given_kernel(const T *__restrict__ x, int64_t ld_x, const T *__restrict__ q, int nq, int64_t ld_q, int d, float scale, int row_lanes,
                                                        const int32_t *__restrict__ ids, int given, const float *__restrict__ g, const float *__restrict__ lse,
                                                        const GradCoef *__restrict__ coef, const Ranges *__restrict__ ranges, const float *__restrict__ x_inv, const float *__restrict__ q_inv, int64_t lo,
                                                        int64_t rows, Rows16 G)
{
    extern __shared__ char lds[];
    T *qs = (T *)lds;
    for (int64_t i = blockIdx.x; i < (int64_t)nq * given; i += gridDim.x) {
        const int64_t t = i / given, j = i - t * given;
        const int64_t id = ids[i];
        if (id < lo || id >= lo + rows) continue;
        float sum = 0.0f;
        bool earlier = false;
        for (int64_t o = threadIdx.x; o < given; o += 64)
            if (ids[t * given + o] == id) {
                earlier = earlier || o < j;
                sum += g[t * given + o];
            }
        if (__any(earlier)) continue;
        sum = group_sum<64>(sum);
        float c = scale;
        Scoring how{row_lanes, 1.0f};
        if (PATH == kByTiles && sizeof(T) == 4) {
            how.q_scale = 1.0f / (kRowUnit * q_inv[t]);
            c = c * q_inv[t];
        }
        __syncthreads(); // (the query before has been read)
        stage_query(qs, q + t * ld_q, d, false, 64);
        __syncthreads();
        score_rows<PATH, 8>(qs, d, how, [&](int) { return x + id * ld_x; }, [&](int) { return x_inv[id]; }, [&](int slot, float product) {
            if (slot != 0) return;
            const bool odd = PATH == kByTiles && sizeof(T) == 4 && x_inv[id] == INFINITY; // (a logit of -infinity, whatever the scale's sign)
            const float logp = odd ? -INFINITY : __fmaf_rn(product, c, -lse[t]);
            const GradCoef k = coef[t];
            const float p = __builtin_amdgcn_exp2f(logp * 1.44269504088896341f);
            f32x8 one = {};
            one[0] = (sum - (p > 0.0f || p != p ? p * __fmaf_rn(k.h, logp, k.a) : 0.0f)) * (k.factor * grad_constant(ranges));
            Quad hi, low{};
            put16(one, &hi, &low, T{});
            uint16_t *to = (uint16_t *)G.p + block16<sizeof(T) == 4>(t) * G.block + (id - lo) * G.row + turned16((int)t & 15);
            *to = (uint16_t)hi.w[0];
            if (sizeof(T) == 4) to[G.block] = (uint16_t)low.w[0];
        });
    }
}

// fn for every four rows side by side of a lane's accumulators acc[a][j][4 b ..]. One after the other: the compiler would
// otherwise keep the addresses of all of them in registers at once.
template <int A, int B, int J> struct QuadAt { static constexpr int a = A, b = B, j = J; };
template <int I = 0, class Fn> __device__ __forceinline__ void for_quads(Fn fn)
{
    if constexpr (I < 32) {
        fn(QuadAt<I / 4 % 4, I % 4, I / 16>{});
        asm volatile("" ::: "memory");
        for_quads<I + 1>(fn);
    }
}

// A tile of dx by the fp32 matrix instruction, two queries at a time; acc as the other form has it.
template <class T>
__device__ __forceinline__ void rows_by_fp32(const Rows16 &G, int64_t row0, const T *__restrict__ q, int64_t ld_q, int nq, int d, int64_t c0, const GradCoef *__restrict__ coef, f32x16 (&acc)[4][2])
{
    constexpr bool SPLIT = sizeof(T) == 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const uint16_t *g[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = G.p + min(row0 + (wave >> 1) * 128 + i * 32 + (lane & 31), G.rows - 1) * G.row + half * 8;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    }
    for (int t0 = 0; t0 < nq; t0 += 16) {
        float ga[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint16_t *from = g[i] + block16<SPLIT>(t0) * G.block;
            uint16_t hi[8], lo[8];
            __builtin_memcpy(hi, from, 16);
            if (SPLIT) __builtin_memcpy(lo, from + G.block, 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) ga[i][e] = SPLIT ? to_f32(f16_t{hi[e]}) + to_f32(f16_t{lo[e]}) : to_f32(f16_t{hi[e]});
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int t = t0 + turned16(half * 8 + e);
            const float inverse = t < nq ? coef[t].inverse : 0.0f;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t c = c0 + (wave & 1) * 64 + j * 32 + (lane & 31);
                const float b = inverse != 0.0f && c < d ? to_f32(q[t * ld_q + c]) * inverse : 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(ga[i][e], b, acc[i][j], 0, 0, 0);
            }
        }
    }
}

// dx of the part's rows: 256 rows by 128 dimensions.
// PAIRS: 16-bit types of rows on 4 bytes, of an even number of elements.
template <class T, class H, bool SPLIT, bool ACCUMULATE, bool PAIRS>
__global__ __launch_bounds__(kTileThreads, 2) void grad_rows_kernel(Rows16 G, Rows16 Qt, int steps, float scale, const Ranges *__restrict__ ranges, int parts, int others, int64_t rows,
                                                                    int d, const T *__restrict__ q, int64_t ld_q, int nq, const GradCoef *__restrict__ coef, T *__restrict__ dx, int64_t ld_dx)
{
    extern __shared__ char lds[];
    const Place place = place_of(blockIdx.x, others);
    const int64_t tiles = (rows + kTileM - 1) / kTileM, c0 = (int64_t)place.other * kTileN;
    int64_t first;
    int count;
    part_tiles(tiles, parts, place.part, &first, &count);
    const bool apart = weights_apart<T>(ranges);
    const float f = (kHasFactor<T> && !apart ? scale * (1.0f / range_scale(ranges->weighted)) : scale) / grad_constant(ranges);
    typedef RowCopies<true, true> Copies;
    auto store = [&](int i, f32x16 (&acc)[4][2]) __attribute__((always_inline)) {
        const int64_t row0 = (first + i) * kTileM + acc_row(0, 0);
        const int64_t left = rows - row0; // rows from this lane's first one on
        for_quads([&](auto at) {
            constexpr int a = decltype(at)::a, b = decltype(at)::b, j = decltype(at)::j;
            const int64_t c = c0 + acc_col(j);
            T *to = dx + (row0 + a * 32 + b * 8) * ld_dx + c;
            if (PAIRS) {
                // two lanes, two rows: each stores both columns of one
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float v0 = acc[a][j][4 * b + e] * f, v1 = acc[a][j][4 * b + e + 1] * f;
                    const bool odd = threadIdx.x & 1;
                    const float other = __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(odd ? v0 : v1), 0xB1 /* quad_perm [1, 0, 3, 2] */, 0xF, 0xF, true));
                    T *at = to + (odd ? ld_dx - 1 : 0);
                    if (c < d && a * 32 + b * 8 + e + (odd ? 1 : 0) < left) {
                        Pack<T, 2> o;
                        float lo = odd ? other : v0, hi = odd ? v1 : other;
                        if (ACCUMULATE) { o = *(const Pack<T, 2> *)at; lo += to_f32(o.e[0]); hi += to_f32(o.e[1]); }
                        o.e[0] = from_f32<T>(lo);
                        o.e[1] = from_f32<T>(hi);
                        *(Pack<T, 2> *)at = o;
                    }
                    to += 2 * ld_dx;
                }
                return;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (c < d && a * 32 + b * 8 + e < left) {
                    const float v = acc[a][j][4 * b + e] * f;
                    *to = from_f32<T>(ACCUMULATE ? to_f32(*to) + v : v);
                }
                to += ld_dx;
            }
        });
    };
    if (kHasFactor<T> && apart) {
        for (int i = 0; i < count; ++i) {
            f32x16 acc[4][2];
            rows_by_fp32<T>(G, (first + i) * kTileM, q, ld_q, nq, d, c0, coef, acc);
            store(i, acc);
        }
        return;
    }
    run_tiles<H, SPLIT, true, Copies>(G, Qt, steps, count, lds, [&](int i, Copies &c) { c.seek(G, (first + i) * kTileM, Qt, c0); }, store);
}

// A tile of dq by the fp32 matrix instruction, 16 rows [row0, row0 + 16 steps) at a time, of which x has `rows`; acc as the other form has it.
__device__ __forceinline__ void queries_by_fp32(const Rows16 &G, int64_t t0, int width, const float *__restrict__ x, int64_t ld_x, int64_t rows, int64_t row0, int steps, int d, int64_t c0,
                                                f32x16 (&acc)[4][2])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const uint16_t *g[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t p = t0 + (wave >> 1) * 128 + i * 32 + (lane & 31), at = p < width ? p : 0; // (places past the last are not stored)
        g[i] = G.p + block16<true>(at) * G.block + (at & 15);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    }
    for (int s = 0; s < steps; ++s) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t row = row0 + (int64_t)s * 16 + half * 8 + e, at = min(row, rows - 1);
            float ga[4], b[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) ga[i] = row < rows ? to_f32(f16_t{g[i][at * G.row]}) + to_f32(f16_t{g[i][G.block + at * G.row]}) : 0.0f;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t c = c0 + (wave & 1) * 64 + j * 32 + (lane & 31);
                const float v = c < d ? x[at * ld_x + c] : 0.0f;
                b[j] = fabsf(v) < INFINITY ? v : 0.0f; // (as zeros stand for odd rows among the pairs)
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(ga[i], b[j], acc[i][j], 0, 0, 0);
        }
    }
}

// The part's share of dq, split over the part's rows: sums[split][nq][d] in fp32, begun (first) or added to. x: the part's rows as they
// are, for fp32 tables whose rows are apart.
template <class H, bool SPLIT>
__global__ __launch_bounds__(kTileThreads, 2) void grad_queries_kernel(Rows16 G, Rows16 X, int nq, int width, int d, int splits, int q_tiles, int d_tiles, int begin, const float *__restrict__ x,
                                                                       int64_t ld_x, const Ranges *__restrict__ ranges, float *__restrict__ sums)
{
    extern __shared__ char lds[];
    const Place place = place_of(blockIdx.x, q_tiles * d_tiles);
    const int64_t t0 = (int64_t)(place.other % q_tiles) * kTileM, c0 = (int64_t)(place.other / q_tiles) * kTileN;
    typedef ColumnCopies<SPLIT> Copies;
    const int64_t steps = (G.rows + Copies::kRows - 1) / Copies::kRows;
    int64_t first;
    int count;
    part_tiles(steps, splits, place.part, &first, &count);
    float *mine = sums + (int64_t)place.part * nq * d;
    auto store = [&](int, f32x16 (&acc)[4][2]) {
        // the order of 16 queries is turned: position 8 b + 4 h + e of a block is query 8 h + 4 b + e
        const int half = (threadIdx.x & 63) >> 5;
        const int64_t row0 = t0 + (acc_row(0, 0) - 4 * half) + 8 * half, left = nq - row0;
        for_quads([&](auto at) {
            constexpr int a = decltype(at)::a, b = decltype(at)::b, j = decltype(at)::j;
            constexpr int off = a * 32 + (b >> 1) * 16 + (b & 1) * 4;
            const int64_t c = c0 + acc_col(j);
            float *to = mine + (row0 + off) * d + c;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (c < d && off + e < left) *to = begin ? acc[a][j][4 * b + e] : *to + acc[a][j][4 * b + e];
                to += d;
            }
        });
    };
    if (count == 0) { // (a workgroup without rows still begins its sums)
        f32x16 none[4][2] = {};
        if (begin) store(0, none);
        return;
    }
    if (SPLIT && rows_apart(ranges)) {
        f32x16 acc[4][2];
        queries_by_fp32(G, t0, width, x, ld_x, X.rows, first * Copies::kRows, count, d, c0, acc);
        store(0, acc);
        return;
    }
    run_tiles<H, SPLIT, true, Copies>(G, X, count, 1, lds, [&](int, Copies &c) { c.row = first * Copies::kRows; c.seek(G, t0, width, X, c0); }, store);
}

// dq = the splits' sums, in their order
template <class T>
__global__ __launch_bounds__(256) void grad_join_kernel(const float *__restrict__ sums, int splits, int nq, int d, float scale, int fp32, const Ranges *__restrict__ ranges,
                                                        const GradCoef *__restrict__ coef, T *__restrict__ out, int64_t ld)
{
    const int64_t all = (int64_t)nq * d;
    const float f = scale * (fp32 && !rows_apart(ranges) ? __uint_as_float(ranges->inverse) * (1.0f / kRowUnit) : 1.0f) / grad_constant(ranges);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        float s = 0.0f;
#pragma unroll 8
        for (int p = 0; p < splits; ++p) s += sums[p * all + i];
        out[(i / d) * ld + i % d] = from_f32<T>(s * coef[i / d].inverse * f);
    }
}

template <class T>
__global__ __launch_bounds__(256) void grad_zero_kernel(T *__restrict__ out, int64_t rows, int d, int64_t ld)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = threadIdx.x; c < d; c += 256) out[r * ld + c] = T{};
}

constexpr int kGradGroups = 512;                  // two workgroups a compute unit
constexpr size_t kGradBytes = (size_t)1 << 30;    // most that G of a part takes where a part has more than the least rows

struct ProbGradScratch {
    bool pack;
    int steps, d_steps, qw, q_steps, splits, q_tiles, d_tiles; // steps of products over dimensions, of packed rows, of products over queries
    int64_t part;                                              // rows at a time
    Ranges *ranges; GradCoef *coef; float *factor, *x_inv, *q_inv, *sums; uint16_t *q16, *qt16, *x16, *G;
    size_t bytes;
};

static ProbGradScratch prob_grad_scratch(const ProbGradParams &p, void *base)
{
    ProbGradScratch s{};
    const int pair = p.type == AVQ_F32 ? 2 : 1;
    const bool split = pair == 2;
    s.q_tiles = (p.nq + kTileM - 1) / kTileM;
    s.d_tiles = (p.d + kTileN - 1) / kTileN;
    s.steps = split ? steps_of<true>(p.d) : steps_of<false>(p.d);
    s.d_steps = s.d_tiles * (kTileN * pair / 32); // (the product over rows reads whole tiles of columns)
    s.qw = (p.nq + 31) / 32 * 32;
    s.q_steps = s.qw * pair / 32;
    const size_t row_bytes = (size_t)s.d_steps * kStepBytes, g_bytes = (size_t)s.q_steps * kStepBytes;
    // (base == NULL: the size for rows that need packing, whatever their place and stride)
    s.pack = !base || split || p.d % kTileN != 0 || (uintptr_t)p.points % 16 != 0 || p.ld_points % 8 != 0 || p.ld_points >= kMaxRow16;
    const int64_t most = (int64_t)(kGradBytes / std::max(row_bytes, g_bytes)) / kTileM * kTileM;
    s.part = std::min<int64_t>((p.n + kTileM - 1) / kTileM * kTileM, std::max<int64_t>(4096, most));
    const int64_t launches = (p.n + s.part - 1) / s.part; // parts of equal size
    s.part = std::min(s.part, ((p.n + launches - 1) / launches + kTileM - 1) / kTileM * kTileM);
    s.splits = parts_for(std::max<int64_t>(1, s.part / 128), s.q_tiles * s.d_tiles, kGradGroups);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *q = base ? (char *)base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return q;
    };
    s.ranges = (Ranges *)take(sizeof(Ranges));
    s.coef = (GradCoef *)take(sizeof(GradCoef) * (size_t)p.nq);
    s.factor = (float *)take(sizeof(float) * (size_t)p.nq);
    s.x_inv = split ? (float *)take(sizeof(float) * (size_t)p.n) : nullptr;
    s.q_inv = split ? (float *)take(sizeof(float) * (size_t)p.nq) : nullptr;
    s.sums = (float *)take(sizeof(float) * (size_t)s.splits * p.nq * p.d);
    s.q16 = (uint16_t *)take(packed_bytes(p.nq, s.steps));
    s.qt16 = (uint16_t *)take(packed_bytes(p.d, s.q_steps));
    s.G = (uint16_t *)take(packed_bytes(s.part, s.q_steps));
    if (s.pack) s.x16 = (uint16_t *)take(packed_bytes(s.part, s.d_steps));
    s.bytes = at;
    return s;
}

size_t log_probs_grad_scratch_bytes(int type, int64_t n, int d, int nq, int given)
{
    if (grad_few_takes(type, d, nq, given)) return grad_few_scratch_bytes(type, d, nq);
    ProbGradParams p{};
    p.type = type; p.n = n; p.d = d; p.nq = nq;
    return nq == 0 ? 0 : prob_grad_scratch(p, nullptr).bytes;
}

template <class T, class H, bool SPLIT>
static int log_probs_grad_typed(const ProbGradParams &p, hipStream_t st)
{
    if (p.nq == 0) {
        if (p.dpoints && !p.accumulate) {
            grad_zero_kernel<T><<<dim3((unsigned)std::min<int64_t>(p.n, 65536)), dim3(256), 0, st>>>((T *)p.dpoints, p.n, p.d, p.ld_dpoints);
            AVQ_HIP(hipGetLastError());
        }
        return AVQ_OK;
    }
    const ProbGradScratch s = prob_grad_scratch(p, p.scratch);
    static LdsLimitOnce once[3];
    AVQ_TRY(set_lds_limit((const void *)grad_tile_kernel<T, H, SPLIT, false>, kTileLds, &once[0]));
    AVQ_TRY(set_lds_limit((const void *)grad_tile_kernel<T, H, SPLIT, true>, kTileLds, &once[1]));
    AVQ_TRY(set_lds_limit((const void *)grad_queries_kernel<H, SPLIT>, kTileLds, &once[2]));
    const float c2 = p.scale * 1.44269504088896341f;
    const T *q = (const T *)p.queries;
    AVQ_TRY(launch_clear_ranges(s.ranges, st));
    grad_coef_kernel<T><<<dim3((p.nq + 3) / 4), dim3(256), 0, st>>>(q, p.ld_queries, p.d, p.ids, p.n, p.nq, p.given, p.grad_logp, p.grad_entropy, p.entropy, p.grad_lse, s.coef, s.ranges);
    AVQ_HIP(hipGetLastError());
    const Rows16 Q = packed_rows(s.q16, p.nq), Qt = packed_rows(s.qt16, p.d);
    if (SPLIT) {
        AVQ_TRY(launch_pack_queries((const float *)p.queries, p.nq, p.d, p.ld_queries, s.steps, Q, s.q_inv, OddRows{}, false, st));
        AVQ_TRY(launch_common_inverses((const float *)p.points, p.n, p.d, p.ld_points, s.x_inv, s.ranges, st));
    } else {
        AVQ_TRY(launch_pack_rows(p.queries, p.type, p.nq, p.d, p.ld_queries, s.steps, Q, nullptr, false, st));
    }
    if (p.dpoints) {
        if (kHasFactor<T>) {
            grad_factor_kernel<<<dim3((p.nq + 255) / 256), dim3(256), 0, st>>>(s.coef, p.nq, s.ranges, s.factor);
            AVQ_HIP(hipGetLastError());
        }
        AVQ_TRY(launch_pack_transposed(p.queries, p.type, p.nq, p.d, p.ld_queries, s.q_steps, Qt, kHasFactor<T> ? s.factor : nullptr, st));
    }
    for (int64_t lo = 0; lo < p.n; lo += s.part) {
        const int64_t rows = std::min<int64_t>(s.part, p.n - lo), whole = (rows + kTileN - 1) / kTileN * kTileN; // rows past the last have G = 0
        const T *x = (const T *)p.points + lo * p.ld_points;
        Rows16 X{(const uint16_t *)x, p.ld_points, 16, rows};
        if (s.pack) {
            X = SPLIT ? packed_rows(s.x16, rows) : Rows16{s.x16, (int64_t)s.d_steps * 32, 16, rows};
            AVQ_TRY(launch_pack_rows(x, p.type, rows, p.d, p.ld_points, s.d_steps, X, SPLIT ? s.x_inv + lo : nullptr, false, st));
        }
        const Rows16 G = packed_rows(s.G, whole);
        const int parts = parts_for((rows + kTileN - 1) / kTileN, s.q_tiles, kGradGroups);
        const dim3 grid((unsigned)(parts * s.q_tiles));
        const float *x_inv = SPLIT ? s.x_inv + lo : nullptr;
        if (p.grad_entropy) grad_tile_kernel<T, H, SPLIT, true><<<grid, dim3(kTileThreads), kTileLds, st>>>(Q, X, s.steps, c2, x_inv, s.q_inv, p.lse, s.coef, s.ranges, parts, s.q_tiles, G, s.qw);
        else grad_tile_kernel<T, H, SPLIT, false><<<grid, dim3(kTileThreads), kTileLds, st>>>(Q, X, s.steps, c2, x_inv, s.q_inv, p.lse, s.coef, s.ranges, parts, s.q_tiles, G, s.qw);
        AVQ_HIP(hipGetLastError());
        if (p.given > 0) {
            auto run = [&](auto kernel) {
                kernel<<<dim3((unsigned)std::min((int64_t)p.nq * p.given, kGivenGroups)), dim3(64), staged_query_bytes(p.d), st>>>((const T *)p.points, p.ld_points, q, p.nq, p.ld_queries, p.d, p.scale, row_lanes(sizeof(T), p.d),
                                                                                                    p.ids, p.given, p.grad_logp, p.lse, s.coef, s.ranges, s.x_inv, s.q_inv, lo, rows, G);
            };
            const int path = prob_path(sizeof(T), p.d, p.nq);
            if (path == kByTiles) run(grad_given_kernel<kByTiles, T>);
            else if (path == kByStream) run(grad_given_kernel<kByStream, T>);
            else run(grad_given_kernel<kByRow, T>);
            AVQ_HIP(hipGetLastError());
        }
        if (p.dpoints) {
            const int row_parts = parts_for((rows + kTileM - 1) / kTileM, s.d_tiles, kGradGroups);
            T *dx = (T *)p.dpoints + lo * p.ld_dpoints;
            const bool pairs = sizeof(T) == 2 && (uintptr_t)p.dpoints % 4 == 0 && p.ld_dpoints % 2 == 0 && p.d % 2 == 0;
            auto run = [&](auto accumulate, auto pair) -> int {
                constexpr bool ACCUMULATE = decltype(accumulate)::value, PAIRS = decltype(pair)::value;
                static LdsLimitOnce row_once;
                AVQ_TRY(set_lds_limit((const void *)grad_rows_kernel<T, H, SPLIT, ACCUMULATE, PAIRS>, kTileLds, &row_once));
                grad_rows_kernel<T, H, SPLIT, ACCUMULATE, PAIRS><<<dim3((unsigned)(row_parts * s.d_tiles)), dim3(kTileThreads), kTileLds, st>>>(
                    G, Qt, steps_of<SPLIT>(p.nq), p.scale, s.ranges, row_parts, s.d_tiles, rows, p.d, q, p.ld_queries, p.nq, s.coef, dx, p.ld_dpoints);
                AVQ_HIP(hipGetLastError());
                return AVQ_OK;
            };
            typedef std::integral_constant<bool, sizeof(T) == 2> Paired;
            if (pairs) AVQ_TRY(p.accumulate ? run(std::true_type{}, Paired{}) : run(std::false_type{}, Paired{}));
            else AVQ_TRY(p.accumulate ? run(std::true_type{}, std::false_type{}) : run(std::false_type{}, std::false_type{}));
        }
        if (p.dqueries) {
            grad_queries_kernel<H, SPLIT><<<dim3((unsigned)(s.splits * s.q_tiles * s.d_tiles)), dim3(kTileThreads), kTileLds, st>>>(G, X, p.nq, s.qw, p.d, s.splits, s.q_tiles, s.d_tiles,
                                                                                                                             lo == 0, (const float *)x, p.ld_points, s.ranges, s.sums);
            AVQ_HIP(hipGetLastError());
        }
    }
    if (p.dqueries) {
        grad_join_kernel<T><<<dim3((unsigned)std::min<int64_t>(((int64_t)p.nq * p.d + 255) / 256, 1 << 22)), dim3(256), 0, st>>>(s.sums, s.splits, p.nq, p.d, p.scale, SPLIT, s.ranges, s.coef, (T *)p.dqueries,
                                                                                                   p.ld_dqueries);
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

int launch_log_probs_grad(const ProbGradParams &p, hipStream_t st)
{
    if (grad_few_takes(p.type, p.d, p.nq, p.given)) return launch_grad_few(p, st);
    if (p.type == AVQ_F32) return log_probs_grad_typed<float, f16_t, true>(p, st);
    return p.type == AVQ_BF16 ? log_probs_grad_typed<bf16_t, bf16_t, false>(p, st) : log_probs_grad_typed<f16_t, f16_t, false>(p, st);
}

} // namespace avq
