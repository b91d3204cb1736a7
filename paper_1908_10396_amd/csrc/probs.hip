// Log probabilities of rows of a table under the softmax of a query's inner products with all rows:
//   s_i = c <q, x_i>,  lse = log sum_i e^s_i,  log p_i = s_i - lse,  H = lse - sum_i p_i s_i,
// and the k rows of largest s_i (ties: the lower id). One pass over the rows keeps, per query and lane, the running maximum m
// and the sums of e^(s - m) and e^(s - m) (s - m) in fp32; the logits are never stored. For the best rows it leaves the
// largest inner product of every 32 rows; the k groups with the largest of those hold the k best rows, which are scored again.
#include "mma_tiles.h"
#include "probs.h"
#include "row_types.h"
#include "wg_select.h"

#include <type_traits>

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

// ---- a few queries: the rows streamed once -------------------------------------------------

constexpr int kStreamThreads = 256, kStreamWaves = kStreamThreads / 64;

// A wave takes 32 rows at a time, a query tile is QT x 16 queries. The rows' operands come straight from memory (a lane's 16
// bytes are the matrix instruction's layout), the queries' from LDS, where they lie in the same order (QLDS), or from memory.
template <class T, int QT, bool ALIGNED, bool QLDS>
__global__ __launch_bounds__(kStreamThreads) void prob_stream_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, int nq, int64_t ld_q,
                                                                     float c2, int negate, float4 *__restrict__ stats, float *__restrict__ gmax, int64_t gstride)
{
    extern __shared__ Frag qs[]; // [step][QT][64]
    __shared__ float4 joined[kStreamWaves][QT * 16];
    constexpr int S = kStepElems<T>, E = kFragElems<T>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r16 = lane & 15, kg = lane >> 4;
    const int q0 = blockIdx.y * QT * 16;
    const int steps = (d + S - 1) / S;
    if (QLDS) {
        for (int i = threadIdx.x; i < steps * QT * 64; i += kStreamThreads) {
            const int l = i & 63, t = (i >> 6) % QT, s = (i >> 6) / QT;
            const int row = q0 + t * 16 + (l & 15);
            Frag f{};
            if (row < nq) f = load_frag<T, false>(q + (int64_t)row * ld_q, s * S + (l >> 4) * E, d);
            qs[i] = negate ? negated<T>(f) : f;
        }
        __syncthreads();
    }
    float m[QT], l[QT], t[QT];
#pragma unroll
    for (int i = 0; i < QT; ++i) { m[i] = -INFINITY; l[i] = 0.0f; t[i] = 0.0f; }
    const int64_t tiles = (n + 31) / 32;
    const int64_t waves = (int64_t)gridDim.x * kStreamWaves;
    for (int64_t tile = (int64_t)blockIdx.x * kStreamWaves + wave; tile < tiles; tile += waves) {
        const int64_t r0 = tile * 32 + r16, r1 = r0 + 16;
        const T *p0 = x + (r0 < n ? r0 : n - 1) * ld_x, *p1 = x + (r1 < n ? r1 : n - 1) * ld_x;
        f32x4 acc[2][QT];
#pragma unroll
        for (int i = 0; i < QT; ++i) acc[0][i] = acc[1][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        auto step = [&](int s, const Frag &a0, const Frag &a1) {
            const int k = s * S + kg * E;
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                Frag b{};
                if (QLDS) {
                    b = qs[(s * QT + i) * 64 + lane];
                } else {
                    const int row = q0 + i * 16 + r16;
                    if (row < nq) b = load_frag<T, false>(q + (int64_t)row * ld_q, k, d);
                    if (negate) b = negated<T>(b);
                }
                acc[0][i] = mma16(a0, b, acc[0][i], T{});
                acc[1][i] = mma16(a1, b, acc[1][i], T{});
            }
        };
        // whole steps, four of them asked for at a time
        const int whole = d / S;
        int s = 0;
        for (; s + 4 <= whole; s += 4) {
            Frag a[2][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                a[0][u] = load_whole<T, ALIGNED>(p0 + (s + u) * S + kg * E);
                a[1][u] = load_whole<T, ALIGNED>(p1 + (s + u) * S + kg * E);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) step(s + u, a[0][u], a[1][u]);
        }
        for (; s < steps; ++s) step(s, load_frag<T, ALIGNED>(p0, s * S + kg * E, d), load_frag<T, ALIGNED>(p1, s * S + kg * E, d));
        // lane: query i * 16 + (lane & 15), rows 4 (lane >> 4) + 0 .. 3 of either half
        const int valid = (int)(n - tile * 32 < 32 ? n - tile * 32 : 32);
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (h * 16 + kg * 4 + r < valid) top = fmaxf(top, acc[h][i][r]);
            if (top > m[i]) {
                if (m[i] > -INFINITY) {
                    const float down = (m[i] - top) * c2, f = __builtin_amdgcn_exp2f(down);
                    t[i] = f * __fmaf_rn(l[i], down, t[i]);
                    l[i] *= f;
                }
                m[i] = top;
            }
            const float shift = m[i] > -INFINITY ? -(m[i] * c2) : 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (h * 16 + kg * 4 + r < valid) {
                        const float s2 = __fmaf_rn(acc[h][i][r], c2, shift), e = __builtin_amdgcn_exp2f(s2);
                        l[i] += e;
                        t[i] = __fmaf_rn(e, s2, t[i]);
                    }
            if (gmax) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                if (kg == 0 && q0 + i * 16 + r16 < nq) gmax[(int64_t)(q0 + i * 16 + r16) * gstride + tile] = top;
            }
        }
    }
    // the four lanes of a query, then the waves
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        Stat a{m[i] > -INFINITY ? m[i] * c2 : -INFINITY, l[i], t[i]};
#pragma unroll
        for (int x16 = 16; x16 < 64; x16 *= 2) a = join(a, Stat{__shfl_xor(a.m, x16, 64), __shfl_xor(a.l, x16, 64), __shfl_xor(a.t, x16, 64)});
        if (kg == 0) joined[wave][i * 16 + r16] = make_float4(a.m, a.l, a.t, 0.0f);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < QT * 16; i += kStreamThreads) {
        if (q0 + i >= nq) continue;
        Stat a{joined[0][i].x, joined[0][i].y, joined[0][i].z};
        for (int w = 1; w < kStreamWaves; ++w) a = join(a, Stat{joined[w][i].x, joined[w][i].y, joined[w][i].z});
        stats[(size_t)blockIdx.x * nq + q0 + i] = make_float4(a.m, a.l, a.t, 0.0f);
    }
}

// ---- many queries: tiles of a matrix product ----------------------------------------------------

// Statistics of 128 queries over a part of the rows, 256 rows at a time; a lane has two queries, 64 of a tile's rows of each.
// X: the launch's rows, Q: all queries, negated where the scale is.
template <class H, int TERMS, bool BEST>
__global__ __launch_bounds__(kTileThreads, 2) void prob_tile_kernel(Rows16 X, Rows16 Q, int halves, float c2, const Largest *__restrict__ largest, const float *__restrict__ q_inv, int parts,
                                                                    int others, float4 *__restrict__ stats, float *__restrict__ gmax, int64_t gstride)
{
    extern __shared__ char lds[];
    const Place place = place_of(blockIdx.x, others);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles = (X.rows + kTileM - 1) / kTileM;
    int64_t first;
    int count;
    part_tiles(tiles, parts, place.part, &first, &count);
    const int64_t q0 = (int64_t)place.other * kTileN;
    float cq[2], m[2], l[2], t[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        cq[j] = c2;
        if (TERMS > 1) {
            const int64_t q = min(q0 + acc_col(j), Q.rows - 1);
            cq[j] = c2 * q_inv[q] * (1.0f / range_scale(largest->points));
        }
        m[j] = -INFINITY;
        l[j] = t[j] = 0.0f;
    }
    run_tiles<H, TERMS, BEST, RowCopies>(X, Q, halves, count, lds, [&](int i, RowCopies &c) { c.seek(X, (first + i) * kTileM, Q, q0); },
        [&](int i, f32x16 (&acc)[4][2]) {
            const int64_t row0 = (first + i) * kTileM;
            const bool whole = row0 + kTileM <= X.rows;
            const int valid = whole ? kTileM : (int)(X.rows - row0);
            auto take = [&](auto tail) {
                constexpr bool TAIL = decltype(tail)::value;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float group[4];
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        float g = -INFINITY;
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (!TAIL || acc_row(a, r) < valid) g = fmaxf(g, acc[a][j][r]);
                        group[a] = g;
                    }
                    const float top = fmaxf(fmaxf(group[0], group[1]), fmaxf(group[2], group[3]));
                    if (top > m[j]) {
                        if (m[j] > -INFINITY) {
                            const float down = (m[j] - top) * cq[j], f = __builtin_amdgcn_exp2f(down);
                            t[j] = f * __fmaf_rn(l[j], down, t[j]);
                            l[j] *= f;
                        }
                        m[j] = top;
                    }
                    const float shift = m[j] > -INFINITY ? -(m[j] * cq[j]) : 0.0f;
                    // four sums side by side, then one
                    float ls[4] = {}, ts[4] = {};
#pragma unroll
                    for (int a = 0; a < 4; ++a)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (!TAIL || acc_row(a, r) < valid) {
                                const float s2 = __fmaf_rn(acc[a][j][r], cq[j], shift), e = __builtin_amdgcn_exp2f(s2);
                                ls[a] += e;
                                ts[a] = __fmaf_rn(e, s2, ts[a]);
                            }
                    l[j] += (ls[0] + ls[1]) + (ls[2] + ls[3]);
                    t[j] += (ts[0] + ts[1]) + (ts[2] + ts[3]);
                    if (BEST) {
#pragma unroll
                        for (int a = 0; a < 4; ++a) group[a] = fmaxf(group[a], __shfl_xor(group[a], 32, 64));
                        const int64_t q = q0 + acc_col(j);
                        if (lane < 32 && q < Q.rows)
                            *(float4 *)(gmax + q * gstride + (first + i) * (kTileM / 32) + (wave >> 1) * 4) = make_float4(group[0], group[1], group[2], group[3]);
                    }
                }
            };
            if (whole) take(std::false_type{});
            else take(std::true_type{});
        });
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        Stat a{m[j] > -INFINITY ? m[j] * cq[j] : -INFINITY, l[j], t[j]};
        a = join(a, Stat{__shfl_xor(a.m, 32, 64), __shfl_xor(a.l, 32, 64), __shfl_xor(a.t, 32, 64)});
        const int64_t q = q0 + acc_col(j);
        if (lane < 32 && q < Q.rows) stats[(size_t)(place.part * 2 + (wave >> 1)) * Q.rows + q] = make_float4(a.m, a.l, a.t, 0.0f);
    }
}

// ---- what a query's statistics give ----------------------------------------------------------

constexpr int kFinishThreads = 512, kFinishWaves = kFinishThreads / 64;

__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f); // (-0 is 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// <q, x> by 16 lanes (fp32, in a fixed order); every lane of the group gets it
template <class T>
__device__ __forceinline__ float dot16(const float *__restrict__ qf, const T *__restrict__ row, int d, int lane16)
{
    constexpr int E = kFragElems<T>;
    float s = 0.0f;
    for (int k = lane16 * E; k < d; k += 16 * E) {
        const Frag f = load_frag<T, false>(row, k, d);
        T e[E];
        __builtin_memcpy(e, &f, 16);
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (k + j < d) s = __fmaf_rn(qf[k + j], to_f32(e[j]), s);
    }
    return group_sum<16>(s);
}

// A workgroup a query: joins the statistics, scores the given rows and the best ones.
template <class T>
__global__ __launch_bounds__(kFinishThreads) void prob_finish_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, int nq, int64_t ld_q, float scale,
                                                                     const float4 *__restrict__ stats, int parts, const int32_t *__restrict__ ids, int given,
                                                                     float *__restrict__ logp_out, float *__restrict__ lse_out, float *__restrict__ entropy_out,
                                                                     const float *__restrict__ gmax, int64_t gstride, int k, int32_t *__restrict__ alt_ids, float *__restrict__ alt_logp)
{
    __shared__ WgSelectScratch sel;
    __shared__ Stat wave_stat[kFinishWaves];
    __shared__ uint32_t list_count;
    extern __shared__ char lds[];
    float *qf = (float *)lds;                                       // [d]
    u64 *keys = (u64 *)(lds + (((size_t)d * 4 + 15) & ~(size_t)15)); // [32 k] scores of the listed groups' rows
    u64 *best = keys + 32 * (size_t)k;                               // [k]
    uint32_t *groups = (uint32_t *)(best + k);                       // [k]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x;
    for (int c = tid; c < d; c += kFinishThreads) qf[c] = to_f32(q[(int64_t)row * ld_q + c]);
    Stat a{-INFINITY, 0.0f, 0.0f};
    for (int p = tid; p < parts; p += kFinishThreads) {
        const float4 v = stats[(size_t)p * nq + row];
        a = join(a, Stat{v.x, v.y, v.z});
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) a = join(a, Stat{__shfl_xor(a.m, w, 64), __shfl_xor(a.l, w, 64), __shfl_xor(a.t, w, 64)});
    if (lane == 0) wave_stat[wave] = a;
    __syncthreads();
    a = wave_stat[0];
    for (int w = 1; w < kFinishWaves; ++w) a = join(a, wave_stat[w]);
    constexpr float ln2 = 0.693147180559945309f;
    const float log_l = logf(a.l), lse = __fmaf_rn(a.m, ln2, log_l);
    if (tid == 0) {
        lse_out[row] = lse;
        if (entropy_out) entropy_out[row] = log_l - ln2 * (a.t / a.l);
    }
    const int sub = tid >> 4, subs = kFinishThreads / 16, lane16 = tid & 15;
    for (int j = sub; j < given; j += subs) {
        const int32_t id = ids[(int64_t)row * given + j];
        const bool real = id >= 0 && (int64_t)id < n;
        const float s = real ? dot16<T>(qf, x + (int64_t)id * ld_x, d, lane16) * scale : 0.0f;
        if (lane16 == 0) logp_out[(int64_t)row * given + j] = real ? s - lse : -INFINITY;
    }
    if (k == 0) return;

    const uint32_t n_groups = (uint32_t)((n + 31) / 32);
    if (tid == 0) list_count = 0;
    auto group_key = [&](uint32_t g) { return ((u64)order_of(gmax[row * gstride + g]) << 32) | (u64)(0xffffffffu - g); };
    const u64 least = wg_select_threshold_of([&](auto &&fn) { for (uint32_t g = tid; g < n_groups; g += kFinishThreads) fn(group_key(g)); }, k, &sel);
    __syncthreads();
    for (uint32_t g = tid; g < n_groups; g += kFinishThreads)
        if (group_key(g) >= least) {
            const uint32_t at = atomicAdd(&list_count, 1u); // (the order of the list does not matter)
            if (at < (uint32_t)k) groups[at] = g;
        }
    __syncthreads();
    const uint32_t rows = min(list_count, (uint32_t)k) * 32u;
    for (uint32_t i = sub; i < rows; i += subs) {
        const int64_t id = (int64_t)groups[i / 32] * 32 + (i & 31);
        u64 key = 0;
        if (id < n) {
            const float s = dot16<T>(qf, x + id * ld_x, d, lane16) * scale;
            key = ((u64)order_of(s) << 32) | (u64)(0xffffffffu - (uint32_t)id);
        }
        if (lane16 == 0) keys[i] = key;
    }
    if (tid == 0) list_count = 0;
    __syncthreads();
    const u64 kth = wg_select_threshold_of([&](auto &&fn) { for (uint32_t i = tid; i < rows; i += kFinishThreads) if (keys[i]) fn(keys[i]); }, k, &sel);
    __syncthreads();
    for (uint32_t i = tid; i < rows; i += kFinishThreads)
        if (keys[i] && keys[i] >= kth) {
            const uint32_t at = atomicAdd(&list_count, 1u);
            if (at < (uint32_t)k) best[at] = keys[i];
        }
    __syncthreads();
    const uint32_t found = min(list_count, (uint32_t)k);
    for (uint32_t i = tid; i < found; i += kFinishThreads) {
        const u64 mine = best[i];
        uint32_t rank = 0;
        for (uint32_t o = 0; o < found; ++o) rank += best[o] > mine;
        alt_ids[(int64_t)row * k + rank] = (int32_t)(0xffffffffu - (uint32_t)mine);
        alt_logp[(int64_t)row * k + rank] = value_of((uint32_t)(mine >> 32)) - lse;
    }
}

// ---- launches ----------------------------------------------------------------------------------

// Workgroups that share the rows of the stream.
static int stream_groups(int64_t n, int query_tiles)
{
    const int64_t tiles = (n + 31) / 32, most = std::max(1, 1024 / query_tiles);
    return (int)std::max<int64_t>(1, std::min<int64_t>((tiles + kStreamWaves - 1) / kStreamWaves, most));
}

// Query tiles of 16 that a workgroup takes: as many as fit LDS beside another workgroup's, at most 4 (64 queries).
static int stream_tile(int type, int d, int nq)
{
    const size_t step = 64 * sizeof(Frag), bytes = step * (size_t)((d * type_bytes(type) + 63) / 64);
    int qt = 1;
    while (qt < 4 && qt * 16 < nq && 2 * qt * bytes <= 80 * 1024) qt *= 2;
    return qt;
}

// From how many queries on the tiles take over: up to 64 the stream reads the rows once.
static bool by_tiles(int nq) { return nq > 64; }

constexpr int kTileGroups = 512; // two workgroups a compute unit
constexpr size_t kPackBytes = (size_t)1 << 30; // most that packed rows take at a time

struct ProbScratch {
    float4 *stats; float *gmax; int64_t gstride;
    int groups, qt, query_tiles;                         // stream
    bool pack; int width, parts, launches; int64_t part; // tiles: rows a launch
    uint16_t *x16, *q16; int64_t x_plane, q_plane; float *q_inv; Largest *largest;
    size_t bytes;
};

static ProbScratch prob_scratch(const ProbParams &p, void *base)
{
    ProbScratch s{};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *q = base ? (char *)base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return q;
    };
    s.gstride = (p.n + kTileM - 1) / kTileM * (kTileM / 32);
    if (!by_tiles(p.nq)) {
        s.qt = stream_tile(p.type, p.d, p.nq);
        s.query_tiles = (p.nq + 16 * s.qt - 1) / (16 * s.qt);
        s.groups = stream_groups(p.n, s.query_tiles);
        s.stats = (float4 *)take((size_t)s.groups * p.nq * sizeof(float4));
    } else {
        const int planes = p.type == AVQ_F32 ? 2 : 1;
        s.width = (p.d + 31) / 32 * 32;
        // (base == NULL: the size for rows that need packing, whatever their place and stride)
        s.pack = !base || p.type == AVQ_F32 || s.width != p.d || (uintptr_t)p.points % 16 != 0 || p.ld_points % 8 != 0;
        s.part = p.n;
        if (s.pack) s.part = std::min<int64_t>(p.n, std::max<int64_t>(65536, (int64_t)(kPackBytes / (2 * planes * (size_t)s.width)) / kTileM * kTileM));
        s.launches = (int)((p.n + s.part - 1) / s.part);
        s.query_tiles = (p.nq + kTileN - 1) / kTileN;
        s.parts = parts_for((s.part + kTileM - 1) / kTileM, s.query_tiles, kTileGroups);
        // (as many statistics with one launch as with several: the number of parts only falls with the rows a launch has)
        s.stats = (float4 *)take((size_t)s.launches * std::max(s.parts, parts_for((p.n + kTileM - 1) / kTileM, s.query_tiles, kTileGroups)) * 2 * p.nq * sizeof(float4));
        s.q_plane = (int64_t)p.nq * s.width;
        s.q16 = (uint16_t *)take((size_t)s.q_plane * 2 * planes);
        s.q_inv = (float *)take((size_t)p.nq * sizeof(float));
        s.largest = (Largest *)take(sizeof(Largest));
        s.x_plane = s.part * s.width;
        if (s.pack) s.x16 = (uint16_t *)take((size_t)s.x_plane * 2 * planes);
    }
    s.gmax = p.k > 0 ? (float *)take((size_t)s.gstride * p.nq * sizeof(float)) : nullptr;
    s.bytes = at;
    return s;
}

size_t log_probs_scratch_bytes(int type, int64_t n, int d, int nq, int given, int k)
{
    (void)given;
    ProbParams p{};
    p.type = type; p.n = n; p.d = d; p.nq = nq; p.k = k;
    return nq == 0 ? 0 : prob_scratch(p, nullptr).bytes;
}

template <class T, int QT, bool ALIGNED, bool QLDS>
static int stream_run(const ProbParams &p, const ProbScratch &s, hipStream_t st)
{
    static LdsLimitOnce once;
    const size_t lds = QLDS ? (size_t)QT * 64 * sizeof(Frag) * ((p.d + kStepElems<T> - 1) / kStepElems<T>) : 0;
    AVQ_TRY(set_lds_limit((const void *)prob_stream_kernel<T, QT, ALIGNED, QLDS>, kMaxDynLds - sizeof(float4) * kStreamWaves * 64, &once));
    const float c2 = fabsf(p.scale) * 1.44269504088896341f;
    prob_stream_kernel<T, QT, ALIGNED, QLDS><<<dim3(s.groups, s.query_tiles), dim3(kStreamThreads), lds, st>>>(
        (const T *)p.points, p.n, p.d, p.ld_points, (const T *)p.queries, p.nq, p.ld_queries, c2, p.scale < 0.0f, s.stats, s.gmax, s.gstride);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool ALIGNED>
static int stream_sized(const ProbParams &p, const ProbScratch &s, hipStream_t st)
{
    // beyond what LDS holds for 16 queries (10,000 bytes a query), the queries' operands come from the caches
    if ((size_t)p.d * sizeof(T) > 8192) return stream_run<T, 1, ALIGNED, false>(p, s, st);
    if (s.qt == 1) return stream_run<T, 1, ALIGNED, true>(p, s, st);
    return s.qt == 2 ? stream_run<T, 2, ALIGNED, true>(p, s, st) : stream_run<T, 4, ALIGNED, true>(p, s, st);
}

template <class H, int TERMS>
static int tiles_run(const ProbParams &p, const ProbScratch &s, hipStream_t st)
{
    const int size = type_bytes(p.type);
    const float c2 = fabsf(p.scale) * 1.44269504088896341f;
    AVQ_TRY(launch_pack_rows(p.queries, p.type, p.nq, p.d, p.ld_queries, p.nq, s.width, s.q16, s.q_plane, nullptr, s.q_inv, p.scale < 0.0f, st));
    if (TERMS > 1) {
        AVQ_TRY(launch_clear_largest(s.largest, st));
        AVQ_TRY(launch_largest((const float *)p.points, p.n, p.d, p.ld_points, &s.largest->points, st));
    }
    static LdsLimitOnce with_best, without;
    const Rows16 Q{s.q16, s.width, s.q_plane, p.nq};
    for (int i = 0; i < s.launches; ++i) {
        const int64_t lo = i * s.part, rows = std::min<int64_t>(s.part, p.n - lo);
        const char *from = (const char *)p.points + lo * p.ld_points * size;
        Rows16 X{(const uint16_t *)from, p.ld_points, 0, rows};
        if (s.pack) {
            AVQ_TRY(launch_pack_rows(from, p.type, rows, p.d, p.ld_points, rows, s.width, s.x16, s.x_plane, &s.largest->points, nullptr, false, st));
            X = Rows16{s.x16, s.width, s.x_plane, rows};
        }
        float4 *stats = s.stats + (size_t)i * s.parts * 2 * p.nq;
        const dim3 grid((unsigned)(s.parts * s.query_tiles));
        if (p.k > 0) {
            AVQ_TRY(set_lds_limit((const void *)prob_tile_kernel<H, TERMS, true>, kTileLds, &with_best));
            prob_tile_kernel<H, TERMS, true><<<grid, dim3(kTileThreads), kTileLds, st>>>(X, Q, (p.d + 15) / 16, c2, s.largest, s.q_inv, s.parts, s.query_tiles, stats,
                                                                                      s.gmax + lo / 32, s.gstride);
        } else {
            AVQ_TRY(set_lds_limit((const void *)prob_tile_kernel<H, TERMS, false>, kTileLds, &without));
            prob_tile_kernel<H, TERMS, false><<<grid, dim3(kTileThreads), kTileLds, st>>>(X, Q, (p.d + 15) / 16, c2, s.largest, s.q_inv, s.parts, s.query_tiles, stats, nullptr, 0);
        }
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

template <class T>
static int log_probs_typed(const ProbParams &p, hipStream_t st)
{
    const ProbScratch s = prob_scratch(p, p.scratch);
    int parts = s.groups;
    if (by_tiles(p.nq)) {
        if constexpr (sizeof(T) == 4) AVQ_TRY((tiles_run<f16_t, 3>(p, s, st)));
        else AVQ_TRY((tiles_run<T, 1>(p, s, st)));
        parts = s.launches * s.parts * 2;
    } else {
        const bool aligned = ((uintptr_t)p.points % 16) == 0 && (p.ld_points * sizeof(T)) % 16 == 0;
        AVQ_TRY(aligned ? (stream_sized<T, true>(p, s, st)) : (stream_sized<T, false>(p, s, st)));
    }
    static LdsLimitOnce once;
    AVQ_TRY(set_lds_limit((const void *)prob_finish_kernel<T>, kFinishLds, &once));
    prob_finish_kernel<T><<<dim3(p.nq), dim3(kFinishThreads), finish_lds(p.d, p.k), st>>>((const T *)p.points, p.n, p.d, p.ld_points, (const T *)p.queries, p.nq, p.ld_queries, p.scale,
                                                                                       s.stats, parts, p.ids, p.given, p.logp, p.lse, p.entropy, s.gmax, s.gstride, p.k, p.alt_ids,
                                                                                       p.alt_logp);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

int launch_log_probs(const ProbParams &p, hipStream_t st)
{
    if (p.nq == 0) return AVQ_OK;
    if (p.type == AVQ_F32) return log_probs_typed<float>(p, st);
    return p.type == AVQ_BF16 ? log_probs_typed<bf16_t>(p, st) : log_probs_typed<f16_t>(p, st);
}

} // namespace avq
