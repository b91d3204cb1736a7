// Log probabilities under a softmax over a list of rows of each query's own, s_tj = c <q_t, x_id_tj> + o_tj, and their gradient:
//   lse_t = log sum_j e^s_tj,  log p_tj = s_tj - lse_t,
//   G_tj = g_tj - p_tj (sum_j g_tj - l_t),  dq_t = c sum_j G_tj x_id_tj,  dx_i = c sum over id_tj = i of G_tj q_t,  do_tj = G_tj.
// Entries whose id is outside [0, n) have no share; neither do entries whose log p is -infinity in the gradient.
//
// Bound by memory: the listed rows are gathered, once for the scores and once more for dq; dx writes the whole table, by the sorted sums of
// the lookup's gradient (embed.hip) with G as weights. A workgroup a query: its scores stay in LDS between the products and the softmax. 2,047 lists of
// 200 rows of 1,024 bf16: 64 us (0.76 GB gathered, 425 MB of it from beyond the L2s at 6.6 TB/s: the 205 MB of different rows twice, since each of eight L2s
// fetches those of its queries; lists of 409,400 different rows fetch 845 MB in 149 us, of 1,500 ones 31 MB in 38). 1,024 lists of 64 different rows of 1,024 fp32, 2,048 bf16,
// 4,096 bf16 and 4,096 fp32: 44, 46, 131 and 186 us, 6.1, 5.8, 4.1 and 5.8 TB/s. 2,048 of 127 rows of 100 fp32, with offsets: 23 for the scores, 161 for the gradient, of
// which zeros for 1,183,514 rows alone are 69.
#include <math.h>

#include "fill_rows.h"
#include "row_types.h"

namespace avq {

constexpr int kListThreads = 256, kListWaves = kListThreads / 64;

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) v = fmaxf(v, __shfl_xor(v, w, 64));
    return v;
}

// over the workgroup of a query, a wave or four; red: a value a wave
template <int THREADS> __device__ __forceinline__ float list_max(float v, float *red)
{
    v = wave_max(v);
    if (THREADS == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

template <int THREADS> __device__ __forceinline__ float list_sum(float v, float *red)
{
    v = group_sum<64>(v);
    if (THREADS == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// A few queries with long lists: a workgroup takes a part of a query's list, so that there are a thousand of them, 32 entries at
// least (2,986 rows of 813 fp32 for one query: 15 us, by 64 entries 25).
constexpr int kListGroups = 1024, kListPart = 32;
constexpr int kListWhole = 128; // a list that is not worth a second launch
struct ListParts { int parts, each; };
__host__ __device__ inline ListParts list_parts(int nq, int m)
{
    const int most = (m + kListPart - 1) / kListPart, want = (kListGroups + nq - 1) / nq;
    const int parts = want < most ? want : most;
    if (m <= kListWhole || parts <= 1) return ListParts{1, m};
    const int each = (m + parts - 1) / parts;
    return ListParts{(m + each - 1) / each, each};
}

// log p of a query's m entries from their scores, and lse. The sum is kept relative to the largest score without the 1
// of that itself, so that log p keeps its relative accuracy where p is nearly 1. By THREADS threads, EACH entries a thread in registers.
template <int THREADS, int EACH>
__device__ __forceinline__ void list_softmax(const float *scores, const int32_t *ids, int64_t n, int m, float *red, float *logp, float *lse)
{
    float s[EACH], top = -INFINITY;
    int32_t id[EACH];
    bool real[EACH];
    if (m > 0) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int j = min((int)threadIdx.x + i * THREADS, m - 1); // (an entry always, so that no load waits for a branch)
            id[i] = ids[j];
            s[i] = scores[j];
        }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        real[i] = (int)threadIdx.x + i * THREADS < m && id[i] >= 0 && (int64_t)id[i] < n;
        if (real[i]) top = fmaxf(top, s[i]);
    }
    top = list_max<THREADS>(top, red);
    const float base = top > -INFINITY ? top : 0.0f;
    float beside = 0.0f, at_top = 0.0f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (!real[i]) continue;
        if (s[i] == base) at_top += 1.0f;
        else beside += expf(s[i] - base); // (NaN goes on in the sum)
    }
    beside = list_sum<THREADS>(beside, red);
    at_top = list_sum<THREADS>(at_top, red);
    // (nothing but masks: log p and lse are -infinity; a score of +infinity: no result is a number)
    float sum = top > -INFINITY ? log1pf((at_top - 1.0f) + beside) : beside;
    if (top == INFINITY) sum = NAN;
    const float low = top > -INFINITY ? 0.0f : -INFINITY;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int j = threadIdx.x + i * THREADS;
        if (j < m) logp[j] = real[i] ? (s[i] - base) - sum + low : -INFINITY;
    }
    if (threadIdx.x == 0) *lse = base + sum + low;
}

// Lists of up to kListFused get their softmax from the workgroup that scored them, longer ones and those in parts from list_softmax_kernel: its
// sixteen entries a thread would cost the gather registers, and with them loads in flight. One wave does lists of up to 256: no barrier, and the
// other waves make room for the next query's.
constexpr int kListFused = 1024;
__device__ __forceinline__ void list_softmax_fused(const float *scores, const int32_t *ids, int64_t n, int m, float *red, float *logp, float *lse)
{
    if (m <= 256) {
        if (threadIdx.x < 64) list_softmax<64, 4>(scores, ids, n, m, red, logp, lse);
    } else {
        list_softmax<kListThreads, 4>(scores, ids, n, m, red, logp, lse);
    }
}

// a mask is one whatever the row holds
__device__ __forceinline__ float list_score(float product, float scale, float offset) { return offset == -INFINITY ? -INFINITY : __fmaf_rn(product, scale, offset); }

// ids of a part in LDS, -1 for padding
template <int THREADS> __device__ __forceinline__ void list_ids(const int32_t *__restrict__ ids, int64_t n, int count, int32_t *to)
{
    for (int j = threadIdx.x; j < count; j += THREADS) {
        const int32_t id = ids[j];
        to[j] = id >= 0 && (int64_t)id < n ? id : -1;
    }
}

// acc + the inner product of two units. 16-bit elements two at a time, their products exact and two roundings at most a pair; subnormal elements count.
__device__ __forceinline__ float unit_product(const Unit<float> &a, const Unit<float> &b, float acc)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __fmaf_rn(a.e[e], b.e[e], acc);
    return acc;
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
struct Pairs { uint32_t w[4]; };
__device__ __forceinline__ float unit_product(const Unit<bf16_t> &a, const Unit<bf16_t> &b, float acc)
{
    const Pairs x = __builtin_bit_cast(Pairs, a), y = __builtin_bit_cast(Pairs, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x.w[e]), __builtin_bit_cast(bf16x2, y.w[e]), acc, false);
    return acc;
}
__device__ __forceinline__ float unit_product(const Unit<f16_t> &a, const Unit<f16_t> &b, float acc)
{
    const Pairs x = __builtin_bit_cast(Pairs, a), y = __builtin_bit_cast(Pairs, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x.w[e]), __builtin_bit_cast(f16x2, y.w[e]), acc, false);
    return acc;
}

// Scores of a part of a query's list, and where that is all of it the softmax. A row lies across L lanes that hold NV units of it each, and of
// the query; eight loads at a time a lane.
template <class T, bool RAGGED, int L, int NV, int THREADS>
__global__ __launch_bounds__(THREADS, NV == 4 || (RAGGED && (NV == 2 || sizeof(T) == 2)) ? 4 : 8) void list_probs_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, int64_t ld_q, float scale,
                                                                  const int32_t *__restrict__ ids, int m, int parts, int each, const float *__restrict__ offset,
                                                                  float *__restrict__ logp, float *__restrict__ lse)
{
    extern __shared__ int32_t lds[]; // the part's ids and scores
    __shared__ float red[kListWaves];
    constexpr int V = kUnit<T>, kTeams = THREADS / L, kRows = NV == 1 ? 8 : 4;
    const int per_row = units_of<T>(d), lane = threadIdx.x % L, team = threadIdx.x / L;
    const int64_t t = blockIdx.x / (uint32_t)parts;
    const int first = (int)(blockIdx.x - (uint32_t)t * parts) * each, count = min(each, m - first);
    int32_t *listed = lds;
    float *scores = (float *)(lds + each);
    list_ids<THREADS>(ids + t * m + first, n, count, listed);
    Unit<T> qv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int u = lane + i * L;
        qv[i] = Unit<T>{};
        if (u < per_row) qv[i] = load_unit<T, true>(q + t * ld_q, u * V, d);
    }
    __syncthreads();
    for (int j0 = 0; j0 < count; j0 += kTeams * kRows) {
        Unit<T> v[kRows][NV];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int j = j0 + r * kTeams + team, id = j < count ? max(listed[j], 0) : 0; // (a row always, so that no load waits for a branch)
            const T *row = x + (int64_t)id * ld_x;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int u = lane + i * L;
                v[r][i] = load_unit<T, RAGGED>(row, (u < per_row ? u : 0) * V, d);
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int j = j0 + r * kTeams + team;
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (lane + i * L < per_row) s = unit_product(v[r][i], qv[i], s);
            }
            s = group_sum<L>(s);
            if (lane == 0 && j < count) scores[j] = s;
        }
    }
    __syncthreads();
    const int64_t at = t * m + first;
    const bool fused = parts == 1 && m <= kListFused;
    for (int j = threadIdx.x; j < count; j += THREADS) {
        const float s = offset ? list_score(scores[j], scale, offset[at + j]) : scores[j] * scale;
        if (fused) scores[j] = s;
        else logp[at + j] = s;
    }
    if (!fused) return;
    __syncthreads();
    if (THREADS == 64) list_softmax<64, 1>(scores, listed, n, m, red, logp + at, lse + t); // (lists of up to 64)
    else list_softmax_fused(scores, listed, n, m, red, logp + at, lse + t);
}

// The same for rows that registers do not hold: a wave a row, the query in LDS.
template <class T, bool RAGGED>
__global__ __launch_bounds__(kListThreads) void list_probs_long_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, int64_t ld_q, float scale,
                                                                       const int32_t *__restrict__ ids, int m, int parts, int each, const float *__restrict__ offset,
                                                                       float *__restrict__ logp, float *__restrict__ lse)
{
    extern __shared__ int32_t lds[]; // the part's ids and scores, the query in fp32, zeros to a whole unit
    __shared__ float red[kListWaves];
    constexpr int V = kUnit<T>;
    const int per_row = units_of<T>(d), lane = threadIdx.x & 63;
    const int64_t t = blockIdx.x / (uint32_t)parts;
    const int first = (int)(blockIdx.x - (uint32_t)t * parts) * each, count = min(each, m - first);
    int32_t *listed = lds;
    float *scores = (float *)(lds + each), *qs = scores + each;
    list_ids<kListThreads>(ids + t * m + first, n, count, listed);
    for (int k = threadIdx.x; k < per_row * V; k += kListThreads) qs[k] = k < d ? to_f32(q[t * ld_q + k]) : 0.0f;
    __syncthreads();
    const int64_t at = t * m + first;
    const bool fused = parts == 1 && m <= kListFused;
    for (int j = threadIdx.x >> 6; j < count; j += kListWaves) {
        const T *row = x + (int64_t)max(listed[j], 0) * ld_x;
        float s = 0.0f;
#pragma unroll 4
        for (int u = lane; u < per_row; u += 64) {
            const Unit<T> v = load_unit<T, RAGGED>(row, u * V, d);
#pragma unroll
            for (int e = 0; e < V; ++e) s = __fmaf_rn(to_f32(v.e[e]), qs[u * V + e], s);
        }
        s = group_sum<64>(s);
        if (lane == 0) {
            s = offset ? list_score(s, scale, offset[at + j]) : s * scale;
            if (fused) scores[j] = s;
            else logp[at + j] = s;
        }
    }
    if (!fused) return;
    __syncthreads();
    list_softmax_fused(scores, listed, n, m, red, logp + at, lse + t);
}

// Scores in logp, a workgroup a query, in place.
__global__ __launch_bounds__(kListThreads) void list_softmax_kernel(const int32_t *__restrict__ ids, int64_t n, int m, float *logp, float *lse)
{
    __shared__ float red[kListWaves];
    const int64_t t = blockIdx.x;
    if (m <= 4 * kListThreads) list_softmax<kListThreads, 4>(logp + t * m, ids + t * m, n, m, red, logp + t * m, lse + t);
    else list_softmax<kListThreads, 16>(logp + t * m, ids + t * m, n, m, red, logp + t * m, lse + t);
}

// Sums of `count` weighted rows, by all of the workgroup: a row's units lie across `lanes` lanes, kAhead rows at a time a team of them, then the
// teams' sums in order. row(j), weight(j): of the j-th (a readable row always); finish(u, acc): once for each unit, by the first team. A weight of 0 adds
// nothing, whatever its row holds. Units [from, to) of the rows.
template <class T, bool RAGGED, int THREADS, class RowOf, class WeightOf, class Finish>
__device__ __forceinline__ void weighted_rows(int count, int d, int from, int to, int lanes, float *sums, RowOf row, WeightOf weight, Finish finish)
{
    constexpr int V = kUnit<T>, kAhead = 8;
    const int per_row = to, teams = THREADS / lanes, team = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    for (int u0 = from; u0 < per_row; u0 += lanes) {
        const int u = u0 + lane;
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
        if (u < per_row)
            for (int j0 = team; j0 < count; j0 += teams * kAhead) {
                Unit<T> v[kAhead];
                float w[kAhead];
#pragma unroll
                for (int r = 0; r < kAhead; ++r) {
                    const int j = min(j0 + r * teams, count - 1);
                    w[r] = j0 + r * teams < count ? weight(j) : 0.0f;
                    v[r] = load_unit<T, RAGGED>(row(j), u * V, d);
                }
#pragma unroll
                for (int r = 0; r < kAhead; ++r)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] = w[r] != 0.0f ? __fmaf_rn(w[r], to_f32(v[r].e[e]), acc[e]) : acc[e];
            }
        if (teams > 1) {
#pragma unroll
            for (int e = 0; e < V; ++e) sums[threadIdx.x * V + e] = acc[e];
            __syncthreads();
        }
        if (team == 0 && u < per_row) {
            for (int o = 1; o < teams; ++o)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += sums[(o * lanes + lane) * V + e];
            finish(u, acc);
        }
        if (teams > 1) __syncthreads();
    }
}

// G of a part of a query's list, and what its rows add to dq: dq itself where the part is the list, else sums for list_join.
template <class T, bool RAGGED, int THREADS>
__global__ __launch_bounds__(THREADS) void list_grad_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, float scale, const int32_t *__restrict__ ids, int m, int parts,
                                                                 int each, const float *__restrict__ logp, const float *__restrict__ g, const float *__restrict__ g_lse, int lanes,
                                                                 float *__restrict__ dscores, T *__restrict__ dq, int64_t ld_dq, float *__restrict__ partial, unsigned own, FillJob fill)
{
    if (blockIdx.x >= own) { fill_rows(fill, blockIdx.x - own, gridDim.x - own); return; }
    extern __shared__ int32_t lds[]; // the part's ids and G, the teams' sums of a unit column
    __shared__ float red[kListWaves];
    constexpr int V = kUnit<T>;
    const int64_t t = blockIdx.x / (uint32_t)parts;
    const int part = (int)(blockIdx.x - (uint32_t)t * parts), first = part * each, count = min(each, m - first);
    int32_t *listed = lds;
    float *G = (float *)(lds + each), *sums = G + each;
    ids += t * m;
    logp += t * m;
    g += t * m;
    float a = 0.0f;
    for (int j0 = threadIdx.x; j0 < m; j0 += 4 * THREADS) {
        int32_t id[4];
        float lp[4], up[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = min(j0 + i * THREADS, m - 1); // (an entry always, so that no load waits for a branch)
            id[i] = ids[j];
            lp[i] = logp[j];
            up[i] = g[j];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j0 + i * THREADS < m && id[i] >= 0 && (int64_t)id[i] < n && !(lp[i] == -INFINITY)) a += up[i];
    }
    a = list_sum<THREADS>(a, red);
    if (g_lse) a -= g_lse[t];
    for (int j = threadIdx.x; j < count; j += THREADS) {
        const int32_t id = ids[first + j];
        const float lp = logp[first + j], up = g[first + j];
        float v = 0.0f;
        if (id >= 0 && (int64_t)id < n && !(lp == -INFINITY)) {
            // (an answer that is nearly certain: 1 - p by itself)
            v = lp > -0.5f ? __fmaf_rn(-a, expm1f(lp), up - a) : __fmaf_rn(-a, expf(lp), up);
        }
        listed[j] = v == 0.0f ? 0 : id; // (a row of no weight is read as row 0 and left out, whatever it holds)
        G[j] = v;
        dscores[t * m + first + j] = v;
    }
    if (!dq) return;
    __syncthreads();
    const int per_row = units_of<T>(d);
    weighted_rows<T, RAGGED, THREADS>(count, d, 0, per_row, lanes, sums, [&](int j) { return x + (int64_t)listed[j] * ld_x; }, [&](int j) { return G[j]; }, [&](int u, const float (&acc)[V]) {
        if (parts == 1) {
            Unit<T> out;
#pragma unroll
            for (int e = 0; e < V; ++e) out.e[e] = from_f32<T>(acc[e] * scale);
            store_unit<T, RAGGED>(dq + t * ld_dq, u * V, d, out);
        } else {
            Pack<float, V> out;
#pragma unroll
            for (int e = 0; e < V; ++e) out.e[e] = acc[e];
            *(Pack<float, V> *)(partial + ((t * parts + part) * per_row + u) * V) = out;
        }
    });
}

// 64 units of dq of a query from its parts' sums, by all of the workgroup: its waves take the parts in turns, and their sums are added in order.
template <class T, bool RAGGED>
__device__ __forceinline__ void list_join(const float *__restrict__ partial, int64_t t, int u0, int parts, int d, float scale, T *__restrict__ dq, int64_t ld_dq, float *sums)
{
    constexpr int V = kUnit<T>;
    const int per_row = units_of<T>(d), lane = threadIdx.x & 63, wave = threadIdx.x >> 6, u = u0 + lane;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.0f;
    if (u < per_row) {
#pragma unroll 8
        for (int p = wave; p < parts; p += kListWaves) {
            const Pack<float, V> v = *(const Pack<float, V> *)(partial + ((t * parts + p) * per_row + u) * V);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += v.e[e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) sums[threadIdx.x * V + e] = acc[e];
    __syncthreads();
    if (wave != 0 || u >= per_row) return;
    Unit<T> out;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        for (int w = 1; w < kListWaves; ++w) acc[e] += sums[(w * 64 + lane) * V + e];
        out.e[e] = from_f32<T>(acc[e] * scale);
    }
    store_unit<T, RAGGED>(dq + t * ld_dq, u * V, d, out);
}

template <class T, bool RAGGED>
__global__ __launch_bounds__(kListThreads) void list_join_kernel(const float *__restrict__ partial, int parts, int d, float scale, T *__restrict__ dq, int64_t ld_dq)
{
    __shared__ float sums[kListThreads * kUnit<T>];
    list_join<T, RAGGED>(partial, blockIdx.x, blockIdx.y * 64, parts, d, scale, dq, ld_dq, sums);
}

// dx of a few entries without sorting them: a workgroup an entry and 64 units of its row, which looks for its id among those before, and if it is the
// first adds up all that have it, in their order; the workgroups past the entries join dq. (Forward and gradient of 8 lists of 234 rows of 43 bf16: 33
// us, where sorting, sums and joins take 84.) Every workgroup reads all ids, so that their number is held to 4,096.
constexpr int kListFew = 4096;
__host__ __device__ constexpr int few_lanes(int per_row) { return per_row <= 4 ? 4 : per_row <= 8 ? 8 : per_row <= 16 ? 16 : per_row <= 32 ? 32 : 64; }
static bool few_entries(int64_t count, int per_row) { return count > 0 && count * ((per_row + 63) / 64) <= kListFew; }

template <class T, bool RAGGED>
__global__ __launch_bounds__(kListThreads) void list_few_rows_kernel(const T *__restrict__ q, int64_t ld_q, int d, float scale, const int32_t *__restrict__ ids, int count, int m, int64_t n,
                                                                     const float *__restrict__ G, int blocks, T *__restrict__ dx, int64_t ld_dx, int accumulate,
                                                                     const float *__restrict__ partial, int parts, int per_query, T *__restrict__ dq, int64_t ld_dq)
{
    __shared__ float sums[kListThreads * kUnit<T>];
    __shared__ int listed[kListFew], found[kListWaves];
    if ((int)blockIdx.x >= count * blocks) {
        const int b = blockIdx.x - count * blocks;
        list_join<T, RAGGED>(partial, b / per_query, b % per_query * 64, parts, d, scale, dq, ld_dq, sums);
        return;
    }
    const int i = blockIdx.x / (uint32_t)blocks, block = blockIdx.x % (uint32_t)blocks;
    const int32_t id = ids[i];
    if (id < 0 || (int64_t)id >= n) return;
    constexpr int kEach = kListFew / kListThreads;
    int32_t v[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        if (k * kListThreads >= count) break;
        v[k] = ids[min(k * kListThreads + (int)threadIdx.x, count - 1)]; // (an entry always: no load waits for a branch)
    }
    bool earlier = false;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        if (k * kListThreads >= i) break;
        earlier |= k * kListThreads + (int)threadIdx.x < i && v[k] == id;
    }
    if (__syncthreads_or(earlier)) return;
    int many = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        if (k * kListThreads >= count) break;
        const int j = k * kListThreads + threadIdx.x;
        const bool same = j < count && v[k] == id;
        const u64 which = __ballot(same);
        if ((threadIdx.x & 63) == 0) found[threadIdx.x >> 6] = __popcll(which);
        __syncthreads();
        int at = many + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(which >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)which, 0u));
        for (int w = 0; w < kListWaves; ++w) {
            if (w < (int)(threadIdx.x >> 6)) at += found[w];
            many += found[w];
        }
        if (same) listed[at] = j;
        __syncthreads();
    }
    const int per_row = units_of<T>(d);
    weighted_rows<T, RAGGED, kListThreads>(many, d, block * 64, min(per_row, block * 64 + 64), few_lanes(per_row), sums, [&](int j) { return q + (int64_t)(listed[j] / m) * ld_q; },
                                           [&](int j) { return G[listed[j]]; }, [&](int u, const float (&acc)[kUnit<T>]) {
        write_row<T, RAGGED>(dx + (int64_t)id * ld_dx, u * kUnit<T>, d, acc, scale, accumulate != 0);
    });
}

// Short lists of many queries have a wave each: nothing waits for a barrier, and no wave is left without rows (9,110 lists of 11 rows of 126 f16:
// 16 us, by four waves 43; G and dq 19 and 58).
static bool by_waves(int nq, int m) { return m <= 64 && nq >= 4096; }

template <class T, bool RAGGED, int L, int NV>
static int list_run(const ListParams &p, const ListParts &by, hipStream_t st)
{
    const bool wave = by_waves(p.nq, p.m);
    const auto kernel = wave ? list_probs_kernel<T, RAGGED, L, NV, 64> : list_probs_kernel<T, RAGGED, L, NV, kListThreads>;
    kernel<<<dim3((unsigned)p.nq * by.parts), dim3(wave ? 64 : kListThreads), (size_t)by.each * 8, st>>>(
        (const T *)p.points, p.n, p.d, p.ld_points, (const T *)p.queries, p.ld_queries, p.scale, p.ids, p.m, by.parts, by.each, p.offset, p.logp, p.lse);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool RAGGED>
static int list_run_long(const ListParams &p, const ListParts &by, hipStream_t st)
{
    static LdsLimitOnce limit;
    AVQ_TRY(set_lds_limit((const void *)list_probs_long_kernel<T, RAGGED>, kMaxDynLds, &limit));
    list_probs_long_kernel<T, RAGGED><<<dim3((unsigned)p.nq * by.parts), dim3(kListThreads), (size_t)by.each * 8 + (size_t)units_of<T>(p.d) * kUnit<T> * 4, st>>>(
        (const T *)p.points, p.n, p.d, p.ld_points, (const T *)p.queries, p.ld_queries, p.scale, p.ids, p.m, by.parts, by.each, p.offset, p.logp, p.lse);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool RAGGED>
static int list_scores(const ListParams &p, const ListParts &by, hipStream_t st)
{
    const int per_row = units_of<T>(p.d);
    if (per_row <= 8) return list_run<T, RAGGED, 8, 1>(p, by, st);
    if (per_row <= 16) return list_run<T, RAGGED, 16, 1>(p, by, st);
    if (per_row <= 32) return list_run<T, RAGGED, 32, 1>(p, by, st);
    if (per_row <= 64) return list_run<T, RAGGED, 64, 1>(p, by, st);
    if (per_row <= 128) return list_run<T, RAGGED, 64, 2>(p, by, st);
    if (per_row <= 256) return list_run<T, RAGGED, 64, 4>(p, by, st);
    return list_run_long<T, RAGGED>(p, by, st);
}

template <class T>
static int list_typed(const ListParams &p, hipStream_t st)
{
    const ListParts by = list_parts(p.nq, p.m);
    AVQ_TRY((whole_units(p.points, p.ld_points, p.d, sizeof(T)) ? list_scores<T, false>(p, by, st) : list_scores<T, true>(p, by, st)));
    if (by.parts > 1 || p.m > kListFused) {
        list_softmax_kernel<<<dim3(p.nq), dim3(kListThreads), 0, st>>>(p.ids, p.n, p.m, p.logp, p.lse);
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

// the parts' sums of dq (fp32, rows of whole units), then the scratch of the sorted sums
static size_t list_partial_bytes(int d, int nq, int m)
{
    const ListParts by = list_parts(nq, m);
    return by.parts == 1 ? 0 : ((size_t)nq * by.parts * ((d + 7) / 8 * 8) * sizeof(float) + 255) & ~(size_t)255;
}

template <class T> static bool few_entries(const ListGradParams &p) { return few_entries((int64_t)p.nq * p.m, units_of<T>(p.d)); }

template <class T, bool RAGGED>
static int list_grad_run(const ListGradParams &p, const FillJob &fill, hipStream_t st)
{
    const ListParts by = list_parts(p.nq, p.m);
    const int per_row = units_of<T>(p.d);
    const bool wave = by_waves(p.nq, p.m);
    const int threads = wave ? 64 : kListThreads;
    int lanes = 4;
    while (lanes < threads && lanes < per_row) lanes *= 2;
    const size_t lds = (size_t)by.each * 8 + (size_t)threads * kUnit<T> * sizeof(float);
    const unsigned own = (unsigned)p.nq * by.parts;
    const auto kernel = wave ? list_grad_kernel<T, RAGGED, 64> : list_grad_kernel<T, RAGGED, kListThreads>;
    kernel<<<dim3(own + fill_groups(fill)), dim3(threads), lds, st>>>((const T *)p.points, p.n, p.d, p.ld_points, p.scale, p.ids, p.m, by.parts, by.each, p.logp, p.grad_logp, p.grad_lse, lanes,
                                                                    p.dscores, (T *)p.dqueries, p.ld_dqueries, (float *)p.scratch, own, fill);
    AVQ_HIP(hipGetLastError());
    if (p.dpoints && few_entries<T>(p)) {
        const int blocks = (per_row + 63) / 64, per_query = p.dqueries && by.parts > 1 ? blocks : 0;
        list_few_rows_kernel<T, RAGGED><<<dim3((unsigned)(p.nq * p.m * blocks + p.nq * per_query)), dim3(kListThreads), 0, st>>>(
            (const T *)p.queries, p.ld_queries, p.d, p.scale, p.ids, p.nq * p.m, p.m, p.n, p.dscores, blocks, (T *)p.dpoints, p.ld_dpoints, p.accumulate, (const float *)p.scratch, by.parts,
            per_query, (T *)p.dqueries, p.ld_dqueries);
        AVQ_HIP(hipGetLastError());
    } else if (p.dqueries && by.parts > 1) {
        list_join_kernel<T, RAGGED><<<dim3(p.nq, (per_row + 63) / 64), dim3(kListThreads), 0, st>>>((const float *)p.scratch, by.parts, p.d, p.scale, (T *)p.dqueries, p.ld_dqueries);
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

template <class T>
static int list_grad_typed(const ListGradParams &p, const FillJob &fill, hipStream_t st)
{
    const bool whole = whole_units(p.points, p.ld_points, p.d, sizeof(T)) && (!p.dqueries || whole_units(p.dqueries, p.ld_dqueries, p.d, sizeof(T))) &&
                       (!p.dpoints || !few_entries<T>(p) || (whole_units(p.queries, p.ld_queries, p.d, sizeof(T)) && whole_units(p.dpoints, p.ld_dpoints, p.d, sizeof(T))));
    return whole ? list_grad_run<T, false>(p, fill, st) : list_grad_run<T, true>(p, fill, st);
}

int launch_list_probs(const ListParams &p, hipStream_t st)
{
    if (p.nq == 0) return AVQ_OK;
    if (p.type == AVQ_F32) return list_typed<float>(p, st);
    return p.type == AVQ_BF16 ? list_typed<bf16_t>(p, st) : list_typed<f16_t>(p, st);
}

size_t list_grad_scratch_bytes(int64_t n, int d, int nq, int m)
{
    const int64_t count = (int64_t)nq * m;
    // (fp32 rows have the most units: few entries of theirs are few of any type's)
    return count == 0 ? 0 : list_partial_bytes(d, nq, m) + (few_entries(count, units_of<float>(d)) ? 0 : embed_grad_scratch_bytes(n, d, count));
}

int launch_list_grad(const ListGradParams &p, hipStream_t st)
{
    // the launch that forms dq clears a share of dx too, as those of the sort do, or all of it
    const int size = type_bytes(p.type);
    const int64_t count = (int64_t)p.nq * p.m;
    const bool few = p.type == AVQ_F32 ? few_entries<float>(p) : few_entries<bf16_t>(p);
    FillJob fill{(char *)p.dpoints, 0, 0, p.ld_dpoints * size, (int64_t)p.d * size};
    if (p.dpoints && !p.accumulate && count > 0) fill.hi = few ? p.n : p.n / (1 + embed_grad_launches(p.n, count));
    if (p.nq > 0) {
        if (p.type == AVQ_F32) AVQ_TRY(list_grad_typed<float>(p, fill, st));
        else if (p.type == AVQ_BF16) AVQ_TRY(list_grad_typed<bf16_t>(p, fill, st));
        else AVQ_TRY(list_grad_typed<f16_t>(p, fill, st));
    }
    if (!p.dpoints || few) return AVQ_OK;
    EmbedGradParams rows{p.queries, p.type, p.ld_queries, p.ids, count, p.scale, p.dpoints, p.n, p.d, p.ld_dpoints, p.accumulate,
                         (char *)p.scratch + (p.nq > 0 ? list_partial_bytes(p.d, p.nq, p.m) : 0)};
    rows.weights = p.dscores;
    rows.per_row = p.m;
    rows.cleared = fill.hi;
    return launch_embed_grad(rows, st);
}

} // namespace avq
