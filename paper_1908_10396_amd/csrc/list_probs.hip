// Log probabilities under a softmax over a list of rows of each query's own, s_tj = c <q_t, x_id_tj> + o_tj, and their gradient:
//   lse_t = log sum_j e^s_tj,  log p_tj = s_tj - lse_t,
//   G_tj = g_tj - p_tj (sum_j g_tj - l_t),  dq_t = c sum_j G_tj x_id_tj,  dx_i = c sum over id_tj = i of G_tj q_t,  do_tj = G_tj.
// Entries whose id is outside [0, n) have no share; neither do entries whose log p is -infinity in the gradient.
//
// Bound by memory: the listed rows are gathered, once for the scores and once more for dq; dx writes the whole table, by the sorted sums of
// the lookup's gradient (embed.hip) with G as weights. A workgroup a query: its scores stay in LDS between the products and the softmax.
#include <math.h>

#include "row_types.h"

namespace avq {

constexpr int kListThreads = 256, kListWaves = kListThreads / 64;

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) v = fmaxf(v, __shfl_xor(v, w, 64));
    return v;
}

// over the workgroup; red: a value a wave
__device__ __forceinline__ float list_max(float v, float *red)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

__device__ __forceinline__ float list_sum(float v, float *red)
{
    v = group_sum<64>(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// log p of a query's m entries from their scores (padding: NaN or anything, by its id), and lse. The sum is kept relative to the largest
// score without the 1 of that itself, so that log p keeps its relative accuracy where p is nearly 1.
__device__ __forceinline__ void list_softmax(const float *scores, const int32_t *__restrict__ ids, int64_t n, int m, float *red, float *logp, float *lse)
{
    float top = -INFINITY;
    for (int j = threadIdx.x; j < m; j += kListThreads) {
        const int32_t id = ids[j];
        if (id >= 0 && (int64_t)id < n) top = fmaxf(top, scores[j]);
    }
    top = list_max(top, red);
    const float base = top > -INFINITY ? top : 0.0f;
    float beside = 0.0f, at_top = 0.0f;
    for (int j = threadIdx.x; j < m; j += kListThreads) {
        const int32_t id = ids[j];
        if (!(id >= 0 && (int64_t)id < n)) continue;
        const float s = scores[j];
        if (s == base) at_top += 1.0f;
        else beside += expf(s - base); // (NaN goes on in the sum)
    }
    beside = list_sum(beside, red);
    at_top = list_sum(at_top, red);
    // (nothing but masks: log p and lse are -infinity; a score of +infinity: no result is a number)
    float sum = top > -INFINITY ? log1pf((at_top - 1.0f) + beside) : beside;
    if (top == INFINITY) sum = NAN;
    const float low = top > -INFINITY ? 0.0f : -INFINITY;
    for (int j = threadIdx.x; j < m; j += kListThreads) {
        const int32_t id = ids[j];
        logp[j] = id >= 0 && (int64_t)id < n ? (scores[j] - base) - sum + low : -INFINITY;
    }
    if (threadIdx.x == 0) *lse = base + sum + low;
}

// The query in LDS in fp32, zeros to a whole unit.
template <class T> __device__ __forceinline__ void list_query(const T *__restrict__ q, int d, float *qs)
{
    const int padded = units_of<T>(d) * kUnit<T>;
    for (int k = threadIdx.x; k < padded; k += kListThreads) qs[k] = k < d ? to_f32(q[k]) : 0.0f;
}

template <class T, bool RAGGED>
__global__ __launch_bounds__(kListThreads) void list_probs_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, int64_t ld_q, float scale,
                                                                  const int32_t *__restrict__ ids, int m, const float *__restrict__ offset, float *__restrict__ logp,
                                                                  float *__restrict__ lse)
{
    extern __shared__ float lds[]; // the query, the scores
    __shared__ float red[kListWaves];
    constexpr int V = kUnit<T>;
    const int per_row = units_of<T>(d), lane = threadIdx.x & 63;
    float *qs = lds, *scores = lds + per_row * V;
    const int64_t t = blockIdx.x;
    ids += t * m;
    list_query(q + t * ld_q, d, qs);
    __syncthreads();
    for (int j = threadIdx.x >> 6; j < m; j += kListWaves) {
        const int32_t id = ids[j];
        const T *row = x + (id >= 0 && (int64_t)id < n ? (int64_t)id * ld_x : 0);
        float s = 0.0f;
        for (int u = lane; u < per_row; u += 64) {
            const Unit<T> v = load_unit<T, RAGGED>(row, u * V, d);
#pragma unroll
            for (int e = 0; e < V; ++e) s = __fmaf_rn(to_f32(v.e[e]), qs[u * V + e], s);
        }
        s = group_sum<64>(s);
        if (lane == 0) scores[j] = offset ? __fmaf_rn(s, scale, offset[t * m + j]) : s * scale;
    }
    __syncthreads();
    list_softmax(scores, ids, n, m, red, logp + t * m, lse + t);
}

// G and dq of a query.
template <class T, bool RAGGED>
__global__ __launch_bounds__(kListThreads) void list_grad_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, float scale, const int32_t *__restrict__ ids, int m,
                                                                 const float *__restrict__ logp, const float *__restrict__ g, const float *__restrict__ g_lse, int lanes,
                                                                 float *__restrict__ dscores, T *__restrict__ dq, int64_t ld_dq)
{
    extern __shared__ float lds[]; // G, the teams' sums of a unit column
    __shared__ float red[kListWaves];
    constexpr int V = kUnit<T>;
    float *G = lds, *sums = lds + m;
    const int64_t t = blockIdx.x;
    ids += t * m;
    float a = 0.0f;
    for (int j = threadIdx.x; j < m; j += kListThreads) {
        const int32_t id = ids[j];
        if (id >= 0 && (int64_t)id < n && !(logp[t * m + j] == -INFINITY)) a += g[t * m + j];
    }
    a = list_sum(a, red);
    if (g_lse) a -= g_lse[t];
    for (int j = threadIdx.x; j < m; j += kListThreads) {
        const int32_t id = ids[j];
        const float lp = logp[t * m + j];
        float v = 0.0f;
        if (id >= 0 && (int64_t)id < n && !(lp == -INFINITY)) {
            const float up = g[t * m + j];
            // (an answer that is nearly certain: 1 - p by itself)
            v = lp > -0.5f ? __fmaf_rn(-a, expm1f(lp), up - a) : __fmaf_rn(-a, expf(lp), up);
        }
        G[j] = v;
        dscores[t * m + j] = v;
    }
    if (!dq) return;
    __syncthreads();
    const int per_row = units_of<T>(d), teams = kListThreads / lanes, team = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    for (int u0 = 0; u0 < per_row; u0 += lanes) {
        const int u = u0 + lane;
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
        if (u < per_row)
            for (int j = team; j < m; j += teams) {
                const float w = G[j];
                if (w == 0.0f) continue; // (padding, and rows of no weight whatever they hold)
                const Unit<T> v = load_unit<T, RAGGED>(x + (int64_t)ids[j] * ld_x, u * V, d);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = __fmaf_rn(w, to_f32(v.e[e]), acc[e]);
            }
#pragma unroll
        for (int e = 0; e < V; ++e) sums[threadIdx.x * V + e] = acc[e];
        __syncthreads();
        if (team == 0 && u < per_row) {
            for (int o = 1; o < teams; ++o)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += sums[(o * lanes + lane) * V + e];
            Unit<T> out;
#pragma unroll
            for (int e = 0; e < V; ++e) out.e[e] = from_f32<T>(acc[e] * scale);
            store_unit<T, RAGGED>(dq + t * ld_dq, u * V, d, out);
        }
        __syncthreads();
    }
}

template <class T, bool RAGGED>
static int list_run(const ListParams &p, hipStream_t st)
{
    static LdsLimitOnce limit;
    AVQ_TRY(set_lds_limit((const void *)list_probs_kernel<T, RAGGED>, kMaxDynLds, &limit));
    const size_t lds = ((size_t)units_of<T>(p.d) * kUnit<T> + p.m) * sizeof(float);
    list_probs_kernel<T, RAGGED><<<dim3(p.nq), dim3(kListThreads), lds, st>>>((const T *)p.points, p.n, p.d, p.ld_points, (const T *)p.queries, p.ld_queries, p.scale, p.ids, p.m,
                                                                           p.offset, p.logp, p.lse);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool RAGGED>
static int list_grad_run(const ListGradParams &p, hipStream_t st)
{
    int lanes = 4;
    while (lanes < kListThreads && lanes < units_of<T>(p.d)) lanes *= 2;
    const size_t lds = ((size_t)p.m + kListThreads * kUnit<T>) * sizeof(float);
    list_grad_kernel<T, RAGGED><<<dim3(p.nq), dim3(kListThreads), lds, st>>>((const T *)p.points, p.n, p.d, p.ld_points, p.scale, p.ids, p.m, p.logp, p.grad_logp, p.grad_lse, lanes,
                                                                          p.dscores, (T *)p.dqueries, p.ld_dqueries);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T>
static int list_typed(const ListParams &p, hipStream_t st)
{
    return whole_units(p.points, p.ld_points, p.d, sizeof(T)) ? list_run<T, false>(p, st) : list_run<T, true>(p, st);
}

template <class T>
static int list_grad_typed(const ListGradParams &p, hipStream_t st)
{
    const bool whole = whole_units(p.points, p.ld_points, p.d, sizeof(T)) && (!p.dqueries || whole_units(p.dqueries, p.ld_dqueries, p.d, sizeof(T)));
    return whole ? list_grad_run<T, false>(p, st) : list_grad_run<T, true>(p, st);
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
    return count == 0 ? 0 : embed_grad_scratch_bytes(n, d, count);
}

int launch_list_grad(const ListGradParams &p, hipStream_t st)
{
    if (p.nq > 0) {
        if (p.type == AVQ_F32) AVQ_TRY(list_grad_typed<float>(p, st));
        else if (p.type == AVQ_BF16) AVQ_TRY(list_grad_typed<bf16_t>(p, st));
        else AVQ_TRY(list_grad_typed<f16_t>(p, st));
    }
    if (!p.dpoints) return AVQ_OK;
    EmbedGradParams rows{p.queries, p.type, p.ld_queries, p.ids, (int64_t)p.nq * p.m, p.scale, p.dpoints, p.n, p.d, p.ld_dpoints, p.accumulate, p.scratch};
    rows.weights = p.dscores;
    rows.per_row = p.m;
    return launch_embed_grad(rows, st);
}

} // namespace avq
