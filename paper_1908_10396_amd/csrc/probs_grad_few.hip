// The gradient of the log probabilities of a few queries (G, dq and dx as in probs_grad.hip), in one pass over the rows: one to eight
// queries leave the tiles of the matrix instructions, 256 queries wide, almost empty, while a row that is in registers needs nothing
// else. What a lane's registers hold without spilling comes here (grad_few_takes): fp32 rows of up to 1,024 elements for one and two
// queries, 512 for four, 256 for eight; 16-bit rows of 2,048 for one, 1,024 for two, 512 for four. A row lies across 16, 32 or 64 lanes as units of 16 bytes; its logits are sums over those lanes, G stays in fp32, and the same
// registers then give dx_i = c sum_t G_ti q_t, written at once, and a lane's share of dq_t = c sum_i G_ti x_i, which stays in registers
// until the rows are done: waves, then workgroups, are added in a fixed order. Rows are read once and dx is written once.
// Rows among the given ids are found by a map of 2^16 bits in LDS, which nearly all rows pass by one read; the others look through
// the ids and score their row by the arithmetic of the pass that lse is of.
// 1 - p of a row with nearly all of the probability would have the rounding of lse, 2^-24 |lse| / (1 - p) of it. fp32: the pass also sums
// p over all rows, Z = 1 + delta; to first order p (a + h log p) is too large by delta p (a + h log p + h), which the given rows'
// entries of G get back at the end, in dq and in dx (elsewhere it is a part in millions of what is there). 16-bit types keep that
// rounding: with lse near 20 it reaches a bf16 result's own where 1 - p is below 2^-12, an f16 one's below 2^-9.
// Bound: the rows read and dx written; 16-bit types and eight queries: the arithmetic around them, a lane's registers leaving two
// waves a SIMD. 1,183,514 x 100 fp32 (0.95 GB): 192 us for one query (4.9 TB/s), 199 for two, 238 for four, 484 for eight, where the
// tiles take 905 to 950; 200,000 x 1,024 bf16 (0.82 GB): 179 us for one, 208 for two, the tiles 395. Z and what the given rows get back
// cost 4 to 6 us of an fp32 call.
#include "prob_score.h"
#include "probs.h"
#include "row_types.h"

#include <type_traits>

namespace avq {

constexpr int kFewThreads = 256, kFewWaves = kFewThreads / 64;
constexpr int kFewGroups = 1024; // four workgroups a compute unit, where registers allow it
constexpr int kFewGiven = 1024;  // ids in LDS
constexpr int kFewHeld = 32;     // values of queries that a lane holds, and as many sums
constexpr int kMapWords = 2048;

constexpr int few_ahead(int units, int queries) { return std::max(1, (queries <= 2 ? 4 : 2) / units); } // a lane's rows in flight

struct FewArgs {
    const void *x; int64_t n, ld_x; int d;
    const void *q; int64_t ld_q; int nq; float scale;
    const int32_t *ids; int given; const float *lse, *g, *h, *entropy, *gl;
    void *dx; int64_t ld_dx; int accumulate;
    float *sums;   // [workgroup][NQ][units * V]
    float2 *z;     // [workgroup][NQ] sums of p below 1/4, and of the others (fp32)
    float *shares; // [nq][given] p (a + h log p + h); of a query's equal ids the first has it (fp32)
};

template <class T, bool RAGGED, int L, int NV, int NQ>
__global__ __launch_bounds__(kFewThreads, 2) void grad_few_kernel(FewArgs p)
{
    constexpr int V = kUnit<T>, kPer = 64 / L, U = few_ahead(NV, NQ); // rows a wave has side by side, and in flight
    constexpr int PATH = NQ == 1 ? kByRow : kByStream;                                                   // of the pass that lse is of
    constexpr bool MEND = sizeof(T) == 4;
    extern __shared__ char lds[]; // the queries as that pass multiplies with them; at the end, sums
    __shared__ uint32_t map[kMapWords];
    __shared__ int32_t given_id[kFewGiven];
    __shared__ float given_g[kFewGiven];
    __shared__ float coef[NQ][3]; // a, h and lse
    const int d = p.d, units = units_of<T>(d), wave = threadIdx.x >> 6, lane = threadIdx.x & 63, in_row = lane % L;
    const T *x = (const T *)p.x, *q = (const T *)p.q;
    T *dx = (T *)p.dx;
    const int listed = p.nq * p.given, staged = (d + 31) / 32 * 32;

    for (int i = threadIdx.x; i < kMapWords; i += kFewThreads) map[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < listed; i += kFewThreads) {
        const int32_t id = p.ids[i];
        const bool real = id >= 0 && (int64_t)id < p.n;
        given_id[i] = real ? id : -1;
        given_g[i] = real ? p.g[i] : 0.0f;
        if (MEND && !real && blockIdx.x == 0) p.shares[i] = 0.0f;
        if (real) atomicOr(&map[(id & 0xFFFF) / 32], 1u << (id & 31)); // (bits: no order matters)
    }
    if (listed > 0)
        for (int t = 0; t < p.nq; ++t) stage_query((T *)lds + t * staged, q + t * p.ld_q, d, false, kFewThreads);
    __syncthreads();
    if (threadIdx.x < NQ) {
        const int t = threadIdx.x;
        float a = 0.0f, h = 0.0f, l = 0.0f;
        if (t < p.nq) {
            for (int j = 0; j < p.given; ++j) a += given_g[t * p.given + j];
            if (p.gl) a -= p.gl[t];
            if (p.h) { h = p.h[t]; a += h * p.entropy[t]; }
            l = p.lse[t];
        }
        coef[t][0] = a;
        coef[t][1] = h;
        coef[t][2] = l;
    }
    __syncthreads();

    float qs[NQ][NV * V], acc[NQ][NV * V], a[NQ], h[NQ], lse[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        a[t] = coef[t][0];
        h[t] = coef[t][1];
        lse[t] = coef[t][2];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int k = (in_row + j * L) * V + e;
                qs[t][j * V + e] = t < p.nq && k < d ? to_f32(q[t * p.ld_q + k]) : 0.0f;
                acc[t][j * V + e] = 0.0f;
            }
    }
    float z_low = 0.0f, z_high = 0.0f; // of query in_row
    constexpr float log2e = 1.44269504088896341f;
    for (int64_t base = ((int64_t)blockIdx.x * kFewWaves + wave) * (kPer * U); base < p.n; base += (int64_t)gridDim.x * kFewWaves * (kPer * U)) {
        Unit<T> v[U][NV];
        int64_t row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = base + u * kPer + lane / L;
            const T *from = x + min(row[u], p.n - 1) * p.ld_x;
#pragma unroll
            for (int j = 0; j < NV; ++j) v[u][j] = load_unit<T, RAGGED>(from, min(in_row + j * L, units - 1) * V, d);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool real = row[u] < p.n;
            float xs[NV * V], s[NQ];
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) xs[j * V + e] = real && in_row + j * L < units ? to_f32(v[u][j].e[e]) : 0.0f;
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                s[t] = 0.0f;
#pragma unroll
                for (int k = 0; k < NV * V; ++k) s[t] = __fmaf_rn(xs[k], qs[t][k], s[t]);
                s[t] = group_sum<L>(s[t]);
            }
            float more[NQ] = {}; // the given ids' share of G
            const bool maybe = real && (map[((uint32_t)row[u] & 0xFFFF) / 32] >> ((uint32_t)row[u] & 31) & 1u) != 0;
            if (__any(maybe)) {
                uint32_t own = 0; // queries that this row is given for
                if (maybe) {
#pragma unroll
                    for (int t = 0; t < NQ; ++t) {
                        if (t >= p.nq) continue;
                        for (int j = 0; j < p.given; ++j)
                            if (given_id[t * p.given + j] == (int32_t)row[u]) {
                                more[t] += given_g[t * p.given + j];
                                own |= 1u << t;
                            }
                    }
                }
                // the wave scores those rows, one after the other (two steps' loads in flight: sixteen's registers cost half of the
                // waves, 292 against 190 us for two queries of 1,183,514 x 100 fp32)
#pragma unroll 1
                for (int t = 0; t < p.nq; ++t)
                    for (uint64_t left = __ballot((own >> t & 1u) != 0 && in_row == 0); left != 0; left &= left - 1) {
                        const int from = __ffsll((unsigned long long)left) - 1; // the first lane of that row
                        const T *at = x + (base + u * kPer + from / L) * p.ld_x;
                        float product = 0.0f;
                        score_rows<PATH, 8, 2>((const T *)lds + t * staged, d, Scoring{L, 1.0f}, [&](int) { return at; }, [](int) { return 1.0f; }, [&](int slot, float v) { if (slot == 0) product = v; });
                        product = __shfl(product, 0, 64);
#pragma unroll
                        for (int i = 0; i < NQ; ++i) s[i] = i == t && lane / L == from / L ? product : s[i];
                        if (MEND && lane == 0) {
                            const int32_t id = (int32_t)(base + u * kPer + from / L);
                            const float logp = __fmaf_rn(product, p.scale, -coef[t][2]), w = __builtin_amdgcn_exp2f(logp * log2e), h = coef[t][1];
                            float share = w == 0.0f ? 0.0f : w * (__fmaf_rn(h, logp, coef[t][0]) + h);
                            for (int j = 0; j < p.given; ++j)
                                if (given_id[t * p.given + j] == id) {
                                    p.shares[t * p.given + j] = share;
                                    share = 0.0f;
                                }
                        }
                    }
            }
            float o[NV * V] = {};
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                const float logp = __fmaf_rn(s[t], p.scale, -lse[t]), w = __builtin_amdgcn_exp2f(logp * log2e); // (one rounding of s - lse: only lse's own is in p)
                float G = more[t] - (w == 0.0f ? 0.0f : w * __fmaf_rn(h[t], logp, a[t])); // (p log p)
                if (!real || (NQ > 2 && t >= p.nq)) G = 0.0f; // (a place past the last query is 0 times the row: NaN where that holds an infinity)
                if (MEND) {
                    const float mine = real && in_row == t ? w : 0.0f;
                    z_low += mine >= 0.25f ? 0.0f : mine;
                    z_high += mine >= 0.25f ? mine : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < NV * V; ++k) {
                    acc[t][k] = __fmaf_rn(G, xs[k], acc[t][k]);
                    o[k] = __fmaf_rn(G, qs[t][k], o[k]);
                }
            }
            if (dx && real) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int k = (in_row + j * L) * V;
                    if (in_row + j * L >= units) continue;
                    Unit<T> r;
                    if (p.accumulate) r = load_unit<T, RAGGED>(dx + row[u] * p.ld_dx, k, d);
#pragma unroll
                    for (int e = 0; e < V; ++e) r.e[e] = from_f32<T>(p.accumulate ? to_f32(r.e[e]) + o[j * V + e] * p.scale : o[j * V + e] * p.scale);
                    store_unit<T, RAGGED>(dx + row[u] * p.ld_dx, k, d, r);
                }
            }
        }
    }
    if (MEND) {
        __shared__ float2 waves_z[kFewWaves][NQ];
#pragma unroll
        for (int m = L; m < 64; m <<= 1) {
            z_low += __shfl_xor(z_low, m, 64);
            z_high += __shfl_xor(z_high, m, 64);
        }
        if (lane < NQ) waves_z[wave][lane] = make_float2(z_low, z_high);
        __syncthreads();
        if (threadIdx.x < NQ) {
            float2 v = waves_z[0][threadIdx.x];
            for (int w = 1; w < kFewWaves; ++w) { v.x += waves_z[w][threadIdx.x].x; v.y += waves_z[w][threadIdx.x].y; }
            p.z[(int64_t)blockIdx.x * NQ + threadIdx.x] = v;
        }
    }
    if (!p.sums) return;
    // the wave's rows, then the workgroup's waves one after the other
    float *all = (float *)lds;
    constexpr int kWide = L * NV * V;
    for (int w = 0; w < kFewWaves; ++w) {
        __syncthreads(); // (also: the queries there have been read)
        if (w != wave) continue;
#pragma unroll
        for (int t = 0; t < NQ; ++t)
#pragma unroll
            for (int k = 0; k < NV * V; ++k) {
                float v = acc[t][k];
#pragma unroll
                for (int m = L; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
                const int at = t * kWide + (in_row + k / V * L) * V + k % V;
                if (lane < L) all[at] = w == 0 ? v : all[at] + v;
            }
    }
    __syncthreads();
    const int wide = units * V;
    for (int i = threadIdx.x; i < NQ * kWide; i += kFewThreads) {
        const int t = i / kWide, k = i % kWide;
        if (k < wide) p.sums[((int64_t)blockIdx.x * NQ + t) * wide + k] = all[i];
    }
}

// delta of each query, a workgroup each. More than lse's rounding (2^-24 of it) and that of the sums (2^-20) is not mended: such an lse
// is of more rows than these (a part of a table). What other rows may have that little in is then lost to 1 - p, as it is to lse.
__global__ __launch_bounds__(kFewGroups) void grad_few_delta_kernel(const float2 *__restrict__ z, int groups, int held, const float *__restrict__ lse, float *__restrict__ delta)
{
    __shared__ double all[kFewGroups];
    const int i = threadIdx.x, t = blockIdx.x;
    const float2 v = i < groups ? z[(int64_t)i * held + t] : make_float2(0.0f, 0.0f);
    all[i] = (double)v.x + (double)v.y;
    for (int m = kFewGroups / 2; m > 0; m >>= 1) {
        __syncthreads();
        if (i < m) all[i] += all[i + m];
    }
    const float v1 = (float)(all[0] - 1.0);
    if (i == 0) delta[t] = fabsf(v1) <= 0x1p-24f * fabsf(lse[t]) + 0x1p-20f ? v1 : 0.0f;
}

// dq = the workgroups' sums and, in fp32, what the given rows' G gets back: 64 columns a workgroup, sixteen strips of workgroups, and of
// ids, side by side
template <class T>
__global__ __launch_bounds__(1024) void grad_few_join_kernel(FewArgs p, int groups, int held, int wide, const float *__restrict__ delta, T *__restrict__ dq, int64_t ld)
{
    __shared__ float strips[16][64];
    const int col = threadIdx.x & 63, strip = threadIdx.x >> 6, k = blockIdx.x * 64 + col, t = blockIdx.y;
    float s = 0.0f;
    if (k < p.d) {
        const float *from = p.sums + (int64_t)t * wide + k;
#pragma unroll 16
        for (int g = strip; g < groups; g += 16) s += from[(int64_t)g * held * wide];
        if (delta) {
            for (int j = strip; j < p.given; j += 16) {
                const float share = p.shares[t * p.given + j];
                if (share != 0.0f) s = __fmaf_rn(share * delta[t], to_f32(((const T *)p.x)[(int64_t)p.ids[t * p.given + j] * p.ld_x + k]), s);
            }
        }
    }
    strips[strip][col] = s;
    __syncthreads();
    if (strip != 0 || k >= p.d) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += strips[i][col];
    dq[(int64_t)t * ld + k] = from_f32<T>(s * p.scale);
}

// The same for dx: a row at the first of all ids that name it, of all queries.
__global__ __launch_bounds__(1024) void grad_few_mend_kernel(FewArgs p, const float *__restrict__ delta)
{
    __shared__ float strips[16][64];
    const int col = threadIdx.x & 63, strip = threadIdx.x >> 6, k = blockIdx.x * 64 + col, i = blockIdx.y, listed = p.nq * p.given;
    const int32_t id = p.ids[i];
    if (id < 0 || (int64_t)id >= p.n) return;
    bool later = false;
    float s = 0.0f;
    for (int e = strip; e < listed; e += 16) {
        if (p.ids[e] != id) continue;
        later = later || e < i;
        const int t = e / p.given;
        if (k < p.d) s = __fmaf_rn(p.shares[e] * delta[t], ((const float *)p.q)[t * p.ld_q + k], s);
    }
    if (__syncthreads_or(later)) return;
    strips[strip][col] = s;
    __syncthreads();
    if (strip != 0 || k >= p.d) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += strips[w][col];
    float *to = (float *)p.dx + (int64_t)id * p.ld_dx + k;
    *to = __fmaf_rn(s, p.scale, *to);
}

// What a lane holds of a row, in units; 0: more than it can.
static int few_units(int size, int d)
{
    const int units = (d * size + 15) / 16;
    return units <= 64 ? 1 : units <= 128 ? 2 : units <= 256 ? 4 : 0;
}
static int few_queries(int nq) { return nq <= 2 ? nq : nq <= 4 ? 4 : 8; }

bool grad_few_takes(int type, int d, int nq, int given)
{
    const int size = type == AVQ_F32 ? 4 : 2, nv = few_units(size, d);
    return nq >= 1 && nq <= 8 && nv != 0 && nv * (16 / size) * few_queries(nq) <= kFewHeld && (int64_t)nq * given <= kFewGiven;
}

struct FewScratch { float *sums; float2 *z; float *shares, *delta; size_t bytes; };

static FewScratch few_scratch(int size, int d, int nq, void *base)
{
    FewScratch s{};
    const int v = 16 / size, held = few_queries(nq);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *q = base ? (char *)base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return q;
    };
    s.sums = (float *)take(sizeof(float) * kFewGroups * held * ((d + v - 1) / v * v));
    s.z = (float2 *)take(sizeof(float2) * kFewGroups * held);
    s.shares = (float *)take(sizeof(float) * kFewGiven);
    s.delta = (float *)take(sizeof(float) * held);
    s.bytes = at;
    return s;
}

size_t grad_few_scratch_bytes(int type, int d, int nq) { return few_scratch(type == AVQ_F32 ? 4 : 2, d, nq, nullptr).bytes; }

template <class T, bool RAGGED, int L, int NV, int NQ>
static int few_run(const ProbGradParams &p, hipStream_t st)
{
    constexpr int V = kUnit<T>, kRows = kFewWaves * (64 / L) * few_ahead(NV, NQ);
    const FewScratch s = few_scratch(sizeof(T), p.d, p.nq, p.scratch);
    const int groups = (int)std::min<int64_t>(kFewGroups, (p.n + kRows - 1) / kRows);
    const size_t lds = std::max((size_t)NQ * L * NV * V * sizeof(float), (size_t)p.nq * ((p.d + 31) / 32 * 32) * sizeof(T));
    const FewArgs args{p.points, p.n, p.ld_points, p.d, p.queries, p.ld_queries, p.nq, p.scale, p.ids, p.given, p.lse, p.grad_logp, p.grad_entropy, p.entropy, p.grad_lse, p.dpoints,
                       p.ld_dpoints, p.accumulate, p.dqueries ? s.sums : nullptr, s.z, s.shares};
    grad_few_kernel<T, RAGGED, L, NV, NQ><<<dim3(groups), dim3(kFewThreads), lds, st>>>(args);
    AVQ_HIP(hipGetLastError());
    const bool mend = sizeof(T) == 4 && p.given > 0;
    if (mend) {
        grad_few_delta_kernel<<<dim3(p.nq), dim3(kFewGroups), 0, st>>>(s.z, groups, NQ, p.lse, s.delta);
        AVQ_HIP(hipGetLastError());
    }
    const unsigned columns = (unsigned)((p.d + 63) / 64);
    if (p.dqueries) {
        grad_few_join_kernel<T><<<dim3(columns, p.nq), dim3(1024), 0, st>>>(args, groups, NQ, units_of<T>(p.d) * V, mend ? s.delta : nullptr, (T *)p.dqueries, p.ld_dqueries);
        AVQ_HIP(hipGetLastError());
    }
    if (mend && p.dpoints) {
        grad_few_mend_kernel<<<dim3(columns, p.nq * p.given), dim3(1024), 0, st>>>(args, s.delta);
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

template <class T, bool RAGGED, int NQ>
static int few_sized(const ProbGradParams &p, hipStream_t st)
{
    constexpr int V = kUnit<T>;
    const int units = units_of<T>(p.d);
    if constexpr (V * NQ <= kFewHeld) {
        if (units <= 16) return few_run<T, RAGGED, 16, 1, NQ>(p, st);
        if (units <= 32) return few_run<T, RAGGED, 32, 1, NQ>(p, st);
        if (units <= 64) return few_run<T, RAGGED, 64, 1, NQ>(p, st);
    }
    if constexpr (2 * V * NQ <= kFewHeld) if (units <= 128) return few_run<T, RAGGED, 64, 2, NQ>(p, st);
    if constexpr (4 * V * NQ <= kFewHeld) if (units <= 256) return few_run<T, RAGGED, 64, 4, NQ>(p, st);
    set_error("rows of %d are too long for the pass of a few queries", p.d); // (grad_few_takes says so before)
    return AVQ_EINVAL;
}

template <class T>
static int few_typed(const ProbGradParams &p, hipStream_t st)
{
    const bool whole = whole_units(p.points, p.ld_points, p.d, sizeof(T)) && (!p.dpoints || whole_units(p.dpoints, p.ld_dpoints, p.d, sizeof(T)));
    auto run = [&](auto ragged) {
        constexpr bool RAGGED = decltype(ragged)::value;
        return p.nq == 1 ? few_sized<T, RAGGED, 1>(p, st) : p.nq == 2 ? few_sized<T, RAGGED, 2>(p, st) : p.nq <= 4 ? few_sized<T, RAGGED, 4>(p, st) : few_sized<T, RAGGED, 8>(p, st);
    };
    return whole ? run(std::false_type{}) : run(std::true_type{});
}

int launch_grad_few(const ProbGradParams &p, hipStream_t st)
{
    return p.type == AVQ_F32 ? few_typed<float>(p, st) : p.type == AVQ_BF16 ? few_typed<bf16_t>(p, st) : few_typed<f16_t>(p, st);
}

} // namespace avq
