// The gradient of log probabilities, entropy and log-sum-exp with respect to queries and rows. With s_ti = c <q_t, x_i> and
// upstream g_tj (of log p of id_tj), h_t (of H_t), l_t (of lse_t):
//   G_ti = sum_j g_tj [id_tj = i] - p_ti (a_t + h_t log p_ti),  a_t = sum_j g_tj - l_t + h_t H_t,
//   dq_t = c sum_i G_ti x_i,  dx_i = c sum_t G_ti q_t.
// A part of the rows at a time: its logits once more, G of them, and the two products.
#include "probs.h"
#include "row_types.h"

namespace avq {

// a_t and h_t
__global__ void grad_coef_kernel(const int32_t *__restrict__ ids, int64_t n, int nq, int given, const float *__restrict__ g, const float *__restrict__ h, const float *__restrict__ entropy,
                                 const float *__restrict__ gl, float2 *__restrict__ coef)
{
    const int t = blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= nq) return;
    float a = 0.0f;
    for (int j = 0; j < given; ++j) {
        const int32_t id = ids[(int64_t)t * given + j];
        if (id >= 0 && (int64_t)id < n) a += g[(int64_t)t * given + j];
    }
    if (gl) a -= gl[t];
    if (h) a += h[t] * entropy[t];
    coef[t] = make_float2(a, h ? h[t] : 0.0f);
}

// 64 x 64 tile of A B^T over k, 4 x 4 values a thread.
template <class LoadA, class LoadB, class Store>
__device__ __forceinline__ void tile_product(int64_t rows_a, int64_t rows_b, int64_t depth, LoadA load_a, LoadB load_b, Store store)
{
    __shared__ float sa[16][68], sb[16][68];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t a0 = (int64_t)blockIdx.y * 64, b0 = (int64_t)blockIdx.x * 64;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < depth; k0 += 16) {
        __syncthreads();
        for (int i = threadIdx.x; i < 1024; i += 256) {
            const int64_t r = i >> 4, k = k0 + (i & 15);
            sa[i & 15][r] = a0 + r < rows_a && k < depth ? load_a(a0 + r, k) : 0.0f;
            sb[i & 15][r] = b0 + r < rows_b && k < depth ? load_b(b0 + r, k) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __fmaf_rn(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (a0 + ty * 4 + i < rows_a && b0 + tx * 4 + j < rows_b) store(a0 + ty * 4 + i, b0 + tx * 4 + j, acc[i][j]);
}

template <class T>
__global__ __launch_bounds__(256) void grad_logits_kernel(const T *__restrict__ q, int nq, int64_t ld_q, const T *__restrict__ x, int64_t rows, int64_t ld_x, int d, float scale,
                                                          const float *__restrict__ lse, const float2 *__restrict__ coef, float *__restrict__ G)
{
    tile_product(nq, rows, d, [&](int64_t t, int64_t k) { return to_f32(q[t * ld_q + k]); }, [&](int64_t i, int64_t k) { return to_f32(x[i * ld_x + k]); },
                 [&](int64_t t, int64_t i, float s) {
                     const float logp = s * scale - lse[t];
                     const float2 c = coef[t];
                     G[t * rows + i] = -__expf(logp) * __fmaf_rn(c.y, logp, c.x);
                 });
}

// G += g at the given ids; a thread per given id, the first of equal ones adds for all of them
__global__ void grad_given_kernel(const int32_t *__restrict__ ids, int nq, int given, const float *__restrict__ g, int64_t lo, int64_t rows, float *__restrict__ G)
{
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (int64_t)nq * given) return;
    const int64_t t = i / given, j = i - t * given;
    const int64_t id = ids[i];
    if (id < lo || id >= lo + rows) return;
    float sum = 0.0f;
    for (int64_t o = 0; o < given; ++o)
        if (ids[t * given + o] == id) {
            if (o < j) return;
            sum += g[t * given + o];
        }
    G[t * rows + (id - lo)] += sum;
}

template <class T>
__global__ __launch_bounds__(256) void grad_queries_kernel(const float *__restrict__ G, const T *__restrict__ x, int64_t rows, int64_t ld_x, int nq, int d, int first, float *__restrict__ dq)
{
    tile_product(nq, d, rows, [&](int64_t t, int64_t i) { return G[t * rows + i]; }, [&](int64_t c, int64_t i) { return to_f32(x[i * ld_x + c]); },
                 [&](int64_t t, int64_t c, float s) { dq[t * d + c] = first ? s : dq[t * d + c] + s; });
}

template <class T>
__global__ __launch_bounds__(256) void grad_rows_kernel(const float *__restrict__ G, const T *__restrict__ q, int nq, int64_t ld_q, int64_t rows, int d, float scale, int accumulate,
                                                        T *__restrict__ dx, int64_t ld_dx)
{
    tile_product(d, rows, nq, [&](int64_t c, int64_t t) { return to_f32(q[t * ld_q + c]); }, [&](int64_t i, int64_t t) { return G[t * rows + i]; },
                 [&](int64_t c, int64_t i, float s) { T *to = dx + i * ld_dx + c; *to = from_f32<T>(accumulate ? to_f32(*to) + s * scale : s * scale); });
}

template <class T>
__global__ void grad_round_kernel(const float *__restrict__ dq, int nq, int d, float scale, T *__restrict__ out, int64_t ld)
{
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < (int64_t)nq * d) out[(i / d) * ld + i % d] = from_f32<T>(dq[i] * scale);
}

template <class T>
__global__ void grad_zero_kernel(T *__restrict__ out, int64_t rows, int d, int64_t ld)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = threadIdx.x; c < d; c += blockDim.x) out[r * ld + c] = T{};
}

struct ProbGradScratch { float2 *coef; float *dq, *G; size_t bytes; int64_t part; };

static ProbGradScratch prob_grad_scratch(int64_t n, int d, int nq, void *base)
{
    ProbGradScratch s{};
    s.part = std::max<int64_t>(64, std::min<int64_t>((n + 63) / 64 * 64, ((int64_t)64 << 20) / nq / 64 * 64));
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *p = base ? (char *)base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return p;
    };
    s.coef = (float2 *)take(sizeof(float2) * (size_t)nq);
    s.dq = (float *)take(sizeof(float) * (size_t)nq * d);
    s.G = (float *)take(sizeof(float) * (size_t)nq * s.part);
    s.bytes = at;
    return s;
}

size_t log_probs_grad_scratch_bytes(int type, int64_t n, int d, int nq, int given)
{
    (void)type; (void)given;
    return nq == 0 ? 0 : prob_grad_scratch(n, d, nq, nullptr).bytes;
}

template <class T>
static int log_probs_grad_typed(const ProbGradParams &p, hipStream_t st)
{
    if (p.nq == 0) {
        if (p.dpoints && !p.accumulate) {
            grad_zero_kernel<T><<<dim3((unsigned)std::min<int64_t>(p.n, 65536)), dim3(256), 0, st>>>((T *)p.dpoints, p.n, p.d, p.ld_dpoints);
            AVQ_HIP(hipGetLastError());
        }
        return AVQ_OK;
    }
    const ProbGradScratch s = prob_grad_scratch(p.n, p.d, p.nq, p.scratch);
    grad_coef_kernel<<<dim3((p.nq + 255) / 256), dim3(256), 0, st>>>(p.ids, p.n, p.nq, p.given, p.grad_logp, p.grad_entropy, p.entropy, p.grad_lse, s.coef);
    AVQ_HIP(hipGetLastError());
    const unsigned qt = (p.nq + 63) / 64, dt = (p.d + 63) / 64;
    for (int64_t lo = 0; lo < p.n; lo += s.part) {
        const int64_t rows = std::min<int64_t>(s.part, p.n - lo);
        const unsigned rt = (unsigned)((rows + 63) / 64);
        const T *x = (const T *)p.points + lo * p.ld_points, *q = (const T *)p.queries;
        grad_logits_kernel<T><<<dim3(rt, qt), dim3(256), 0, st>>>(q, p.nq, p.ld_queries, x, rows, p.ld_points, p.d, p.scale, p.lse, s.coef, s.G);
        AVQ_HIP(hipGetLastError());
        if (p.given > 0) {
            grad_given_kernel<<<dim3((unsigned)(((int64_t)p.nq * p.given + 255) / 256)), dim3(256), 0, st>>>(p.ids, p.nq, p.given, p.grad_logp, lo, rows, s.G);
            AVQ_HIP(hipGetLastError());
        }
        if (p.dqueries) {
            grad_queries_kernel<T><<<dim3(dt, qt), dim3(256), 0, st>>>(s.G, x, rows, p.ld_points, p.nq, p.d, lo == 0, s.dq);
            AVQ_HIP(hipGetLastError());
        }
        if (p.dpoints) {
            grad_rows_kernel<T><<<dim3(rt, dt), dim3(256), 0, st>>>(s.G, q, p.nq, p.ld_queries, rows, p.d, p.scale, p.accumulate, (T *)p.dpoints + lo * p.ld_dpoints, p.ld_dpoints);
            AVQ_HIP(hipGetLastError());
        }
    }
    if (p.dqueries) {
        grad_round_kernel<T><<<dim3((unsigned)(((int64_t)p.nq * p.d + 255) / 256)), dim3(256), 0, st>>>(s.dq, p.nq, p.d, p.scale, (T *)p.dqueries, p.ld_dqueries);
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

int launch_log_probs_grad(const ProbGradParams &p, hipStream_t st)
{
    if (p.type == AVQ_F32) return log_probs_grad_typed<float>(p, st);
    return p.type == AVQ_BF16 ? log_probs_grad_typed<bf16_t>(p, st) : log_probs_grad_typed<f16_t>(p, st);
}

} // namespace avq
