// Layer norm of rows, y = (x - mean) rstd w + b, and its gradient: with xh = (x - mean) rstd and g = dy w,
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy.
// Bound by memory: x (and dy) read once into registers, y (dx) written once. Sums are fp32, over the lanes of a row in a
// fixed order; dw and db are sums of each workgroup's rows, joined in the workgroups' order: the same result every time.
// A row lies across 16 to 64 lanes, so that sums need no barrier and short rows share a wave. 65,536 x 1,024 bf16: 54 us forward (268 MB, 5.0 TB/s),
// 88 backward (403 MB, 4.6 TB/s; 5.5 us of it the join).
#include "row_types.h"

namespace avq {

constexpr int kNormThreads = 256;

// A row by L lanes that hold NV vectors of it each (L = 256: the whole workgroup).
template <int L> __device__ __forceinline__ float row_sum(float v, float *red)
{
    if (L <= 64) return group_sum<(L <= 64 ? L : 64)>(v);
    v = group_sum<64>(v);
    __syncthreads(); // (the values of the sum before have been read)
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

template <class T, bool RAGGED, int L, int NV>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(const T *__restrict__ x, int64_t rows, int d, int64_t ld_x, const T *__restrict__ weight, const T *__restrict__ bias,
                                                            float eps, T *__restrict__ y, int64_t ld_y, float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    __shared__ float red[4];
    constexpr int V = kUnit<T>, kRows = kNormThreads / L; // rows a workgroup has at a time
    const int per_row = units_of<T>(d), lane = threadIdx.x % L;
    const float inv_d = 1.0f / (float)d;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / L; row - threadIdx.x / L < rows; row += (int64_t)gridDim.x * kRows) {
        const bool real = row < rows;
        Unit<T> v[NV];
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            v[j] = Unit<T>{};
            const int col = lane + j * L;
            if (real && col < per_row) v[j] = load_unit<T, RAGGED>(x + row * ld_x, col * V, d);
#pragma unroll
            for (int e = 0; e < V; ++e) s += to_f32(v[j].e[e]);
        }
        const float mean = row_sum<L>(s, red) * inv_d;
        float q = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = (lane + j * L) * V;
            if (RAGGED) {
#pragma unroll
                for (int e = 0; e < V; ++e) { const float off = k + e < d ? to_f32(v[j].e[e]) - mean : 0.0f; q = __fmaf_rn(off, off, q); }
            } else if (k < d) {
#pragma unroll
                for (int e = 0; e < V; ++e) { const float off = to_f32(v[j].e[e]) - mean; q = __fmaf_rn(off, off, q); }
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<L>(q, red) * inv_d + eps);
        if (!real) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = lane + j * L;
            if (col >= per_row) continue;
            Unit<T> w, b, o;
            if (weight) w = load_unit<T, RAGGED>(weight, col * V, d);
            if (bias) b = load_unit<T, RAGGED>(bias, col * V, d);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float r = (to_f32(v[j].e[e]) - mean) * rstd;
                if (weight) r = r * to_f32(w.e[e]);
                if (bias) r = r + to_f32(b.e[e]);
                o.e[e] = from_f32<T>(r);
            }
            store_unit<T, RAGGED>(y + row * ld_y, col * V, d, o);
        }
        if (lane == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// dx, and the workgroup's sums of dy xh and dy in part[workgroup][2][d].
template <class T, bool RAGGED, int L, int NV>
__global__ __launch_bounds__(kNormThreads) void norm_grad_kernel(const T *__restrict__ dy, int64_t ld_dy, const T *__restrict__ x, int64_t ld_x, int64_t rows, int d,
                                                                 const float *__restrict__ mean_in, const float *__restrict__ rstd_in, const T *__restrict__ weight,
                                                                 T *__restrict__ dx, int64_t ld_dx, float *__restrict__ part)
{
    __shared__ float red[4];
    extern __shared__ float sums[]; // [2][d], of the groups of lanes that were added so far
    constexpr int V = kUnit<T>, kRows = kNormThreads / L;
    const int per_row = units_of<T>(d), lane = threadIdx.x % L, group = threadIdx.x / L;
    const float inv_d = 1.0f / (float)d;
    float dw[NV][V], db[NV][V], w[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int col = lane + j * L;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dw[j][e] = db[j][e] = 0.0f;
            w[j][e] = weight && col * V + e < d ? to_f32(weight[col * V + e]) : 1.0f;
        }
    }
    for (int64_t row = (int64_t)blockIdx.x * kRows + group; row - group < rows; row += (int64_t)gridDim.x * kRows) {
        const bool real = row < rows;
        Unit<T> vx[NV], vg[NV];
        const float mean = real ? mean_in[row] : 0.0f, rstd = real ? rstd_in[row] : 0.0f;
        float sg = 0.0f, sgx = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            vx[j] = vg[j] = Unit<T>{};
            const int col = lane + j * L;
            if (real && col < per_row) {
                vx[j] = load_unit<T, RAGGED>(x + row * ld_x, col * V, d);
                vg[j] = load_unit<T, RAGGED>(dy + row * ld_dy, col * V, d);
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!(real && lane + j * L < per_row)) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float up = to_f32(vg[j].e[e]), xh = (to_f32(vx[j].e[e]) - mean) * rstd, g = up * w[j][e];
                sg += g;
                sgx = __fmaf_rn(g, xh, sgx);
                dw[j][e] = __fmaf_rn(up, xh, dw[j][e]);
                db[j][e] += up;
            }
        }
        const float mg = row_sum<L>(sg, red) * inv_d, mgx = row_sum<L>(sgx, red) * inv_d;
        if (!real) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int col = lane + j * L;
            if (col >= per_row) continue;
            Unit<T> o;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = (to_f32(vx[j].e[e]) - mean) * rstd, g = to_f32(vg[j].e[e]) * w[j][e];
                o.e[e] = from_f32<T>(rstd * (g - mg - xh * mgx));
            }
            store_unit<T, RAGGED>(dx + row * ld_dx, col * V, d, o);
        }
    }
    // the groups' sums, one group after the other
    for (int gi = 0; gi < kRows; ++gi) {
        __syncthreads();
        if (group == gi) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int col = lane + j * L;
                if (col >= per_row) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (RAGGED && col * V + e >= d) break;
                    sums[col * V + e] = gi == 0 ? dw[j][e] : sums[col * V + e] + dw[j][e];
                    sums[d + col * V + e] = gi == 0 ? db[j][e] : sums[d + col * V + e] + db[j][e];
                }
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * d; i += kNormThreads) part[(size_t)blockIdx.x * 2 * d + i] = sums[i];
}

// Rows too long for registers: a workgroup a row, which it reads again from the caches.
template <class T>
__global__ __launch_bounds__(kNormThreads) void norm_long_kernel(const T *__restrict__ x, int64_t rows, int d, int64_t ld_x, const T *__restrict__ weight, const T *__restrict__ bias,
                                                                 float eps, T *__restrict__ y, int64_t ld_y, float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    __shared__ float red[4];
    const float inv_d = 1.0f / (float)d;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *r = x + row * ld_x;
        float s = 0.0f, q = 0.0f;
        for (int c = threadIdx.x; c < d; c += kNormThreads) s += to_f32(r[c]);
        const float mean = row_sum<256>(s, red) * inv_d;
        for (int c = threadIdx.x; c < d; c += kNormThreads) { const float off = to_f32(r[c]) - mean; q = __fmaf_rn(off, off, q); }
        const float rstd = 1.0f / sqrtf(row_sum<256>(q, red) * inv_d + eps);
        for (int c = threadIdx.x; c < d; c += kNormThreads) {
            float v = (to_f32(r[c]) - mean) * rstd;
            if (weight) v = v * to_f32(weight[c]);
            if (bias) v = v + to_f32(bias[c]);
            y[row * ld_y + c] = from_f32<T>(v);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

template <class T>
__global__ __launch_bounds__(kNormThreads) void norm_grad_long_kernel(const T *__restrict__ dy, int64_t ld_dy, const T *__restrict__ x, int64_t ld_x, int64_t rows, int d,
                                                                      const float *__restrict__ mean_in, const float *__restrict__ rstd_in, const T *__restrict__ weight,
                                                                      T *__restrict__ dx, int64_t ld_dx)
{
    __shared__ float red[4];
    const float inv_d = 1.0f / (float)d;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *r = x + row * ld_x, *u = dy + row * ld_dy;
        const float mean = mean_in[row], rstd = rstd_in[row];
        float sg = 0.0f, sgx = 0.0f;
        for (int c = threadIdx.x; c < d; c += kNormThreads) {
            const float xh = (to_f32(r[c]) - mean) * rstd, g = to_f32(u[c]) * (weight ? to_f32(weight[c]) : 1.0f);
            sg += g;
            sgx = __fmaf_rn(g, xh, sgx);
        }
        const float mg = row_sum<256>(sg, red) * inv_d, mgx = row_sum<256>(sgx, red) * inv_d;
        for (int c = threadIdx.x; c < d; c += kNormThreads) {
            const float xh = (to_f32(r[c]) - mean) * rstd, g = to_f32(u[c]) * (weight ? to_f32(weight[c]) : 1.0f);
            dx[row * ld_dx + c] = from_f32<T>(rstd * (g - mg - xh * mgx));
        }
    }
}

// Sums of dy xh and dy over a part of the rows, a thread a column, into part[part][2][d].
template <class T>
__global__ __launch_bounds__(kNormThreads) void norm_columns_kernel(const T *__restrict__ dy, int64_t ld_dy, const T *__restrict__ x, int64_t ld_x, int64_t rows, int64_t rows_each,
                                                                    int d, const float *__restrict__ mean_in, const float *__restrict__ rstd_in, float *__restrict__ part)
{
    const int c = blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= d) return;
    const int64_t lo = blockIdx.y * rows_each, hi = min(rows, lo + rows_each);
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = lo; row < hi; ++row) {
        const float up = to_f32(dy[row * ld_dy + c]), xh = (to_f32(x[row * ld_x + c]) - mean_in[row]) * rstd_in[row];
        dw = __fmaf_rn(up, xh, dw);
        db += up;
    }
    part[(size_t)blockIdx.y * 2 * d + c] = dw;
    part[(size_t)blockIdx.y * 2 * d + d + c] = db;
}

// dw and db from the parts' sums: 64 columns a workgroup, sixteen waves take the parts in turns, then their sums in order (four waves
// took 15 us for 1,024 parts of 2,048 columns).
constexpr int kJoinWaves = 16;

template <class T>
__global__ __launch_bounds__(64 * kJoinWaves) void norm_join_kernel(const float *__restrict__ part, int parts, int d, T *__restrict__ dw, T *__restrict__ db)
{
    __shared__ float sums[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < 2 * d) {
#pragma unroll 16
        for (int p = wave; p < parts; p += kJoinWaves) s += part[(size_t)p * 2 * d + c];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < 2 * d) {
        float v = s;
#pragma unroll
        for (int w = 1; w < kJoinWaves; ++w) v += sums[w][lane];
        if (c < d) { if (dw) dw[c] = from_f32<T>(v); }
        else if (db) db[c - d] = from_f32<T>(v);
    }
}

// Workgroups that a pass over `rows` rows takes when each has `each` rows at a time.
static int norm_groups(int64_t rows, int each, int most)
{
    const int64_t g = (rows + each - 1) / each;
    return (int)std::min<int64_t>(std::max<int64_t>(g, 1), most);
}

constexpr int kNormParts = 1024;   // most workgroups that leave sums of dy xh and dy
constexpr int kNormLongParts = 64;

template <class T, bool RAGGED, int L, int NV>
static int norm_run(const NormParams &p, hipStream_t st)
{
    norm_kernel<T, RAGGED, L, NV><<<dim3(norm_groups(p.rows, kNormThreads / L, 8192)), dim3(kNormThreads), 0, st>>>(
        (const T *)p.x, p.rows, p.d, p.ld_x, (const T *)p.weight, (const T *)p.bias, p.eps, (T *)p.y, p.ld_y, p.mean, p.rstd);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool RAGGED, int L, int NV>
static int norm_grad_run(const NormGradParams &p, hipStream_t st)
{
    const int groups = norm_groups(p.rows, kNormThreads / L, kNormParts);
    norm_grad_kernel<T, RAGGED, L, NV><<<dim3(groups), dim3(kNormThreads), 2 * p.d * sizeof(float), st>>>(
        (const T *)p.dy, p.ld_dy, (const T *)p.x, p.ld_x, p.rows, p.d, p.mean, p.rstd, (const T *)p.weight, (T *)p.dx, p.ld_dx, (float *)p.scratch);
    AVQ_HIP(hipGetLastError());
    norm_join_kernel<T><<<dim3((2 * p.d + 63) / 64), dim3(64 * kJoinWaves), 0, st>>>((const float *)p.scratch, groups, p.d, (T *)p.dweight, (T *)p.dbias);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

// lanes a row and units a lane, by the units a row has
#define AVQ_NORM_BY_SIZE(RUN, LONG)                                   \
    const int per_row = units_of<T>(p.d);                             \
    if (per_row <= 16) return RUN<T, RAGGED, 16, 1>(p, st);           \
    if (per_row <= 32) return RUN<T, RAGGED, 32, 1>(p, st);           \
    if (per_row <= 64) return RUN<T, RAGGED, 64, 1>(p, st);           \
    if (per_row <= 128) return RUN<T, RAGGED, 64, 2>(p, st);          \
    if (per_row <= 256) return RUN<T, RAGGED, 64, 4>(p, st);          \
    if constexpr (sizeof(T) == 4) {                                   \
        if (per_row <= 512) return RUN<T, RAGGED, 64, 8>(p, st);      \
    }                                                                 \
    return LONG<T>(p, st);

template <class T>
static int norm_long(const NormParams &p, hipStream_t st)
{
    norm_long_kernel<T><<<dim3(norm_groups(p.rows, 1, 8192)), dim3(kNormThreads), 0, st>>>((const T *)p.x, p.rows, p.d, p.ld_x, (const T *)p.weight, (const T *)p.bias, p.eps,
                                                                                         (T *)p.y, p.ld_y, p.mean, p.rstd);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T>
static int norm_grad_long(const NormGradParams &p, hipStream_t st)
{
    // (dx may be written over x or dy, so it comes last)
    const int64_t each = (p.rows + kNormLongParts - 1) / kNormLongParts;
    norm_columns_kernel<T><<<dim3((p.d + kNormThreads - 1) / kNormThreads, kNormLongParts), dim3(kNormThreads), 0, st>>>((const T *)p.dy, p.ld_dy, (const T *)p.x, p.ld_x, p.rows,
                                                                                                                     each, p.d, p.mean, p.rstd, (float *)p.scratch);
    AVQ_HIP(hipGetLastError());
    norm_grad_long_kernel<T><<<dim3(norm_groups(p.rows, 1, 8192)), dim3(kNormThreads), 0, st>>>((const T *)p.dy, p.ld_dy, (const T *)p.x, p.ld_x, p.rows, p.d, p.mean, p.rstd,
                                                                                              (const T *)p.weight, (T *)p.dx, p.ld_dx);
    AVQ_HIP(hipGetLastError());
    norm_join_kernel<T><<<dim3((2 * p.d + 63) / 64), dim3(64 * kJoinWaves), 0, st>>>((const float *)p.scratch, kNormLongParts, p.d, (T *)p.dweight, (T *)p.dbias);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool RAGGED> static int norm_sized(const NormParams &p, hipStream_t st) { AVQ_NORM_BY_SIZE(norm_run, norm_long) }
template <class T, bool RAGGED> static int norm_grad_sized(const NormGradParams &p, hipStream_t st) { AVQ_NORM_BY_SIZE(norm_grad_run, norm_grad_long) }

template <class T>
static int norm_typed(const NormParams &p, hipStream_t st)
{
    const bool whole = whole_units(p.x, p.ld_x, p.d, sizeof(T)) && whole_units(p.y, p.ld_y, p.d, sizeof(T)) && whole_units(p.weight, p.d, p.d, sizeof(T)) &&
                       whole_units(p.bias, p.d, p.d, sizeof(T)); // (NULL is aligned)
    return whole ? norm_sized<T, false>(p, st) : norm_sized<T, true>(p, st);
}

template <class T>
static int norm_grad_typed(const NormGradParams &p, hipStream_t st)
{
    const bool whole = whole_units(p.x, p.ld_x, p.d, sizeof(T)) && whole_units(p.dy, p.ld_dy, p.d, sizeof(T)) && whole_units(p.dx, p.ld_dx, p.d, sizeof(T));
    return whole ? norm_grad_sized<T, false>(p, st) : norm_grad_sized<T, true>(p, st);
}

size_t norm_grad_scratch_bytes(int64_t rows, int d)
{
    // (a workgroup has at least one row)
    return (size_t)std::max<int64_t>(std::min<int64_t>(rows, kNormParts), kNormLongParts) * 2 * d * sizeof(float);
}

int launch_norm(const NormParams &p, hipStream_t st)
{
    if (p.rows == 0) return AVQ_OK;
    if (p.type == AVQ_F32) return norm_typed<float>(p, st);
    return p.type == AVQ_BF16 ? norm_typed<bf16_t>(p, st) : norm_typed<f16_t>(p, st);
}

int launch_norm_grad(const NormGradParams &p, hipStream_t st)
{
    // (no rows: the one workgroup's sums are zeros, and so are dw and db)
    if (p.type == AVQ_F32) return norm_grad_typed<float>(p, st);
    return p.type == AVQ_BF16 ? norm_grad_typed<bf16_t>(p, st) : norm_grad_typed<f16_t>(p, st);
}

} // namespace avq
