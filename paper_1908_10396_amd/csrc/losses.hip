// Losses of log probabilities, with the gradient that those of log probabilities take as theirs.
//
// Distillation from a teacher's best rows, z its logits of them, P = e^(z / tau - lse) (lse that of the list, or of all of the teacher's rows):
//   loss = sum_j P_j (log P_j - log p_j) [+ R log(R / r), R = max(0, 1 - sum P), r = max(1 - sum p, 2^-20)],
//   d loss / d log p_j = [p_j R / r] - P_j.
// Preferences, D_s the sum (mean) over a sequence's tokens of log p - log p_ref, w preferred to l:
//   x = beta (D_w - D_l) - margin, loss = -(1 - e) log sigma(x) - e log sigma(-x), d loss / d x = e sigma(x) - (1 - e) sigma(-x).
// Policy, per token r = e^(log p - log p_old), k = e^(log p_ref - log p) - (log p_ref - log p) - 1:
//   loss = -min(r A, clamp(r, 1 - lo, 1 + hi) A) + w k, d loss / d log p = -r A [not clipped] + w (1 - e^(log p_ref - log p)).
//
// All of it is formed in 64 bits and rounded once: where student and teacher, or policy and reference, agree, a loss is what is left of much
// larger terms, and a sequence's sum may have tens of thousands of them. (A 64-bit multiply-add takes the time of a 32-bit one here.)
#include <math.h>

#include "row_types.h"

namespace avq {

constexpr int kLossThreads = 256, kLossWaves = kLossThreads / 64;
constexpr double kLeastRest = 0x1p-20; // a student's mass beside the list, at least: its log probabilities are not known better

// e^x to 1e-13 or better: x = n log 2 + f, Taylor's polynomial of degree 11 (|f| <= 0.347: the rest is below 7e-15; log 2 is off by 2^-54
// of itself, n times)
__device__ __forceinline__ double exp_wide(double x)
{
    x = x > 800.0 ? 800.0 : x < -800.0 ? -800.0 : x; // (infinity and 0 there; NaN stays)
    const double n = rint(x * 1.4426950408889634074);
    const double f = fma(n, -0.69314718055994530942, x);
    double p = 1.0 / 39916800.0;
    p = fma(p, f, 1.0 / 3628800.0);
    p = fma(p, f, 1.0 / 362880.0);
    p = fma(p, f, 1.0 / 40320.0);
    p = fma(p, f, 1.0 / 5040.0);
    p = fma(p, f, 1.0 / 720.0);
    p = fma(p, f, 1.0 / 120.0);
    p = fma(p, f, 1.0 / 24.0);
    p = fma(p, f, 1.0 / 6.0);
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}

// over L lanes side by side (L = 256: the workgroup, by a value a wave in red)
template <int L> __device__ __forceinline__ double lanes_sum(double v, double *red)
{
    constexpr int W = L < 64 ? L : 64;
#pragma unroll
    for (int w = 1; w < W; w <<= 1) v += __shfl_xor(v, w, 64);
    if (L <= 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

template <int L> __device__ __forceinline__ float lanes_max(float v, double *red)
{
    constexpr int W = L < 64 ? L : 64;
#pragma unroll
    for (int w = 1; w < W; w <<= 1) v = fmaxf(v, __shfl_xor(v, w, 64));
    if (L <= 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (float)fmax(fmax(red[0], red[1]), fmax(red[2], red[3]));
}

// ---- distillation ----------------------------------------------------------------------------

// Elements k .. k + 3 of a row of m, `none` past its end.
template <class T> __device__ __forceinline__ void load4(const T *__restrict__ row, int k, int m, T none, T (&v)[4])
{
    if (k + 4 <= m) {
        __builtin_memcpy(v, row + k, sizeof(v));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = k + e < m ? row[k + e] : none;
    }
}

template <class T> __device__ __forceinline__ T no_logit();
template <> __device__ __forceinline__ float no_logit<float>() { return -INFINITY; }
template <> __device__ __forceinline__ bf16_t no_logit<bf16_t>() { return bf16_t{0xff80}; }
template <> __device__ __forceinline__ f16_t no_logit<f16_t>() { return f16_t{0xfc00}; }

// A row by L lanes, NV times four elements a lane. ALL: the teacher's lse is that of all of its rows.
template <class T, bool ALL, int L, int NV>
__global__ __launch_bounds__(kLossThreads) void distill_kernel(const float *__restrict__ logp, const T *__restrict__ teacher, int64_t ld_teacher, const float *__restrict__ teacher_lse,
                                                               double per_tau, int64_t rows, int m, float *__restrict__ loss, const float *__restrict__ g, float *__restrict__ out)
{
    __shared__ double red[kLossWaves];
    constexpr int kRows = kLossThreads / L;
    const int lane = threadIdx.x % L;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / L; row - threadIdx.x / L < rows; row += (int64_t)gridDim.x * kRows) {
        const bool real = row < rows;
        float z[NV][4], lp[NV][4];
        float top = -INFINITY, some = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (lane + i * L) * 4;
            T zt[4];
            load4<T>(teacher + (real ? row * ld_teacher : 0), k, real ? m : 0, no_logit<T>(), zt);
            load4<float>(logp + (real ? row * m : 0), k, real ? m : 0, -INFINITY, lp[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[i][e] = to_f32(zt[e]);
                top = fmaxf(top, z[i][e]);
                if (!(z[i][e] == -INFINITY)) some = 1.0f; // (NaN is no padding)
            }
        }
        top = lanes_max<L>(top, red);
        some = lanes_max<L>(some, red);
        const double base = ALL ? (real ? (double)teacher_lse[row] : 0.0) : top > -INFINITY ? (double)top * per_tau : 0.0;
        double P[NV][4], sum = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                P[i][e] = z[i][e] == -INFINITY ? 0.0 : exp_wide(fma((double)z[i][e], per_tau, -base));
                sum += P[i][e];
            }
        sum = lanes_sum<L>(sum, red);
        const double log_sum = ALL ? 0.0 : log(sum), per_sum = ALL ? 1.0 : 1.0 / sum;
        double total = 0.0, mine = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (P[i][e] == 0.0) { if (!ALL || z[i][e] == -INFINITY) continue; }
                else total = fma(P[i][e], fma((double)z[i][e], per_tau, -base) - log_sum - (double)lp[i][e], total);
                if (ALL) mine += exp_wide((double)lp[i][e]);
            }
        total = lanes_sum<L>(total, red) * per_sum;
        double pull = 0.0;
        if (ALL) {
            mine = lanes_sum<L>(mine, red);
            const double rest = 1.0 - sum, left = 1.0 - mine;
            if (!(rest <= 0.0)) { // (NaN goes on)
                total += rest * log(rest / (left > kLeastRest ? left : kLeastRest));
                if (left > kLeastRest) pull = rest / left;
            }
            if (!(left == left)) total = pull = left;
        }
        if (!real) continue;
        if (loss && lane == 0) loss[row] = some > 0.0f ? (float)total : 0.0f;
        if (!out) continue;
        const double up = (double)g[row];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (lane + i * L) * 4;
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                double v = -P[i][e] * per_sum;
                if (ALL) v = fma(pull, exp_wide((double)lp[i][e]), v);
                o[e] = z[i][e] == -INFINITY ? 0.0f : (float)(v * up);
            }
            if (k + 4 <= m) {
                __builtin_memcpy(out + row * m + k, o, sizeof(o));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k + e < m) out[row * m + k + e] = o[e];
            }
        }
    }
}

template <class T, bool ALL, int L, int NV>
static int distill_run(const DistillParams &p, hipStream_t st)
{
    const int64_t groups = (p.rows + kLossThreads / L - 1) / (kLossThreads / L);
    distill_kernel<T, ALL, L, NV><<<dim3((unsigned)std::min<int64_t>(groups, 1 << 22)), dim3(kLossThreads), 0, st>>>(
        p.logp, (const T *)p.teacher, p.ld_teacher, p.teacher_lse, 1.0 / p.temperature, p.rows, p.m, p.loss, p.grad_loss, p.grad_logp);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool ALL>
static int distill_sized(const DistillParams &p, hipStream_t st)
{
    if (p.m <= 16) return distill_run<T, ALL, 4, 1>(p, st);
    if (p.m <= 32) return distill_run<T, ALL, 8, 1>(p, st);
    if (p.m <= 64) return distill_run<T, ALL, 16, 1>(p, st);
    if (p.m <= 128) return distill_run<T, ALL, 32, 1>(p, st);
    if (p.m <= 256) return distill_run<T, ALL, 64, 1>(p, st);
    if (p.m <= 512) return distill_run<T, ALL, 64, 2>(p, st);
    if (p.m <= 1024) return distill_run<T, ALL, 64, 4>(p, st);
    return distill_run<T, ALL, 256, 4>(p, st);
}

template <class T> static int distill_typed(const DistillParams &p, hipStream_t st) { return p.teacher_lse ? distill_sized<T, true>(p, st) : distill_sized<T, false>(p, st); }

int launch_distill(const DistillParams &p, hipStream_t st)
{
    if (p.rows == 0) return AVQ_OK;
    if (p.type == AVQ_F32) return distill_typed<float>(p, st);
    return p.type == AVQ_BF16 ? distill_typed<bf16_t>(p, st) : distill_typed<f16_t>(p, st);
}

// ---- sequences of tokens ------------------------------------------------------------------------

// Sequence s: the tokens [lo, hi). Offsets that are no offsets name no token outside of the call's.
struct Span { int64_t lo, hi; };
__device__ __forceinline__ Span span_of(const int32_t *__restrict__ offsets, int64_t s, int64_t tokens)
{
    const int64_t lo = min(max((int64_t)offsets[s], (int64_t)0), tokens);
    return Span{lo, min(max((int64_t)offsets[s + 1], lo), tokens)};
}

// Zeros for the tokens before the first sequence and behind the last, by the first and the last workgroup.
__device__ __forceinline__ void clear_outside(float *__restrict__ out, const int32_t *__restrict__ offsets, int64_t sequences, int64_t tokens)
{
    if (blockIdx.x == 0) {
        const int64_t to = sequences > 0 ? span_of(offsets, 0, tokens).lo : 0;
        for (int64_t i = threadIdx.x; i < to; i += kLossThreads) out[i] = 0.0f;
    }
    if (blockIdx.x == gridDim.x - 1) {
        const int64_t from = sequences > 0 ? span_of(offsets, sequences - 1, tokens).hi : 0;
        for (int64_t i = from + threadIdx.x; i < tokens; i += kLossThreads) out[i] = 0.0f;
    }
}

// A workgroup a pair.
__global__ __launch_bounds__(kLossThreads) void preference_kernel(const float *__restrict__ logp, const float *__restrict__ ref, const uint8_t *__restrict__ mask, int64_t tokens,
                                                                  const int32_t *__restrict__ offsets, int pairs, double beta, double margin, double smoothing, int average,
                                                                  float *__restrict__ loss, float *__restrict__ logit, float *__restrict__ reward, const float *__restrict__ g,
                                                                  float *__restrict__ out)
{
    __shared__ double red[kLossWaves];
    if (out) clear_outside(out, offsets, 2 * (int64_t)pairs, tokens);
    const int64_t pair = blockIdx.x;
    if (pair >= pairs) return;
    double d[2], share[2];
    Span span[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const Span sp = span[side] = span_of(offsets, 2 * pair + side, tokens);
        double sum = 0.0, many = 0.0;
        for (int64_t i = sp.lo + threadIdx.x; i < sp.hi; i += kLossThreads) {
            if (mask && !mask[i]) continue;
            sum += (double)logp[i] - (ref ? (double)ref[i] : 0.0);
            many += 1.0;
        }
        sum = lanes_sum<256>(sum, red);
        share[side] = average ? 1.0 / fmax(lanes_sum<256>(many, red), 1.0) : 1.0;
        d[side] = beta * sum * share[side];
    }
    const double x = d[0] - d[1] - margin, small = exp(-fabs(x)), more = log1p(small);
    if (threadIdx.x == 0) {
        // -log sigma(x) = max(-x, 0) + log(1 + e^-|x|)
        double v = 0.0; // (a side of no weight counts for nothing, also where it is infinite)
        if (smoothing < 1.0) v = (1.0 - smoothing) * (fmax(-x, 0.0) + more);
        if (smoothing > 0.0) v = fma(smoothing, fmax(x, 0.0) + more, v);
        loss[pair] = (float)v;
        logit[pair] = (float)x;
        if (reward) {
            reward[2 * pair] = (float)d[0];
            reward[2 * pair + 1] = (float)d[1];
        }
    }
    if (!out) return;
    const double minus = (x > 0.0 ? small : 1.0) / (1.0 + small); // sigma(-x)
    const double up = (double)g[pair] * beta * (smoothing * (x > 0.0 ? 1.0 : small) / (1.0 + small) - (1.0 - smoothing) * minus);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const float v = (float)(side ? -up * share[1] : up * share[0]);
        for (int64_t i = span[side].lo + threadIdx.x; i < span[side].hi; i += kLossThreads) out[i] = mask && !mask[i] ? 0.0f : v;
    }
}

size_t preference_scratch_bytes(int64_t, int) { return 0; }

int launch_preference(const PreferenceParams &p, hipStream_t st)
{
    if (p.pairs == 0 && !p.grad_logp) return AVQ_OK;
    preference_kernel<<<dim3(std::max(p.pairs, 1)), dim3(kLossThreads), 0, st>>>(p.logp, p.ref, p.mask, p.tokens, p.offsets, p.pairs, p.beta, p.margin, p.smoothing, p.average, p.loss,
                                                                              p.logit, p.reward, p.grad_loss, p.grad_logp);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

// What one token adds: loss, k, whether it is clipped, and the slope of its loss.
struct PolicyTerm { double loss, kl, over, slope; };
__device__ __forceinline__ PolicyTerm policy_term(double logp, double old, double advantage, bool has_ref, double ref, double least, double most, double weight)
{
    const double r = exp_wide(logp - old);
    const bool over = (advantage > 0.0 && r > most) || (advantage < 0.0 && r < least);
    const double held = over ? (advantage > 0.0 ? most : least) : r;
    PolicyTerm t{-(held * advantage), 0.0, over ? 1.0 : 0.0, over ? 0.0 : -(r * advantage)};
    if (has_ref) {
        const double away = ref - logp, e = expm1(away);
        t.kl = e - away;
        t.loss = fma(weight, t.kl, t.loss);
        t.slope = fma(-weight, e, t.slope);
    }
    return t;
}

// A workgroup a sequence.
__global__ __launch_bounds__(kLossThreads) void policy_kernel(const float *__restrict__ logp, const float *__restrict__ old, const float *__restrict__ ref,
                                                              const float *__restrict__ advantage, int each, const uint8_t *__restrict__ mask, int64_t tokens,
                                                              const int32_t *__restrict__ offsets, int sequences, double least, double most, double weight, int average,
                                                              float *__restrict__ loss, float *__restrict__ kl, float *__restrict__ clipped, const float *__restrict__ g,
                                                              float *__restrict__ out)
{
    __shared__ double red[kLossWaves];
    if (out) clear_outside(out, offsets, sequences, tokens);
    const int64_t s = blockIdx.x;
    if (s >= sequences) return;
    const Span span = span_of(offsets, s, tokens);
    const double a = each ? 0.0 : (double)advantage[s];
    double sum = 0.0, sum_kl = 0.0, over = 0.0, many = 0.0;
    for (int64_t i = span.lo + threadIdx.x; i < span.hi; i += kLossThreads) {
        if (mask && !mask[i]) continue;
        const PolicyTerm t = policy_term(logp[i], old[i], each ? (double)advantage[i] : a, ref != nullptr, ref ? (double)ref[i] : 0.0, least, most, weight);
        sum += t.loss;
        sum_kl += t.kl;
        over += t.over;
        many += 1.0;
    }
    sum = lanes_sum<256>(sum, red);
    sum_kl = lanes_sum<256>(sum_kl, red);
    over = lanes_sum<256>(over, red);
    many = fmax(lanes_sum<256>(many, red), 1.0);
    const double share = average ? 1.0 / many : 1.0;
    if (threadIdx.x == 0) {
        loss[s] = (float)(sum * share);
        if (kl) kl[s] = (float)(sum_kl * share);
        if (clipped) clipped[s] = (float)(over / many);
    }
    if (!out) return;
    const double up = (double)g[s] * share;
    for (int64_t i = span.lo + threadIdx.x; i < span.hi; i += kLossThreads) {
        float v = 0.0f;
        if (!mask || mask[i])
            v = (float)(up * policy_term(logp[i], old[i], each ? (double)advantage[i] : a, ref != nullptr, ref ? (double)ref[i] : 0.0, least, most, weight).slope);
        out[i] = v;
    }
}

size_t policy_scratch_bytes(int64_t, int) { return 0; }

int launch_policy(const PolicyParams &p, hipStream_t st)
{
    if (p.sequences == 0 && !p.grad_logp) return AVQ_OK;
    policy_kernel<<<dim3(std::max(p.sequences, 1)), dim3(kLossThreads), 0, st>>>(p.logp, p.old, p.ref, p.advantage, p.each, p.mask, p.tokens, p.offsets, p.sequences,
                                                                              1.0 - p.clip_low, 1.0 + p.clip_high, p.kl_weight, p.average, p.loss, p.kl, p.clipped, p.grad_loss,
                                                                              p.grad_logp);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

} // namespace avq
