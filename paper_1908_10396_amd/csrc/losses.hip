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
// larger terms, and a sequence's sum may have tens of thousands of them. (A 64-bit multiply-add takes the time of 1.8 32-bit ones here: 2.2 and 1.26 ns
// a wave and SIMD.)
#include <math.h>

#include "row_types.h"

namespace avq {

constexpr int kLossThreads = 256;
constexpr double kLeastRest = 0x1p-20; // a student's mass beside the list, at least: its log probabilities are not known better
constexpr double kLog2 = 0.69314718055994530942, kPerLog2 = 1.4426950408889634074;

// a constant in scalar registers, where a multiply-add takes it from: else it is moved to vector registers first, for each use
__device__ __forceinline__ double held(double c)
{
    asm("" : "+s"(c));
    return c;
}

// x = n log 2 + f with |f| <= log(2) / 2, for x held to +-800 (where e^x is infinity and 0; a NaN is lost)
struct Reduced { double n, f; };
__device__ __forceinline__ Reduced reduced(double x)
{
    x = fmin(fmax(x, -800.0), 800.0);
    const double n = rint(x * held(kPerLog2));
    return Reduced{n, fma(n, held(-kLog2), x)};
}

// e^x to 1e-13 or better (no NaN): the Chebyshev series of e^f on |f| <= log(2) / 2 up to degree 9, 1.9e-14 of it; log 2 is off by 2^-54
// of itself, n times
__device__ __forceinline__ double exp_wide(double x)
{
    const Reduced r = reduced(x);
    double p = fma(held(2.762994375246158e-06), r.f, held(2.4884447491303006e-05));
    p = fma(p, r.f, held(0.00019841197960142717));
    p = fma(p, r.f, held(0.0013888801773822223));
    p = fma(p, r.f, held(0.008333333360426695));
    p = fma(p, r.f, held(0.04166666704037994));
    p = fma(p, r.f, held(0.16666666666642443));
    p = fma(p, r.f, held(0.4999999999943919));
    p = fma(p, r.f, held(0.9999999999999977));
    p = fma(p, r.f, held(1.0000000000000135));
    return ldexp(p, (int)r.n);
}

// e^x - 1 and e^x - 1 - x (no NaN), with their own relative accuracy near 0: Taylor's polynomial of (e^f - 1 - f) / f^2
struct NearOne { double e1, e2; };
__device__ __forceinline__ NearOne exp_near_one(double x)
{
    const Reduced r = reduced(x);
    double q = fma(held(1.0 / 39916800.0), r.f, held(1.0 / 3628800.0));
    q = fma(q, r.f, held(1.0 / 362880.0));
    q = fma(q, r.f, held(1.0 / 40320.0));
    q = fma(q, r.f, held(1.0 / 5040.0));
    q = fma(q, r.f, held(1.0 / 720.0));
    q = fma(q, r.f, held(1.0 / 120.0));
    q = fma(q, r.f, held(1.0 / 24.0));
    q = fma(q, r.f, held(1.0 / 6.0));
    q = fma(q, r.f, 0.5);
    const double square = r.f * r.f, e = ldexp(1.0 + fma(square, q, r.f), (int)r.n);
    const bool near = r.n == 0.0;
    return NearOne{near ? fma(square, q, r.f) : e - 1.0, near ? square * q : (e - 1.0) - fmin(x, 800.0)};
}

// v + its value `CTRL` lanes away, through the adders' operand paths
template <int CTRL> __device__ __forceinline__ double moved_by(double v)
{
    const uint2 w = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_mov_dpp(w.x, CTRL, 0xF, 0xF, true), __builtin_amdgcn_mov_dpp(w.y, CTRL, 0xF, 0xF, true)));
}

// over L lanes side by side, at most a wave
template <int L> __device__ __forceinline__ double group_sum_wide(double v)
{
    if (L > 1) v += moved_by<0xB1>(v);  // the lane beside
    if (L > 2) v += moved_by<0x4E>(v);  // the other pair
    if (L > 4) v += moved_by<0x141>(v); // the other four of eight
    if (L > 8) v += moved_by<0x140>(v); // the other eight of sixteen
    if (L > 16) v += __shfl_xor(v, 16, 64);
    if (L > 32) v += __shfl_xor(v, 32, 64);
    return v;
}

__device__ __forceinline__ double of_lane(double v, int lane)
{
    const uint2 w = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_readlane(w.x, lane), __builtin_amdgcn_readlane(w.y, lane)));
}

// N sums over L lanes side by side: part of a wave, or (L > 64) the whole workgroup by red[wave][N]
template <int L, int N> __device__ __forceinline__ void lanes_sum(double (&v)[N], double *red)
{
    constexpr int W = L < 64 ? L : 64, kWaves = L <= 64 ? 1 : L / 64;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = group_sum_wide<W>(v[i]);
    if (L <= 64) return;
    static_assert(kWaves * N <= 64, "a lane a value");
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) red[(threadIdx.x >> 6) * N + i] = v[i];
    __syncthreads();
    // every wave joins them: lane i kWaves + w has sum i of wave w
    const int lane = threadIdx.x & 63;
    const double mine = group_sum_wide<kWaves>(lane < kWaves * N ? red[lane % kWaves * N + lane / kWaves] : 0.0);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = of_lane(mine, i * kWaves);
}

// the bits that any of L lanes side by side has, at most a wave
template <int L> __device__ __forceinline__ uint32_t lanes_or(uint32_t v)
{
    if (L > 1) v |= __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);
    if (L > 2) v |= __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);
    if (L > 4) v |= __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true);
    if (L > 8) v |= __builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, true);
    if (L > 16) v |= (uint32_t)__shfl_xor((int)v, 16, 64);
    if (L > 32) v |= (uint32_t)__shfl_xor((int)v, 32, 64);
    return v;
}

template <int L> __device__ __forceinline__ float lanes_max(float v, float *red)
{
    constexpr int W = L < 64 ? L : 64, kWaves = L / 64;
#pragma unroll
    for (int w = 1; w < W; w <<= 1) v = fmaxf(v, __shfl_xor(v, w, 64));
    if (L <= 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < kWaves; ++w) v = fmaxf(v, red[w]);
    return v;
}

// ---- distillation ----------------------------------------------------------------------------

// A row by L lanes, E elements a lane, L apart. ALL: the teacher's lse is that of all of its rows. GRAD: with the gradient. Bound by vector instructions,
// 70 an element of which 39 are in 64 bits: 8,191 rows of 1,000 fp32 20 us (65 MB, 3.2 TB/s), 65,536 of 64 bf16 with the gradient 16.
template <int L> constexpr int kDistillThreads = L > 64 ? L : kLossThreads; // a row has a part of a wave, or a workgroup
template <class T, bool ALL, bool GRAD, int L, int E>
__global__ __launch_bounds__(kDistillThreads<L>) void distill_kernel(const float *__restrict__ logp, const T *__restrict__ teacher, int64_t ld_teacher,
                                                                     const float *__restrict__ teacher_lse, double per_tau, int64_t rows, int m, float *__restrict__ loss,
                                                                     const float *__restrict__ g, float *__restrict__ out)
{
    constexpr int B = kDistillThreads<L>, kRows = B / L;
    __shared__ double red[B / 64 * 3];
    __shared__ float red_max[B / 64];
    __shared__ uint32_t red_odd[B / 64];
    const int lane = threadIdx.x % L;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / L; row - threadIdx.x / L < rows; row += (int64_t)gridDim.x * kRows) {
        const bool real = row < rows;
        float z[E], lp[E], top = -INFINITY;
        {
            const T *zr = teacher + (real ? row : 0) * ld_teacher;
            const float *lr = logp + (real ? row : 0) * m;
            T zt[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int k = min(lane + e * L, m - 1); // (an element always, so that no load waits for a branch; m > 0)
                zt[e] = zr[k];
                lp[e] = lr[k];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = lane + e * L < m ? to_f32(zt[e]) : -INFINITY;
        }
        // what has no place in the exponentials: an entry that is no padding, a NaN of the teacher, of the student, an entry that the
        // student gives nothing and the teacher something
        bool some = false, odd_teacher = false, odd_student = false, none = false;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool there = !(z[e] == -INFINITY);
            some |= there;
            odd_teacher |= z[e] != z[e];
            lp[e] = there ? lp[e] : -INFINITY;
            odd_student |= lp[e] != lp[e];
            if (!ALL) top = fmaxf(top, z[e]);
        }
        if (!ALL) top = lanes_max<L>(top, red_max);
        const double base = ALL ? (real ? (double)teacher_lse[row] : 0.0) : top > -INFINITY ? (double)top * per_tau : 0.0;
        double P[E], p[E], sums[3] = {0.0, 0.0, 0.0}; // of P, of P times (log P up to its constant - log p), of p
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const double a = fma((double)z[e], per_tau, -base);
            P[e] = exp_wide(a);
            sums[0] += P[e];
            const bool counts = P[e] > 0.0, finite = lp[e] > -INFINITY;
            none |= counts & !finite;
            sums[1] = fma(P[e], (counts & finite) ? a - (double)lp[e] : 0.0, sums[1]);
            if (ALL) {
                p[e] = exp_wide((double)lp[e]);
                sums[2] += p[e];
            }
        }
        uint32_t odd = (some ? 1u : 0u) | (odd_teacher ? 2u : 0u) | (odd_student ? 4u : 0u) | (none ? 8u : 0u);
        if (base != base || base == INFINITY) odd |= 2u; // (no teacher's distribution)
        odd = lanes_or<(L < 64 ? L : 64)>(odd);
        if (L > 64) {
            __syncthreads(); // (the row before has been read)
            if ((threadIdx.x & 63) == 0) red_odd[threadIdx.x >> 6] = odd; // (read behind the barriers of the sums)
        }
        lanes_sum<L>(sums, red);
        if (L > 64)
#pragma unroll
            for (int w = 0; w < B / 64; ++w) odd |= red_odd[w];
        if (odd & 2u) sums[0] = NAN;
        if (odd & 4u) sums[1] = sums[2] = NAN;
        const double per_sum = ALL ? 1.0 : 1.0 / sums[0];
        double total = ALL ? sums[1] : fma(sums[1], per_sum, -log(sums[0])), pull = 0.0;
        if (ALL) {
            const double rest = 1.0 - sums[0], left = 1.0 - sums[2];
            if (!(rest <= 0.0)) { // (NaN goes on)
                total += rest * log(rest / (left > kLeastRest ? left : kLeastRest));
                if (left > kLeastRest) pull = rest / left;
            }
            if (left != left) total = pull = left;
        }
        if ((odd & 8u) && total == total) total = INFINITY;
        if (!real) continue;
        if (loss && lane == 0) loss[row] = (odd & 1u) != 0u ? (float)total : 0.0f;
        if (!GRAD) continue;
        const double up = (double)g[row], up_teacher = -up * per_sum;
        pull *= up;
        float *to = out + row * m;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            double v = P[e] * up_teacher;
            if (ALL) v = fma(pull, p[e], v);
            float o = (odd & 2u) != 0u ? NAN : (float)v;
            o = z[e] == -INFINITY ? 0.0f : o;
            if (lane + e * L < m) to[lane + e * L] = o;
        }
    }
}

template <class T, bool ALL, int L, int E>
static int distill_run(const DistillParams &p, hipStream_t st)
{
    constexpr int B = kDistillThreads<L>, kRows = B / L;
    const int64_t groups = (p.rows + kRows - 1) / kRows;
    const auto kernel = p.grad_logp ? distill_kernel<T, ALL, true, L, E> : distill_kernel<T, ALL, false, L, E>;
    kernel<<<dim3((unsigned)std::min<int64_t>(groups, 1 << 16)), dim3(B), 0, st>>>(p.logp, (const T *)p.teacher, p.ld_teacher, p.teacher_lse, 1.0 / p.temperature, p.rows, p.m, p.loss,
                                                                                p.grad_loss, p.grad_logp);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

// Elements a lane: what a row takes beside its exponentials (sums over lanes, logarithm, quotients) is some 400 instructions, shared by a lane's
// elements.
template <class T, bool ALL>
static int distill_sized(const DistillParams &p, hipStream_t st)
{
    if (p.m <= 16) return distill_run<T, ALL, 4, 4>(p, st);
    if (p.m <= 32) return distill_run<T, ALL, 4, 8>(p, st);
    if (p.m <= 64) return distill_run<T, ALL, 8, 8>(p, st);
    if (p.m <= 128) return distill_run<T, ALL, 16, 8>(p, st);
    if (p.m <= 256) return distill_run<T, ALL, 32, 8>(p, st);
    if (p.m <= 512) return distill_run<T, ALL, 64, 8>(p, st);
    if (p.m <= 1024) return distill_run<T, ALL, 64, 16>(p, st);
    return distill_run<T, ALL, 256, 16>(p, st);
}

// lists of no entries: loss 0
__global__ __launch_bounds__(kLossThreads) void no_loss_kernel(float *__restrict__ loss, int64_t rows)
{
    for (int64_t i = blockIdx.x * (int64_t)kLossThreads + threadIdx.x; i < rows; i += gridDim.x * (int64_t)kLossThreads) loss[i] = 0.0f;
}

template <class T> static int distill_typed(const DistillParams &p, hipStream_t st) { return p.teacher_lse ? distill_sized<T, true>(p, st) : distill_sized<T, false>(p, st); }

int launch_distill(const DistillParams &p, hipStream_t st)
{
    if (p.rows == 0) return AVQ_OK;
    if (p.m == 0) {
        if (p.loss) {
            no_loss_kernel<<<dim3((unsigned)std::min<int64_t>((p.rows + kLossThreads - 1) / kLossThreads, 4096)), dim3(kLossThreads), 0, st>>>(p.loss, p.rows);
            AVQ_HIP(hipGetLastError());
        }
        return AVQ_OK;
    }
    if (p.type == AVQ_F32) return distill_typed<float>(p, st);
    return p.type == AVQ_BF16 ? distill_typed<bf16_t>(p, st) : distill_typed<f16_t>(p, st);
}

// ---- sequences of tokens ------------------------------------------------------------------------

// Sequence s: the tokens [lo, hi) of at most 2^28. Offsets that are no offsets name no token outside of the call's.
struct Span { int lo, hi; };
__device__ __forceinline__ Span span_of(const int32_t *__restrict__ offsets, int64_t s, int tokens)
{
    const int lo = min(max(offsets[s], 0), tokens);
    return Span{lo, min(max(offsets[s + 1], lo), tokens)};
}

// Zeros for the tokens before the first sequence and behind the last, by all workgroups.
template <int B> __device__ __forceinline__ void clear_outside(float *__restrict__ out, const int32_t *__restrict__ offsets, int64_t sequences, int tokens)
{
    const int to = sequences > 0 ? span_of(offsets, 0, tokens).lo : 0, from = sequences > 0 ? span_of(offsets, sequences - 1, tokens).hi : 0;
    const int64_t first = blockIdx.x * (int64_t)B + threadIdx.x, step = gridDim.x * (int64_t)B;
    for (int64_t i = first; i < to; i += step) out[i] = 0.0f;
    for (int64_t i = from + first; i < tokens; i += step) out[i] = 0.0f;
}
// Workgroups beyond the sequences' own, for many tokens behind the last one.
inline unsigned sequence_groups(int64_t tokens, int64_t sequences) { return (unsigned)(std::max<int64_t>(sequences, 1) + std::min<int64_t>(tokens >> 13, 512)); }

// A sequence (or pair) has a workgroup of B threads, that take kRound tokens each at a time: a wave for up to 64 tokens in the mean,
// 256 threads up to 256 (pairs 1,024), else 1,024, so that most take one round, whose loads are all in flight.
constexpr int kRound = 4;
inline int sequence_threads(int64_t tokens, int64_t sequences) { return tokens <= 64 * sequences ? 64 : tokens <= 256 * sequences ? 256 : 1024; }

// Few sequences of many tokens: each is taken in parts, 1,024 tokens or a thousand workgroups in all, whose sums a second launch joins. A call
// takes 19 to 21 us that way, up to 1,048,576 tokens of one sequence; by one workgroup a sequence, policy takes 28 for 16,384 tokens and 1,740 for
// 1,048,576, preferences 15, 61 (131,072) and 627. `least`: the tokens from which on that is worth the launch. The parts are those of a sequence among equals: one of
// 1,048,576 tokens has four beside 253 of 100 tokens and takes 908 us (preferences, 254 pairs: 173), and one workgroup beside 299 (1,792 and 335).
constexpr int kPartThreads = 256, kPartTokens = 1024, kPartGroups = 1024, kPartSequences = 256;
constexpr int64_t kPreferenceParts = 24576, kPolicyParts = 8192;
inline int sequence_parts(int64_t tokens, int64_t sequences, int64_t least)
{
    if (sequences == 0 || sequences >= kPartSequences || tokens <= least) return 1;
    return (int)std::min<int64_t>((tokens + kPartTokens - 1) / kPartTokens, kPartGroups / sequences);
}
__device__ __forceinline__ Span part_of(const Span &all, int part, int parts)
{
    const int64_t length = all.hi - all.lo;
    return Span{all.lo + (int)(length * part / parts), all.lo + (int)(length * (part + 1) / parts)};
}

// The parts' sums of a sequence, joined by every workgroup of it in the same order.
__device__ __forceinline__ void join_parts(const double *__restrict__ partial, int64_t sequence, int parts, double (&sums)[4], double *red)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[i] = 0.0;
    for (int p = threadIdx.x; p < parts; p += kPartThreads)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[i] += partial[(sequence * parts + p) * 4 + i];
    lanes_sum<kPartThreads>(sums, red);
}
__device__ __forceinline__ void store_part(double *__restrict__ partial, const double (&sums)[4])
{
    if (threadIdx.x == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) partial[blockIdx.x * (int64_t)4 + i] = sums[i];
}

static size_t parts_bytes(int64_t sequences, int parts) { return parts == 1 ? 0 : (size_t)sequences * parts * 4 * sizeof(double); }
size_t preference_scratch_bytes(int64_t tokens, int pairs) { return parts_bytes(pairs, sequence_parts(tokens, pairs, kPreferenceParts)); }
size_t policy_scratch_bytes(int64_t tokens, int sequences) { return parts_bytes(sequences, sequence_parts(tokens, sequences, kPolicyParts)); }

// ---- preferences ---------------------------------------------------------------------------

struct PreferenceArgs {
    const float *logp, *ref; const uint8_t *mask; const int32_t *offsets; int tokens, pairs, average;
    double beta, margin, smoothing;
    float *loss, *logit, *reward; const float *g; float *out;
};

// Of the pair's tokens in [lo, hi), those before `middle` being the preferred answer's: sums of the ratios and counts of either side.
template <int B> __device__ __forceinline__ void preference_sums(const PreferenceArgs &a, int lo, int middle, int hi, double (&sums)[4])
{
    // (what is not given is read from logp all the same, and left out: no load waits for a branch)
    const float *ref = a.ref ? a.ref : a.logp;
    const uint8_t *mask = a.mask ? a.mask : (const uint8_t *)a.logp;
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[i] = 0.0;
    for (int i0 = lo + (int)threadIdx.x; i0 < hi; i0 += kRound * B) {
        float v[kRound], r[kRound];
        uint8_t set[kRound];
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
            const uint32_t i = (uint32_t)min(i0 + u * B, hi - 1); // (a token of the pair always)
            set[u] = mask[i];
            v[u] = a.logp[i];
            r[u] = ref[i];
        }
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
            const int i = i0 + u * B;
            const bool counts = (i < hi) & (set[u] != 0 || !a.mask);
            const double add = counts ? (double)v[u] - (a.ref ? (double)r[u] : 0.0) : 0.0, one = counts ? 1.0 : 0.0;
            sums[0] += i < middle ? add : 0.0;
            sums[1] += i < middle ? one : 0.0;
            sums[2] += i < middle ? 0.0 : add;
            sums[3] += i < middle ? 0.0 : one;
        }
    }
}

// The pair's results (by whoever `writes`), and what its tokens in [lo, hi) get.
template <int B> __device__ __forceinline__ void preference_finish(const PreferenceArgs &a, int64_t pair, const double (&sums)[4], bool writes, int lo, int middle, int hi)
{
    const double up = a.out ? (double)a.g[pair] : 0.0;
    const double share[2] = {a.average ? 1.0 / fmax(sums[1], 1.0) : 1.0, a.average ? 1.0 / fmax(sums[3], 1.0) : 1.0};
    const double d[2] = {a.beta * sums[0] * share[0], a.beta * sums[2] * share[1]};
    const double x = d[0] - d[1] - a.margin, small = x == x ? exp_wide(-fabs(x)) : x;
    if (writes && threadIdx.x == 0) {
        // -log sigma(x) = max(-x, 0) + log(1 + e^-|x|)
        const double more = log1p(small);
        double v = 0.0; // (a side of no weight counts for nothing, also where it is infinite)
        if (a.smoothing < 1.0) v = (1.0 - a.smoothing) * (fmax(-x, 0.0) + more);
        if (a.smoothing > 0.0) v = fma(a.smoothing, fmax(x, 0.0) + more, v);
        a.loss[pair] = (float)v;
        a.logit[pair] = (float)x;
        if (a.reward) {
            a.reward[2 * pair] = (float)d[0];
            a.reward[2 * pair + 1] = (float)d[1];
        }
    }
    if (!a.out) return;
    const double one = 1.0 / (1.0 + small), rest = small * one; // sigma(|x|), sigma(-|x|)
    const double slope = up * a.beta * (x > 0.0 ? a.smoothing * one - (1.0 - a.smoothing) * rest : a.smoothing * rest - (1.0 - a.smoothing) * one);
    const float to_first = (float)(slope * share[0]), to_second = (float)(-slope * share[1]);
    for (int i = lo + (int)threadIdx.x; i < hi; i += B) {
        const float v = i < middle ? to_first : to_second;
        a.out[i] = a.mask && !a.mask[i] ? 0.0f : v;
    }
}

// (a pair's tokens lie side by side)
struct Pair { Span all; int middle; };
__device__ __forceinline__ Pair pair_of(const PreferenceArgs &a, int64_t pair)
{
    const Span first = span_of(a.offsets, 2 * pair, a.tokens), second = span_of(a.offsets, 2 * pair + 1, a.tokens);
    return Pair{Span{first.lo, max(first.lo, second.hi)}, first.hi};
}

template <int B>
__global__ __launch_bounds__(B) void preference_kernel(PreferenceArgs a)
{
    __shared__ double red[B / 64 * 4];
    if (a.out) clear_outside<B>(a.out, a.offsets, 2 * (int64_t)a.pairs, a.tokens);
    const int64_t pair = blockIdx.x;
    if (pair >= a.pairs) return;
    const Pair p = pair_of(a, pair);
    double sums[4];
    preference_sums<B>(a, p.all.lo, p.middle, p.all.hi, sums);
    lanes_sum<B>(sums, red);
    preference_finish<B>(a, pair, sums, true, p.all.lo, p.middle, p.all.hi);
}

__global__ __launch_bounds__(kPartThreads) void preference_parts_kernel(PreferenceArgs a, int parts, double *__restrict__ partial)
{
    __shared__ double red[kPartThreads / 64 * 4];
    const Pair p = pair_of(a, blockIdx.x / (uint32_t)parts);
    const Span mine = part_of(p.all, blockIdx.x % (uint32_t)parts, parts);
    double sums[4];
    preference_sums<kPartThreads>(a, mine.lo, p.middle, mine.hi, sums);
    lanes_sum<kPartThreads>(sums, red);
    store_part(partial, sums);
}

// A workgroup a part; without a gradient, a workgroup a pair.
__global__ __launch_bounds__(kPartThreads) void preference_join_kernel(PreferenceArgs a, int parts, const double *__restrict__ partial)
{
    __shared__ double red[kPartThreads / 64 * 4];
    const uint32_t each = a.out ? parts : 1;
    if (a.out) clear_outside<kPartThreads>(a.out, a.offsets, 2 * (int64_t)a.pairs, a.tokens);
    const int64_t pair = blockIdx.x / each;
    if (pair >= a.pairs) return;
    const int part = blockIdx.x % each;
    const Pair p = pair_of(a, pair);
    const Span mine = part_of(p.all, part, parts);
    double sums[4];
    join_parts(partial, pair, parts, sums, red);
    preference_finish<kPartThreads>(a, pair, sums, part == 0, mine.lo, p.middle, mine.hi);
}

int launch_preference(const PreferenceParams &p, hipStream_t st)
{
    if (p.pairs == 0 && !p.grad_logp) return AVQ_OK;
    const PreferenceArgs a{p.logp, p.ref, p.mask, p.offsets, (int)p.tokens, p.pairs, p.average, p.beta, p.margin, p.smoothing, p.loss, p.logit, p.reward, p.grad_loss, p.grad_logp};
    const int parts = sequence_parts(p.tokens, p.pairs, kPreferenceParts);
    const int64_t behind = p.grad_logp ? p.tokens : 0;
    if (parts > 1) {
        preference_parts_kernel<<<dim3((unsigned)p.pairs * parts), dim3(kPartThreads), 0, st>>>(a, parts, (double *)p.scratch);
        AVQ_HIP(hipGetLastError());
        preference_join_kernel<<<dim3(sequence_groups(behind, (int64_t)p.pairs * (p.grad_logp ? parts : 1))), dim3(kPartThreads), 0, st>>>(a, parts, (const double *)p.scratch);
    } else {
        const int threads = sequence_threads(p.tokens, 4 * (int64_t)p.pairs);
        const auto kernel = threads == 64 ? preference_kernel<64> : threads == 256 ? preference_kernel<256> : preference_kernel<1024>;
        kernel<<<dim3(sequence_groups(behind, p.pairs)), dim3(threads), 0, st>>>(a);
    }
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

// ---- policy ----------------------------------------------------------------------------------

struct PolicyArgs {
    const float *logp, *old, *ref, *advantage; const uint8_t *mask; const int32_t *offsets; int each, tokens, sequences, average;
    double least, most, weight;
    float *loss, *kl, *clipped; const float *g; float *out;
};

// What one token adds: loss, k, whether it is clipped, and the slope of its loss.
struct PolicyTerm { double loss, kl, over, slope; };
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs &a, double logp, double old, double advantage, double ref)
{
    const double x = logp - old;
    const double r = x == x ? exp_wide(x) : x;
    const bool over = (advantage > 0.0 && r > a.most) || (advantage < 0.0 && r < a.least);
    const double held = over ? (advantage > 0.0 ? a.most : a.least) : r;
    const bool none = advantage == 0.0; // (nothing, also of a ratio that is infinite)
    PolicyTerm t{none ? 0.0 : -(held * advantage), 0.0, over ? 1.0 : 0.0, over || none ? 0.0 : -(r * advantage)};
    if (none && x != x) t.loss = t.slope = x;
    if (a.ref) {
        const double away = ref - logp;
        const NearOne e = exp_near_one(away);
        t.kl = away == away ? e.e2 : away;
        if (a.weight != 0.0) { // (no weight: nothing, also of a divergence that is infinite)
            t.loss = fma(a.weight, t.kl, t.loss);
            t.slope = away == away ? fma(-a.weight, e.e1, t.slope) : away;
        }
    }
    return t;
}

// The terms of kRound tokens of sequence s from i0 on, in steps of B, for those before hi that count: fn(u, the term).
template <int B, class Fn> __device__ __forceinline__ void policy_round(const PolicyArgs &a, int64_t s, int i0, int hi, Fn fn)
{
    // (what is not given is read from logp all the same, and left out: no load waits for a branch)
    const float *ref = a.ref ? a.ref : a.logp;
    const uint8_t *mask = a.mask ? a.mask : (const uint8_t *)a.logp;
    float v[kRound], o[kRound], r[kRound], adv[kRound];
    uint8_t set[kRound];
#pragma unroll
    for (int u = 0; u < kRound; ++u) {
        const uint32_t i = (uint32_t)min(i0 + u * B, hi - 1); // (a token of the sequence always)
        set[u] = mask[i];
        v[u] = a.logp[i];
        o[u] = a.old[i];
        r[u] = ref[i];
        adv[u] = a.advantage[a.each ? i : (uint32_t)s];
    }
#pragma unroll
    for (int u = 0; u < kRound; ++u)
        if ((i0 + u * B < hi) & (set[u] != 0 || !a.mask)) fn(u, policy_term(a, v[u], o[u], adv[u], r[u]));
}

// Sums over [lo, hi) of the losses, of k, of the clipped ones and of those that count; with the slopes of the first round, and which of it count.
template <int B> __device__ __forceinline__ void policy_sums(const PolicyArgs &a, int64_t s, int lo, int hi, double (&sums)[4], double (&slope)[kRound], uint32_t *counted)
{
    const int begin = lo + (int)threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[i] = 0.0;
#pragma unroll
    for (int u = 0; u < kRound; ++u) slope[u] = 0.0;
    uint32_t which = 0;
    if (begin < hi)
        policy_round<B>(a, s, begin, hi, [&](int u, const PolicyTerm &t) __attribute__((always_inline)) {
            sums[0] += t.loss;
            sums[1] += t.kl;
            sums[2] += t.over;
            sums[3] += 1.0;
            slope[u] = t.slope;
            which |= 1u << u;
        });
    *counted = which;
#pragma nounroll
    for (int i0 = begin + kRound * B; i0 < hi; i0 += kRound * B)
        policy_round<B>(a, s, i0, hi, [&](int, const PolicyTerm &t) __attribute__((always_inline)) {
            sums[0] += t.loss;
            sums[1] += t.kl;
            sums[2] += t.over;
            sums[3] += 1.0;
        });
}

// The sequence's results, and what the slopes are multiplied by.
__device__ __forceinline__ double policy_finish(const PolicyArgs &a, int64_t s, const double (&sums)[4], bool writes)
{
    const double many = fmax(sums[3], 1.0), share = a.average ? 1.0 / many : 1.0;
    if (writes && threadIdx.x == 0) {
        a.loss[s] = (float)(sums[0] * share);
        if (a.kl) a.kl[s] = (float)(sums[1] * share);
        if (a.clipped) a.clipped[s] = (float)(sums[2] / many);
    }
    return a.out ? (double)a.g[s] * share : 0.0;
}

// The gradient of the tokens from `from` on, in rounds of B.
template <int B> __device__ __forceinline__ void policy_slopes(const PolicyArgs &a, int64_t s, int from, int hi, double up)
{
#pragma nounroll
    for (int i0 = from + (int)threadIdx.x; i0 < hi; i0 += kRound * B) {
#pragma unroll
        for (int u = 0; u < kRound; ++u)
            if (i0 + u * B < hi) a.out[i0 + u * B] = 0.0f;
        policy_round<B>(a, s, i0, hi, [&](int u, const PolicyTerm &t) __attribute__((always_inline)) { a.out[i0 + u * B] = (float)(up * t.slope); });
    }
}

template <int B>
__global__ __launch_bounds__(B, 8) void policy_kernel(PolicyArgs a)
{
    __shared__ double red[B / 64 * 4];
    if (a.out) clear_outside<B>(a.out, a.offsets, a.sequences, a.tokens);
    const int64_t s = blockIdx.x;
    if (s >= a.sequences) return;
    const Span span = span_of(a.offsets, s, a.tokens);
    double sums[4], slope[kRound];
    uint32_t counted;
    policy_sums<B>(a, s, span.lo, span.hi, sums, slope, &counted);
    lanes_sum<B>(sums, red);
    const double up = policy_finish(a, s, sums, true);
    if (!a.out) return;
    const int begin = span.lo + (int)threadIdx.x;
#pragma unroll
    for (int u = 0; u < kRound; ++u)
        if (begin + u * B < span.hi) a.out[begin + u * B] = counted >> u & 1u ? (float)(up * slope[u]) : 0.0f;
    policy_slopes<B>(a, s, span.lo + kRound * B, span.hi, up);
}

__global__ __launch_bounds__(kPartThreads, 8) void policy_parts_kernel(PolicyArgs a, int parts, double *__restrict__ partial)
{
    __shared__ double red[kPartThreads / 64 * 4];
    const int64_t s = blockIdx.x / (uint32_t)parts;
    const Span mine = part_of(span_of(a.offsets, s, a.tokens), blockIdx.x % (uint32_t)parts, parts);
    double sums[4], slope[kRound];
    uint32_t counted;
    policy_sums<kPartThreads>(a, s, mine.lo, mine.hi, sums, slope, &counted);
    lanes_sum<kPartThreads>(sums, red);
    store_part(partial, sums);
}

// A workgroup a part; without a gradient, a workgroup a sequence.
__global__ __launch_bounds__(kPartThreads, 8) void policy_join_kernel(PolicyArgs a, int parts, const double *__restrict__ partial)
{
    __shared__ double red[kPartThreads / 64 * 4];
    const uint32_t each = a.out ? parts : 1;
    if (a.out) clear_outside<kPartThreads>(a.out, a.offsets, a.sequences, a.tokens);
    const int64_t s = blockIdx.x / each;
    if (s >= a.sequences) return;
    const int part = blockIdx.x % each;
    double sums[4];
    join_parts(partial, s, parts, sums, red);
    const double up = policy_finish(a, s, sums, part == 0);
    if (!a.out) return;
    const Span mine = part_of(span_of(a.offsets, s, a.tokens), part, parts);
    policy_slopes<kPartThreads>(a, s, mine.lo, mine.hi, up);
}

int launch_policy(const PolicyParams &p, hipStream_t st)
{
    if (p.sequences == 0 && !p.grad_logp) return AVQ_OK;
    const PolicyArgs a{p.logp, p.old, p.ref, p.advantage, p.mask, p.offsets, p.each, (int)p.tokens, p.sequences, p.average, 1.0 - p.clip_low, 1.0 + p.clip_high, p.kl_weight,
                       p.loss, p.kl, p.clipped, p.grad_loss, p.grad_logp};
    const int parts = sequence_parts(p.tokens, p.sequences, kPolicyParts);
    const int64_t behind = p.grad_logp ? p.tokens : 0;
    if (parts > 1) {
        policy_parts_kernel<<<dim3((unsigned)p.sequences * parts), dim3(kPartThreads), 0, st>>>(a, parts, (double *)p.scratch);
        AVQ_HIP(hipGetLastError());
        policy_join_kernel<<<dim3(sequence_groups(behind, (int64_t)p.sequences * (p.grad_logp ? parts : 1))), dim3(kPartThreads), 0, st>>>(a, parts, (const double *)p.scratch);
    } else {
        const int threads = sequence_threads(p.tokens, p.sequences);
        const auto kernel = threads == 64 ? policy_kernel<64> : threads == 256 ? policy_kernel<256> : policy_kernel<1024>;
        kernel<<<dim3(sequence_groups(behind, p.sequences)), dim3(threads), 0, st>>>(a);
    }
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

} // namespace avq
