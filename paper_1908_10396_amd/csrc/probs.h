// What the kernels of the log probabilities and of their gradient share.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "avq_internal.h"

namespace avq {

// sum + low + v, low what sum has no room for: what lies beside the maximum's 1 keeps its own relative accuracy, and with it log p
// of an answer that has nearly all of the probability.
__device__ __forceinline__ void add_wide(float &sum, float &low, float v)
{
    const float s = sum + v, part = s - sum;
    low += (sum - (s - part)) + (v - part);
    sum = s;
}

// log(sum + low)
__device__ __forceinline__ float log_wide(float sum, float low)
{
    const float beside = (sum - 1.0f) + low;
    return fabsf(beside) < 0.5f ? log1pf(beside) : logf(sum + low);
}

// Running statistics of logits: the maximum m of the products, and over the logits s, in units of log 2 and relative to that of m,
// the sums of 2^s (l + low; that of m itself is 1, exactly) and of 2^s s.
struct Stat { float m, l, low, t; };

// s where 2^s s is added: that is 0 wherever 2^s is, also where s is -inf (a masked row)
__device__ __forceinline__ float times_power(float s) { return fmaxf(s, -200.0f); }
// sums that are relative to a maximum that is `down` below the new one
__device__ __forceinline__ float lowered(float t, float l, float down, float f) { return f == 0.0f ? 0.0f : f * __fmaf_rn(l, down, t); }

// Of two sets of logits; one without any has m = -inf and sums of 0. c2: from products to logits.
__device__ __forceinline__ Stat join(const Stat &a, const Stat &b, float c2)
{
    const float m = fmaxf(a.m, b.m);
    if (!(m > -INFINITY)) return Stat{m, a.l + b.l, 0.0f, a.t + b.t}; // (NaN goes on in the sums)
    const float da = a.m > -INFINITY ? (a.m - m) * c2 : 0.0f, db = b.m > -INFINITY ? (b.m - m) * c2 : 0.0f;
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    Stat s{m, a.l * fa, a.low * fa, lowered(a.t, a.l, da, fa) + lowered(b.t, b.l, db, fb)};
    add_wide(s.l, s.low, b.l * fb);
    s.low = __fmaf_rn(b.low, fb, s.low);
    return s;
}

// of the lane `mask` away
__device__ __forceinline__ Stat across(const Stat &a, int mask) { return Stat{__shfl_xor(a.m, mask, 64), __shfl_xor(a.l, mask, 64), __shfl_xor(a.low, mask, 64), __shfl_xor(a.t, mask, 64)}; }
__device__ __forceinline__ float4 packed(const Stat &a) { return make_float4(a.m, a.l, a.low, a.t); }
__device__ __forceinline__ Stat unpacked(const float4 &v) { return Stat{v.x, v.y, v.z, v.w}; }

// The pass that forms a query's statistics: one query whose rows fit four loads of a wave goes by rows (two, by a kernel of two sums a
// row: 133 against 117 us through the matrix instructions, 1,183,514 x 100 fp32); up to 64 queries the rows are streamed, once for every 16,
// 32 or 64 queries, as many as LDS has room for (stream_tile: rows of 1,024 fp32 once for 16, of 1,024 bf16 for 32); more go by tiles
// of a matrix product. 64 is where the tiles' 128 queries are half full, whatever the type and length; a crossing of each was not measured.
enum { kByRow = 0, kByStream = 1, kByTiles = 2 };
inline int prob_path(int size, int d, int nq) { return nq > 64 ? kByTiles : nq == 1 && (size_t)d * size <= 64 * 16 * 4 ? kByRow : kByStream; }
// Lanes of a row that goes by rows.
inline int row_lanes(int size, int d)
{
    const int loads = (d * size + 15) / 16;
    return loads <= 16 ? 16 : loads <= 32 ? 32 : 64;
}

// Dynamic LDS of the kernel that finishes a query: the query; candidate groups, then the keys of 32 rows for each of the k
// best groups; the rows that may be among the k best; the groups.
constexpr size_t kFinishLds = kMaxDynLds - 16 * 1024;
constexpr int kFinishList = 2048; // candidate groups that are kept
__host__ __device__ constexpr int finish_best(int k) { return k < 192 ? 256 : k + 64; }
inline size_t finish_lds(int d, int k)
{
    return (size_t)(d + 31) / 32 * 32 * 4 + (k == 0 ? 0 : (size_t)std::max(32 * k, kFinishList) * 8 + (size_t)finish_best(k) * 8 + (size_t)k * 4);
}

// The gradient by one pass over the rows (probs_grad_few.hip): whether it takes a call, what it needs, and the pass.
bool grad_few_takes(int type, int d, int nq, int given);
size_t grad_few_scratch_bytes(int type, int d, int nq);
int launch_grad_few(const ProbGradParams &p, hipStream_t st);

} // namespace avq
