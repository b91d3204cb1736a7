// Log probabilities of rows of a table under the softmax of a query's inner products with all rows:
//   s_i = c <q, x_i>,  lse = log sum_i e^s_i,  log p_i = s_i - lse,  H = lse - sum_i p_i s_i,
// and the k rows of largest s_i (ties: the lower id). One pass over the rows keeps, per query and lane, the running maximum m
// and the sums of e^(s - m) and e^(s - m) (s - m) in fp32, the first with what fp32 has no room for; the logits are never stored. For the best rows it leaves the
// largest inner product of every 32 rows; the k groups with the largest of those hold the k best rows, which are scored again.
// A call: one query, 1,183,514 x 100 fp32, ten best 97 us (pass 72, 6.5 TB/s); 24 queries, 670,091 x 1,024 bf16, twenty best 315 us (pass 256,
// 5.3 TB/s); 2,048 queries, 1,183,514 x 100 fp32 1.95 ms (pass 1.69: 0.86 PFLOP/s of f16, three products for one).
#include "mma_tiles.h"
#include "prob_score.h"
#include "probs.h"
#include "row_types.h"
#include "wg_select.h"

#include <type_traits>

namespace avq {

// ---- a few queries: the rows streamed once -------------------------------------------------

constexpr int kStreamThreads = 256, kStreamWaves = kStreamThreads / 64;
constexpr int kStreamSteps = 8; // steps of a batch: 16 loads of 16 bytes a lane, of which the next batch's are in flight too

// A wave takes 32 rows at a time, a query tile is QT x 16 queries. The rows' operands come straight from memory (a lane's 16
// bytes are the matrix instruction's layout), the queries' from LDS, where they lie in the same order (QLDS), or from memory.
// Bound by memory; a batch is asked for while the one before is multiplied.
template <class T, int QT, bool ALIGNED, bool QLDS>
__global__ __launch_bounds__(kStreamThreads, 2) void prob_stream_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, int nq, int64_t ld_q,
                                                                        float c2, int negate, float4 *__restrict__ stats, float *__restrict__ gmax, int64_t gstride)
{
    extern __shared__ Frag qs[]; // [step][QT][64]
    __shared__ float4 joined[kStreamWaves][QT * 16];
    constexpr int S = kStepElems<T>, E = kFragElems<T>, NB = kStreamSteps;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r16 = lane & 15, kg = lane >> 4;
    const int q0 = blockIdx.y * QT * 16;
    const int steps = (d + S - 1) / S;
    // The last step's 16 bytes may run past the row's end, into what lies between it and the next row or into that: they are read all
    // the same and masked; lanes whose bytes lie past the end altogether read the row's first. The tile that holds the last row, and
    // rows shorter than 16 bytes, go by themselves.
    const int k_last = (steps - 1) * S + kg * E, k_read = k_last < d ? k_last : 0;
    uint32_t mask[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (sizeof(T) == 4) mask[w] = k_last + w < d ? ~0u : 0u;
        else mask[w] = (k_last + 2 * w < d ? 0xffffu : 0u) | (k_last + 2 * w + 1 < d ? 0xffff0000u : 0u);
    }
    float m[QT], l[QT], low[QT], t[QT];
    f32x4 acc[2][QT];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        m[i] = -INFINITY;
        l[i] = low[i] = t[i] = 0.0f;
        acc[0][i] = acc[1][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int64_t tiles = (n + 31) / 32, whole_tiles = d >= E ? (n - 1) / 32 : 0, stride = (int64_t)gridDim.x * kStreamWaves;
    const int batches = (steps + NB - 1) / NB;

    struct Batch { Frag a[2][NB]; };
    auto fetch = [&](Batch &f, int64_t tile, int batch) __attribute__((always_inline)) {
        const T *p0 = x + (tile * 32 + r16) * ld_x, *p1 = p0 + 16 * ld_x;
        const int s0 = batch * NB;
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            if (s0 + u >= steps) break;
            const int k = s0 + u == steps - 1 ? k_read : (s0 + u) * S + kg * E;
            f.a[0][u] = load_whole<T, ALIGNED>(p0 + k);
            f.a[1][u] = load_whole<T, ALIGNED>(p1 + k);
        }
    };
    int64_t tile = (int64_t)blockIdx.x * kStreamWaves + wave;
    Batch here, next;
    if (tile < whole_tiles) fetch(here, tile, 0);
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
    auto multiply_step = [&](int s, const Frag &a0, const Frag &a1) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < QT; ++i) {
            Frag b{};
            if (QLDS) {
                b = qs[(s * QT + i) * 64 + lane];
            } else {
                const int row = q0 + i * 16 + r16;
                if (row < nq) b = load_frag<T, false>(q + (int64_t)row * ld_q, s * S + kg * E, d);
                if (negate) b = negated<T>(b);
            }
            acc[0][i] = mma16(a0, b, acc[0][i], T{});
            acc[1][i] = mma16(a1, b, acc[1][i], T{});
        }
    };
    auto multiply = [&](Batch &f, int batch) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            const int s = batch * NB + u;
            if (s >= steps) break;
            if (s == steps - 1) {
#pragma unroll
                for (int w = 0; w < 4; ++w) { f.a[0][u].w[w] &= mask[w]; f.a[1][u].w[w] &= mask[w]; }
            }
            multiply_step(s, f.a[0][u], f.a[1][u]);
        }
    };
    // lane: query i * 16 + (lane & 15), rows 4 (lane >> 4) + 0 .. 3 of either half
    auto take = [&](int64_t tile) __attribute__((always_inline)) {
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
                    t[i] = lowered(t[i], l[i], down, f);
                    l[i] *= f;
                    low[i] *= f;
                }
                m[i] = top;
            }
            const float base = m[i] > -INFINITY ? m[i] : 0.0f;
            float sum = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (h * 16 + kg * 4 + r < valid) {
                        const float s2 = (acc[h][i][r] - base) * c2, e = __builtin_amdgcn_exp2f(s2);
                        sum += e;
                        t[i] = __fmaf_rn(e, times_power(s2), t[i]);
                    }
            add_wide(l[i], low[i], sum);
            if (gmax) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                if (kg == 0 && q0 + i * 16 + r16 < nq) gmax[(int64_t)(q0 + i * 16 + r16) * gstride + tile] = top;
            }
            acc[0][i] = acc[1][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    };
    if (tile < whole_tiles) {
        int batch = 0;
        // one batch: asks for the one after it, multiplies, and at a tile's end takes its logits; false after the last
        auto turn = [&](Batch &now, Batch &then) __attribute__((always_inline)) {
            int64_t then_tile = tile;
            int then_batch = batch + 1;
            if (then_batch == batches) { then_batch = 0; then_tile += stride; }
            const bool more = then_tile < whole_tiles;
            if (more) fetch(then, then_tile, then_batch);
            multiply(now, batch);
            if (then_batch == 0) take(tile);
            tile = then_tile;
            batch = then_batch;
            return more;
        };
        while (turn(here, next) && turn(next, here)) {}
    }
    for (; tile < tiles; tile += stride) {
        const int64_t r0 = tile * 32 + r16, r1 = r0 + 16;
        const T *p0 = x + (r0 < n ? r0 : n - 1) * ld_x, *p1 = x + (r1 < n ? r1 : n - 1) * ld_x;
#pragma unroll 1
        for (int s = 0; s < steps; ++s) multiply_step(s, load_frag<T, ALIGNED>(p0, s * S + kg * E, d), load_frag<T, ALIGNED>(p1, s * S + kg * E, d));
        take(tile);
    }
    // the four lanes of a query, then the waves
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        Stat a{m[i], l[i], low[i], t[i]};
#pragma unroll
        for (int x16 = 16; x16 < 64; x16 *= 2) a = join(a, across(a, x16), c2);
        if (kg == 0) joined[wave][i * 16 + r16] = packed(a);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < QT * 16; i += kStreamThreads) {
        if (q0 + i >= nq) continue;
        Stat a = unpacked(joined[0][i]);
        for (int w = 1; w < kStreamWaves; ++w) a = join(a, unpacked(joined[w][i]), c2);
        stats[(size_t)blockIdx.x * nq + q0 + i] = packed(a);
    }
}

// ---- one query: rows by lanes side by side ---------------------------------------------------------

constexpr int kRowThreads = 256, kRowWaves = kRowThreads / 64;
constexpr int kRowLoads = 8; // of 16 bytes a lane in flight, and as many of the next rows

// A row by L lanes that hold F times 16 bytes of it each, so that a wave's loads lie side by side in memory (the matrix
// instruction's layout reads 64 bytes here and there). Bound by memory: 1,183,514 x 100 fp32, one query, 71 us (6.7 TB/s), against 98
// through the matrix instructions; with loads that stay in the caches, or with twice the waves, 84. A wave takes 32 rows at a time,
// U x 64 / L of them at once; the lanes' parts of U rows' products are added up together, each exchange halving the rows a lane has.
template <class T, int L, int F, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void prob_row_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, float c2,
                                                               float4 *__restrict__ stats, float *__restrict__ gmax)
{
    constexpr int E = kFragElems<T>, U = kRowLoads / F, kGroups = 64 / L, kAtOnce = U * kGroups, kTurns = 32 / kAtOnce;
    static_assert(kTurns >= 1 && kTurns * kAtOnce == 32, "a wave's 32 rows");
    __shared__ float4 joined[kRowWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in_row = lane % L, group = lane / L;
    const bool mine = in_row < U; // lanes of a row beyond hold the same sums
    float qf[F][E];
    int at[F];         // the lane's elements
    uint32_t mask[F][4]; // those before the row's end
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int k = (f * L + in_row) * E;
        at[f] = k < d ? k : 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (sizeof(T) == 4) mask[f][w] = k + w < d ? ~0u : 0u;
            else mask[f][w] = (k + 2 * w < d ? 0xffffu : 0u) | (k + 2 * w + 1 < d ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) qf[f][e] = k + e < d ? (c2 < 0.0f ? -1.0f : 1.0f) * to_f32(q[k + e]) : 0.0f;
    }
    c2 = fabsf(c2); // (so that the largest product is the largest logit)
    float m = -INFINITY, l = 0.0f, low = 0.0f, t = 0.0f, top = -INFINITY;
    // (16 bytes of the last row may run past the last element: the tile that holds it, and rows shorter than 16 bytes, go by themselves)
    const int64_t tiles = (n + 31) / 32, whole = d >= E ? (n - 1) / 32 : 0, stride = (int64_t)gridDim.x * kRowWaves;

    struct Rows { Frag f[U][F]; };
    auto row_of = [&](int64_t tile, int turn, int u) __attribute__((always_inline)) { return tile * 32 + turn * kAtOnce + u * kGroups + group; };
    auto fetch = [&](Rows &r, int64_t tile, int turn) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const T *p = x + row_of(tile, turn, u) * ld_x + at[f];
                r.f[u][f] = ONCE ? load_once<T>(p) : load_whole<T, false>(p);
            }
    };
    auto take = [&](const Rows &r, int64_t tile, int turn) __attribute__((always_inline)) {
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = 0.0f;
#pragma unroll
            for (int f = 0; f < F; ++f) {
                Frag v = r.f[u][f];
#pragma unroll
                for (int w = 0; w < 4; ++w) v.w[w] &= mask[f][w];
                T e[E];
                __builtin_memcpy(e, &v, 16);
#pragma unroll
                for (int j = 0; j < E; ++j) s[u] = __fmaf_rn(qf[f][j], to_f32(e[j]), s[u]);
            }
        }
        // U sums over L lanes: after log U exchanges lane l has those of row l % U, over the lanes alike but for these bits
#pragma unroll
        for (int w = 1; w < U; w <<= 1) {
            const bool upper = (lane & w) != 0;
#pragma unroll
            for (int u = 0; u < U; u += 2 * w) {
                const float give = upper ? s[u] : s[u + w], keep = upper ? s[u + w] : s[u];
                s[u] = keep + __shfl_xor(give, w, 64);
            }
        }
        float sum = s[0];
#pragma unroll
        for (int w = U; w < L; w <<= 1) sum += __shfl_xor(sum, w, 64);
        const int64_t row = row_of(tile, turn, in_row % U);
        const bool real = mine && row < n;
        if (real && sum > m) {
            if (m > -INFINITY) {
                const float down = (m - sum) * c2, f = __builtin_amdgcn_exp2f(down);
                t = lowered(t, l, down, f);
                l *= f;
                low *= f;
            }
            m = sum;
        }
        const float s2 = m > -INFINITY ? (sum - m) * c2 : sum, e = __builtin_amdgcn_exp2f(s2);
        if (real) {
            add_wide(l, low, e);
            t = __fmaf_rn(e, times_power(s2), t);
            top = fmaxf(top, sum);
        }
        if (turn == kTurns - 1 && gmax) {
            float g = top;
#pragma unroll
            for (int w = 1; w < 64; w <<= 1) g = fmaxf(g, __shfl_xor(g, w, 64));
            if (lane == 0) gmax[tile] = g;
            top = -INFINITY;
        }
    };
    int64_t tile = (int64_t)blockIdx.x * kRowWaves + wave;
    Rows here, next;
    if (tile < whole) {
        int turn = 0;
        fetch(here, tile, 0);
        auto step = [&](Rows &now, Rows &then) __attribute__((always_inline)) {
            int64_t then_tile = tile;
            int then_turn = turn + 1;
            if (then_turn == kTurns) { then_turn = 0; then_tile += stride; }
            const bool more = then_tile < whole;
            if (more) fetch(then, then_tile, then_turn);
            take(now, tile, turn);
            tile = then_tile;
            turn = then_turn;
            return more;
        };
        while (step(here, next) && step(next, here)) {}
    }
    for (; tile < tiles; tile += stride)
#pragma unroll 1
        for (int turn = 0; turn < kTurns; ++turn) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const int64_t row = row_of(tile, turn, u);
                    here.f[u][f] = load_frag<T, false>(x + (row < n ? row : n - 1) * ld_x, (f * L + in_row) * E, d);
                }
            take(here, tile, turn);
        }
    Stat a{m, l, low, t};
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) a = join(a, across(a, w), c2);
    if (lane == 0) joined[wave] = packed(a);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kRowWaves; ++w) a = join(a, unpacked(joined[w]), c2);
        stats[blockIdx.x] = packed(a);
    }
}

// ---- many queries: tiles of a matrix product ----------------------------------------------------

// Statistics of 128 queries over a part of the rows, 256 rows at a time; a lane has two queries, 64 of a tile's rows of each.
// X: the launch's rows, Q: all queries, negated where the scale is. A lane's sums are relative to fl(m c2), one operation a logit instead
// of two; at the end they are made relative to m itself, whose own term is known to the bit. Beyond kTame fl's rounding would be an
// exponent of its own: there differences are taken first.
constexpr float kTame = 0x1p18f;

template <class H, bool SPLIT, bool BEST>
__global__ __launch_bounds__(kTileThreads, 2) void prob_tile_kernel(Rows16 X, Rows16 Q, int steps, float c2, const float *__restrict__ x_inv, const float *__restrict__ tile_inv, const float *__restrict__ q_inv, int parts,
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
    float cq[2], m[2], l[2], low[2], t[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        cq[j] = c2;
        if (SPLIT) {
            const int64_t q = min(q0 + acc_col(j), Q.rows - 1);
            cq[j] = c2 * q_inv[q];
        }
        m[j] = -INFINITY;
        l[j] = low[j] = t[j] = 0.0f;
    }
    typedef RowCopies<SPLIT, true> Copies;
    float ahead = SPLIT && count > 0 ? tile_inv[first] : 1.0f; // (asked for a tile before it is needed)
    run_tiles<H, SPLIT, SPLIT || BEST, Copies>(X, Q, steps, count, lds, [&](int i, Copies &c) { c.seek(X, (first + i) * kTileM, Q, q0); },
        [&](int i, f32x16 (&acc)[4][2]) {
            float unit = ahead; // of the products
            if (SPLIT) ahead = tile_inv[first + (i + 1 < count ? i + 1 : i)];
            if (SPLIT && unit == 0.0f) {
                unit = 1.0f;
                // (the last tile's rows past the end have a place too)
                const float *inv = x_inv + (first + i) * kTileM + (wave >> 1) * 128 + 4 * (lane >> 5);
#pragma unroll
                for (int a = 0; a < 4; ++a)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const float4 v = *(const float4 *)(inv + a * 32 + b * 8);
                        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int r = 0; r < 4; ++r) // (an odd row's 0 times infinity: -infinity)
#pragma unroll
                            for (int j = 0; j < 2; ++j) acc[a][j][4 * b + r] = fmaxf(acc[a][j][4 * b + r] * e[r], -INFINITY);
                    }
            }
            const int64_t row0 = (first + i) * kTileM;
            const bool whole = row0 + kTileM <= X.rows;
            const int valid = whole ? kTileM : (int)(X.rows - row0);
            auto take = [&](auto tail) {
                constexpr bool TAIL = decltype(tail)::value;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float group[4], least = INFINITY;
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        float g = -INFINITY;
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (!TAIL || acc_row(a, r) < valid) {
                                g = fmaxf(g, acc[a][j][r]);
                                if (!TAIL) least = fminf(least, acc[a][j][r]);
                            }
                        group[a] = SPLIT ? g * unit : g;
                    }
                    const float top = fmaxf(fmaxf(group[0], group[1]), fmaxf(group[2], group[3]));
                    if (top > m[j]) {
                        if (m[j] > -INFINITY) {
                            const float from = m[j] * cq[j], to = top * cq[j];
                            const float down = fmaxf(fabsf(from), fabsf(to)) <= kTame ? from - to : (m[j] - top) * cq[j], f = __builtin_amdgcn_exp2f(down);
                            t[j] = lowered(t[j], l[j], down, f);
                            l[j] *= f;
                            low[j] *= f;
                        }
                        m[j] = top;
                    }
                    const float base = m[j] > -INFINITY ? m[j] : 0.0f, shift = -(base * cq[j]);
                    const bool tame = fabsf(shift) <= kTame;
                    const float to_logit = SPLIT ? unit * cq[j] : cq[j];
                    // four sums side by side, then one
                    float ls[4] = {}, ts[4] = {};
                    auto sums = [&](auto any_size) __attribute__((always_inline)) {
#pragma unroll
                        for (int a = 0; a < 4; ++a)
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                if (!TAIL || acc_row(a, r) < valid) {
                                    float s2 = __fmaf_rn(acc[a][j][r], to_logit, shift);
                                    if (decltype(any_size)::value) s2 = tame ? s2 : (SPLIT ? __fmaf_rn(acc[a][j][r], unit, -base) : acc[a][j][r] - base) * cq[j];
                                    const float e = __builtin_amdgcn_exp2f(s2);
                                    ls[a] += e;
                                    ts[a] = __fmaf_rn(e, decltype(any_size)::value ? times_power(s2) : s2, ts[a]);
                                }
                    };
                    // (also where the least logit is -inf)
                    if (TAIL || __any(!(tame && __fmaf_rn(least, to_logit, shift) > -INFINITY))) sums(std::true_type{});
                    else sums(std::false_type{});
#pragma unroll
                    for (int a = 0; a < 4; ++a) add_wide(l[j], low[j], ls[a]);
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
        Stat a{m[j], l[j], low[j], t[j]};
        if (m[j] > -INFINITY) {
            const float s = m[j] * cq[j], over = fabsf(s) <= kTame ? __fmaf_rn(m[j], cq[j], -s) : 0.0f, up = __builtin_amdgcn_exp2f(-over); // (m's own term is 2^over)
            a.t = up * __fmaf_rn(-over, l[j], t[j]);
            a.l = 1.0f;
            a.low = 0.0f;
            add_wide(a.l, a.low, up * ((l[j] - __builtin_amdgcn_exp2f(over)) + low[j]));
        }
        a = join(a, across(a, 32), cq[j]);
        const int64_t q = q0 + acc_col(j);
        if (lane < 32 && q < Q.rows) stats[(size_t)(place.part * 2 + (wave >> 1)) * Q.rows + q] = packed(a);
    }
}

// ---- what a query's statistics give ----------------------------------------------------------

__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f); // (-0 is 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// A workgroup a query: joins the statistics, scores the given rows and the best ones. Latency: the fewest steps that wait for
// one another.
template <int PATH, class T, int NT>
__global__ __launch_bounds__(NT) void prob_finish_kernel(const T *__restrict__ x, int64_t n, int d, int64_t ld_x, const T *__restrict__ q, int nq, int64_t ld_q, float scale, int row_lanes,
                                                         const float *__restrict__ x_inv, const float *__restrict__ q_inv, const uint32_t *__restrict__ odd_seen, const float4 *__restrict__ stats, int parts, const int32_t *__restrict__ ids, int given, float *__restrict__ logp_out,
                                                         float *__restrict__ lse_out, float *__restrict__ entropy_out, const float *__restrict__ gmax, int64_t gstride, int k,
                                                         int32_t *__restrict__ alt_ids, float *__restrict__ alt_logp)
{
    __shared__ WgSelectScratch sel;
    __shared__ Stat wave_stat[NT / 64];
    __shared__ uint32_t list_count, found_count, bound_shared;
    __shared__ u64 least_best;
    extern __shared__ char lds[];
    T *qs = (T *)lds;                                                // the query (4 bytes a coordinate)
    u64 *keys = (u64 *)(lds + (size_t)((d + 31) / 32 * 32) * 4);     // [max(32 k, kFinishList)]: candidate groups, then rows
    u64 *best = keys + std::max(32 * k, kFinishList);                // [finish_best(k)]
    uint32_t *groups = (uint32_t *)(best + finish_best(k));          // [k]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x;
    uint32_t *tops = (uint32_t *)keys;      // [NT / per] largest product of a class
    const bool by_parts = parts >= 4 * k; // the parts' largest products are classes enough
    uint32_t mine_top = 0;
    stage_query(qs, q + (int64_t)row * ld_q, d, scale < 0.0f, NT);
    // from products to logits, and to logits in units of log 2 as the pass has them
    float c = fabsf(scale), c2 = fabsf(scale) * 1.44269504088896341f;
    Scoring how{row_lanes, 1.0f};
    if (PATH == kByTiles && sizeof(T) == 4) {
        how.q_scale = 1.0f / (kRowUnit * q_inv[row]);
        c = c * q_inv[row];
        c2 = c2 * q_inv[row];
    }
    Stat a{-INFINITY, 0.0f, 0.0f, 0.0f};
    for (int p = tid; p < parts; p += NT) {
        const Stat v = unpacked(stats[(size_t)p * nq + row]);
        a = join(a, v, c2);
        if (by_parts) mine_top = max(mine_top, order_of(v.m));
    }
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) a = join(a, across(a, w), c2);
    if (lane == 0) wave_stat[wave] = a;
    if (tid == 0) { list_count = found_count = bound_shared = 0; least_best = ~0ull; }

    const uint32_t n_groups = (uint32_t)((n + 31) / 32);
    const float *gm = gmax + row * gstride;
    auto each_group = [&](auto &&fn) { // (four groups a load; the last four may lie past the end)
        constexpr int U = 4;
        for (uint32_t g0 = 4 * tid; g0 < n_groups; g0 += 4 * NT * U) {
            float4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = *(const float4 *)(gm + min(g0 + 4 * NT * u, (n_groups - 1) & ~3u));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float e[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t g = g0 + 4 * NT * u + i;
                    if (g < n_groups) fn(g, order_of(e[i]));
                }
            }
        }
    };
    // Classes of groups, 4 k or more where there are: the k-th largest of their maxima bounds the k-th largest group from below. A
    // class is what a few threads see of the parts or, where these are too few, of a pass over the groups.
    int per = 16; // threads a class
    const int seen = by_parts ? min(parts, NT) : NT; // threads that have seen any
    while (per > 1 && seen / per < 4 * k) per /= 2;
    const int classes = (seen + per - 1) / per;
    if (k > 0) {
        if (!by_parts) each_group([&](uint32_t, uint32_t o) { mine_top = max(mine_top, o); });
        for (int w = 1; w < per; w <<= 1) mine_top = max(mine_top, (uint32_t)__shfl_xor((int)mine_top, w, 64));
        // (the last bits make classes different; without them the bound is a little lower)
        if (tid % per == 0) tops[tid / per] = (mine_top & ~1023u) | (uint32_t)(1023 - tid / per);
    }
    __syncthreads();
    a = wave_stat[0];
    if (PATH == kByTiles && sizeof(T) == 4 && odd_seen[row]) a.l = NAN;
    for (int w = 1; w < NT / 64; ++w) a = join(a, wave_stat[w], c2);
    constexpr float ln2 = 0.693147180559945309f;
    const float log_l = log_wide(a.l, a.low), lse = __fmaf_rn(a.m, c, log_l);
    if (tid == 0) {
        lse_out[row] = lse;
        if (entropy_out) entropy_out[row] = log_l - ln2 * (a.t / a.l);
    }
    // s - lse from the parts that lse has, before it is rounded
    auto logp_of = [&](float product) { return __fmaf_rn(product - a.m, c, -log_l); };
    constexpr int kAhead = sizeof(T) == 4 ? 4 : 8; // (what 128 registers hold: four waves a SIMD)
    const int at_once = scored_at_once<PATH>(how);
    for (int j0 = wave * at_once; j0 < given; j0 += NT / 64 * at_once) {
        const int32_t *mine = ids + (int64_t)row * given + j0;
        auto real = [&](int i) { return j0 + i < given && mine[i] >= 0 && (int64_t)mine[i] < n; };
        score_rows<PATH, kAhead>(qs, d, how, [&](int i) { return x + (real(i) ? (int64_t)mine[i] * ld_x : 0); }, [&](int i) { return x_inv[real(i) ? mine[i] : 0]; },
                         [&](int i, float product) { if (j0 + i < given) logp_out[(int64_t)row * given + j0 + i] = real(i) ? logp_of(product) : -INFINITY; });
    }
    if (k == 0) return;

    if (tid < classes) {
        const uint32_t mine = tops[tid];
        uint32_t rank = 0;
#pragma unroll 8
        for (int o = 0; o < classes; ++o) rank += tops[o] > mine;
        if (rank == (uint32_t)k - 1) bound_shared = mine & ~1023u; // (k <= classes)
    }
    __syncthreads();
    const uint32_t bound = bound_shared;
    auto key_of = [](uint32_t g, uint32_t o) { return ((u64)o << 32) | (u64)(0xffffffffu - g); };
    each_group([&](uint32_t g, uint32_t o) {
        if (o < bound) return;
        const uint32_t at = atomicAdd(&list_count, 1u); // (the order of the list does not matter)
        if (at < kFinishList) keys[at] = key_of(g, o);
    });
    __syncthreads();
    const uint32_t listed = list_count;
    if (listed <= 256) {
        for (uint32_t i = tid; i < listed; i += NT) {
            const u64 mine = keys[i];
            uint32_t rank = 0;
#pragma unroll 8
            for (uint32_t o = 0; o < listed; ++o) rank += keys[o] > mine;
            if (rank < (uint32_t)k) groups[rank] = 0xffffffffu - (uint32_t)mine;
        }
        __syncthreads();
    } else {
        u64 least;
        if (listed <= kFinishList) least = wg_select_threshold_of([&](auto &&fn) { for (uint32_t i = tid; i < listed; i += NT) fn(keys[i]); }, k, &sel);
        else least = wg_select_threshold_of([&](auto &&fn) { each_group([&](uint32_t g, uint32_t o) { fn(key_of(g, o)); }); }, k, &sel);
        __syncthreads();
        if (tid == 0) list_count = 0;
        __syncthreads();
        auto choose = [&](u64 key) {
            if (key < least) return;
            const uint32_t at = atomicAdd(&list_count, 1u);
            if (at < (uint32_t)k) groups[at] = 0xffffffffu - (uint32_t)key;
        };
        if (listed <= kFinishList) for (uint32_t i = tid; i < listed; i += NT) choose(keys[i]);
        else each_group([&](uint32_t g, uint32_t o) { choose(key_of(g, o)); });
        __syncthreads();
    }
    const uint32_t chosen = min(min(list_count, listed), (uint32_t)k), rows = chosen * 32u;
    for (uint32_t i0 = wave * at_once; i0 < rows; i0 += NT / 64 * at_once) {
        auto id_of = [&](int i) { return (int64_t)groups[(i0 + i) / 32] * 32 + ((i0 + i) & 31); };
        auto row_of = [&](int i) { return min(i0 + i < rows ? id_of(i) : 0, n - 1); };
        score_rows<PATH, kAhead>(qs, d, how, [&](int i) { return x + row_of(i) * ld_x; }, [&](int i) { return x_inv[row_of(i)]; },
                         [&](int i, float product) {
                             if (i0 + i >= rows) return;
                             const int64_t id = id_of(i);
                             keys[i0 + i] = id < n ? ((u64)order_of(product) << 32) | (u64)(0xffffffffu - (uint32_t)id) : 0;
                         });
    }
    __syncthreads();
    // The best row of every chosen group: with k of them, the least of those bounds the k-th best row from below.
    if (chosen == (uint32_t)k) {
        for (uint32_t i = tid; i < rows; i += NT) { // (32 lanes a group)
            u64 top = keys[i];
#pragma unroll
            for (int w = 1; w < 32; w <<= 1) {
                const u64 o = ((u64)(uint32_t)__shfl_xor((int)(top >> 32), w, 64) << 32) | (uint32_t)__shfl_xor((int)(uint32_t)top, w, 64);
                top = o > top ? o : top;
            }
            if ((i & 31) == 0) atomicMin(&least_best, top);
        }
        __syncthreads();
    }
    const u64 floor_key = chosen == (uint32_t)k ? least_best : 1ull;
    for (uint32_t i = tid; i < rows; i += NT)
        if (keys[i] >= floor_key) {
            const uint32_t at = atomicAdd(&found_count, 1u);
            if (at < (uint32_t)finish_best(k)) best[at] = keys[i];
        }
    __syncthreads();
    uint32_t found = found_count;
    if (found > (uint32_t)finish_best(k)) { // many rows alike
        const u64 kth = wg_select_threshold_of([&](auto &&fn) { for (uint32_t i = tid; i < rows; i += NT) if (keys[i]) fn(keys[i]); }, k, &sel);
        __syncthreads();
        if (tid == 0) found_count = 0;
        __syncthreads();
        for (uint32_t i = tid; i < rows; i += NT)
            if (keys[i] && keys[i] >= kth) {
                const uint32_t at = atomicAdd(&found_count, 1u);
                if (at < (uint32_t)k) best[at] = keys[i];
            }
        __syncthreads();
        found = min(found_count, (uint32_t)k);
    }
    for (uint32_t i = tid; i < found; i += NT) {
        const u64 mine = best[i];
        uint32_t rank = 0;
#pragma unroll 4
        for (uint32_t o = 0; o < found; ++o) rank += best[o] > mine;
        if (rank >= (uint32_t)k) continue;
        alt_ids[(int64_t)row * k + rank] = (int32_t)(0xffffffffu - (uint32_t)mine);
        alt_logp[(int64_t)row * k + rank] = logp_of(value_of((uint32_t)(mine >> 32)));
    }
}

// ---- launches ----------------------------------------------------------------------------------

constexpr int kRowGroups = 512; // two a compute unit

// Workgroups that share the rows of the stream.
static int stream_groups(int64_t n, int query_tiles)
{
    const int64_t tiles = (n + 31) / 32, most = std::max(1, 512 / query_tiles); // two workgroups a compute unit
    return (int)std::max<int64_t>(1, std::min<int64_t>((tiles + kStreamWaves - 1) / kStreamWaves, most));
}

static int row_groups(int64_t n) { return (int)std::min<int64_t>(((n + 31) / 32 + kRowWaves - 1) / kRowWaves, kRowGroups); }

// Query tiles of 16 that a workgroup takes: as many as fit LDS beside another workgroup's, at most 4 (64 queries).
static int stream_tile(int type, int d, int nq)
{
    const size_t step = 64 * sizeof(Frag), bytes = step * (size_t)((d * type_bytes(type) + 63) / 64);
    int qt = 1;
    while (qt < 4 && qt * 16 < nq && 2 * qt * bytes <= 80 * 1024) qt *= 2;
    return qt;
}

constexpr int kTileGroups = 512; // two workgroups a compute unit
constexpr size_t kPackBytes = (size_t)1 << 30; // most that packed rows take at a time
constexpr size_t kGroupBytes = (size_t)1 << 30; // most that the groups' maxima of several query tiles take

// Queries that a call takes at a time: all of them, unless the maxima of their groups would exceed kGroupBytes (7,168 for 1,183,514 rows);
// then parts of equal size, whole query tiles.
static int queries_at_once(int type, int64_t n, int d, int nq, int k)
{
    if (k == 0 || prob_path(type_bytes(type), d, nq) != kByTiles) return nq;
    const size_t each = (size_t)((n + kTileM - 1) / kTileM) * (kTileM / 32) * sizeof(float);
    const int64_t most = std::max<int64_t>(1, (int64_t)(kGroupBytes / each) / kTileN) * kTileN;
    if (nq <= most) return nq;
    const int64_t parts = (nq + most - 1) / most;
    return (int)(((nq + parts - 1) / parts + kTileN - 1) / kTileN * kTileN);
}

struct ProbScratch {
    float4 *stats; float *gmax; int64_t gstride;
    int groups, qt, query_tiles;                         // stream
    bool pack; int steps, parts, launches; int64_t part; // tiles: steps of an inner product, rows a launch
    uint16_t *x16, *q16; float *q_inv, *x_inv, *tile_inv; OddRows odd;
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
    const int path = prob_path(type_bytes(p.type), p.d, p.nq);
    if (path != kByTiles) {
        s.qt = stream_tile(p.type, p.d, p.nq);
        s.query_tiles = (p.nq + 16 * s.qt - 1) / (16 * s.qt);
        s.groups = path == kByRow ? row_groups(p.n) : stream_groups(p.n, s.query_tiles);
        s.stats = (float4 *)take((size_t)s.groups * p.nq * sizeof(float4));
    } else {
        const bool split = p.type == AVQ_F32;
        s.steps = split ? steps_of<true>(p.d) : steps_of<false>(p.d);
        const size_t row_bytes = (size_t)s.steps * kStepBytes; // of a packed row
        // (base == NULL: the size for rows that need packing, whatever their place and stride)
        s.pack = !base || p.type == AVQ_F32 || p.d % 32 != 0 || (uintptr_t)p.points % 16 != 0 || p.ld_points % 8 != 0 || p.ld_points >= kMaxRow16;
        s.part = p.n;
        if (s.pack) s.part = std::min<int64_t>(p.n, std::max<int64_t>(65536, (int64_t)(kPackBytes / row_bytes) / kTileM * kTileM));
        s.launches = (int)((p.n + s.part - 1) / s.part);
        s.query_tiles = (p.nq + kTileN - 1) / kTileN;
        s.parts = parts_for((s.part + kTileM - 1) / kTileM, s.query_tiles, kTileGroups);
        // (as many statistics with one launch as with several: the number of parts only falls with the rows a launch has)
        s.stats = (float4 *)take((size_t)s.launches * std::max(s.parts, parts_for((p.n + kTileM - 1) / kTileM, s.query_tiles, kTileGroups)) * 2 * p.nq * sizeof(float4));
        s.q16 = (uint16_t *)take(packed_bytes(p.nq, s.steps));
        s.q_inv = (float *)take((size_t)p.nq * sizeof(float));
        if (split) {
            const size_t tiles = (size_t)(p.n + kTileM - 1) / kTileM;
            s.x_inv = (float *)take(tiles * kTileM * sizeof(float));
            s.tile_inv = (float *)take(tiles * sizeof(float));
            s.odd = OddRows{(uint32_t *)take(sizeof(uint32_t)), (uint32_t *)take((size_t)p.n * sizeof(uint32_t)), (uint32_t *)take((size_t)p.nq * sizeof(uint32_t))};
        }
        if (s.pack) s.x16 = (uint16_t *)take(packed_bytes(s.part, s.steps));
    }
    s.gmax = p.k > 0 ? (float *)take((size_t)s.gstride * p.nq * sizeof(float)) : nullptr;
    s.bytes = at;
    return s;
}

size_t log_probs_scratch_bytes(int type, int64_t n, int d, int nq, int given, int k)
{
    (void)given;
    ProbParams p{};
    p.type = type; p.n = n; p.d = d; p.nq = queries_at_once(type, n, d, nq, k); p.k = k;
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

template <class T, int L, int F>
static int row_run(const ProbParams &p, const ProbScratch &s, hipStream_t st)
{
    const float c2 = p.scale * 1.44269504088896341f;
    auto run = [&](auto kernel) { kernel<<<dim3(s.groups), dim3(kRowThreads), 0, st>>>((const T *)p.points, p.n, p.d, p.ld_points, (const T *)p.queries, c2, s.stats, s.gmax); };
    // what the Infinity Cache (256 MB) does not hold from one call to the next is loaded past it
    if ((size_t)p.n * p.d * sizeof(T) > ((size_t)256 << 20)) run(prob_row_kernel<T, L, F, true>);
    else run(prob_row_kernel<T, L, F, false>);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T>
static int row_sized(const ProbParams &p, const ProbScratch &s, hipStream_t st)
{
    const int lanes = row_lanes(sizeof(T), p.d), loads = (p.d + kFragElems<T> - 1) / kFragElems<T>; // of 16 bytes
    if (lanes == 16) return row_run<T, 16, 1>(p, s, st);
    if (lanes == 32) return row_run<T, 32, 1>(p, s, st);
    if (loads <= 64) return row_run<T, 64, 1>(p, s, st);
    return loads <= 128 ? row_run<T, 64, 2>(p, s, st) : row_run<T, 64, 4>(p, s, st);
}

template <class T, bool ALIGNED>
static int stream_sized(const ProbParams &p, const ProbScratch &s, hipStream_t st)
{
    // beyond what LDS holds for 16 queries (10,000 bytes a query), the queries' operands come from the caches
    if ((size_t)p.d * sizeof(T) > 8192) return stream_run<T, 1, ALIGNED, false>(p, s, st);
    if (s.qt == 1) return stream_run<T, 1, ALIGNED, true>(p, s, st);
    return s.qt == 2 ? stream_run<T, 2, ALIGNED, true>(p, s, st) : stream_run<T, 4, ALIGNED, true>(p, s, st);
}

// again: a further part of the queries; rows that were laid out at once are there.
template <class H, bool SPLIT>
static int tiles_run(const ProbParams &p, const ProbScratch &s, bool again, hipStream_t st)
{
    const bool laid_out = again && s.launches == 1;
    const int size = type_bytes(p.type);
    const float c2 = fabsf(p.scale) * 1.44269504088896341f;
    const Rows16 Q = packed_rows(s.q16, p.nq);
    if (SPLIT) {
        AVQ_TRY(launch_pack_queries((const float *)p.queries, p.nq, p.d, p.ld_queries, s.steps, Q, s.q_inv, OddRows{again ? nullptr : s.odd.count, nullptr, s.odd.seen}, p.scale < 0.0f, st));
        if (!again) AVQ_TRY(launch_row_inverses((const float *)p.points, p.n, p.d, p.ld_points, s.x_inv, s.tile_inv, s.odd, st));
        AVQ_TRY(launch_odd_rows((const float *)p.points, p.d, p.ld_points, (const float *)p.queries, p.nq, p.ld_queries, p.scale < 0.0f, s.odd, st));
    } else {
        AVQ_TRY(launch_pack_rows(p.queries, p.type, p.nq, p.d, p.ld_queries, s.steps, Q, nullptr, p.scale < 0.0f, st));
    }
    static LdsLimitOnce with_best, without;
    for (int i = 0; i < s.launches; ++i) {
        const int64_t lo = i * s.part, rows = std::min<int64_t>(s.part, p.n - lo);
        const char *from = (const char *)p.points + lo * p.ld_points * size;
        Rows16 X{(const uint16_t *)from, p.ld_points, 16, rows};
        if (s.pack) {
            X = SPLIT ? packed_rows(s.x16, rows) : Rows16{s.x16, (int64_t)s.steps * 32, 16, rows};
            if (!laid_out) AVQ_TRY(launch_pack_rows(from, p.type, rows, p.d, p.ld_points, s.steps, X, SPLIT ? s.x_inv + lo : nullptr, false, st));
        }
        float4 *stats = s.stats + (size_t)i * s.parts * 2 * p.nq;
        const float *x_inv = SPLIT ? s.x_inv + lo : nullptr, *tile_inv = SPLIT ? s.tile_inv + lo / kTileM : nullptr;
        const dim3 grid((unsigned)(s.parts * s.query_tiles));
        if (p.k > 0) {
            AVQ_TRY(set_lds_limit((const void *)prob_tile_kernel<H, SPLIT, true>, kTileLds, &with_best));
            prob_tile_kernel<H, SPLIT, true><<<grid, dim3(kTileThreads), kTileLds, st>>>(X, Q, s.steps, c2, x_inv, tile_inv, s.q_inv, s.parts, s.query_tiles, stats,
                                                                                      s.gmax + lo / 32, s.gstride);
        } else {
            AVQ_TRY(set_lds_limit((const void *)prob_tile_kernel<H, SPLIT, false>, kTileLds, &without));
            prob_tile_kernel<H, SPLIT, false><<<grid, dim3(kTileThreads), kTileLds, st>>>(X, Q, s.steps, c2, x_inv, tile_inv, s.q_inv, s.parts, s.query_tiles, stats, nullptr, 0);
        }
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

template <int PATH, class T, int NT>
static int finish_run(const ProbParams &p, const ProbScratch &s, int parts, hipStream_t st)
{
    static LdsLimitOnce once;
    AVQ_TRY(set_lds_limit((const void *)prob_finish_kernel<PATH, T, NT>, kFinishLds, &once));
    prob_finish_kernel<PATH, T, NT><<<dim3(p.nq), dim3(NT), finish_lds(p.d, p.k), st>>>(
        (const T *)p.points, p.n, p.d, p.ld_points, (const T *)p.queries, p.nq, p.ld_queries, p.scale, row_lanes(sizeof(T), p.d), s.x_inv, s.q_inv, s.odd.seen, s.stats, parts, p.ids, p.given,
        p.logp, p.lse, p.entropy, s.gmax, s.gstride, p.k, p.alt_ids, p.alt_logp);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T>
static int log_probs_typed(const ProbParams &p, hipStream_t st)
{
    const int path = prob_path(sizeof(T), p.d, p.nq);
    if (path == kByTiles) {
        ProbParams part = p;
        part.nq = queries_at_once(p.type, p.n, p.d, p.nq, p.k);
        ProbScratch s = prob_scratch(part, p.scratch);
        for (int q0 = 0; q0 < p.nq; q0 += part.nq) {
            ProbParams now = p;
            now.nq = std::min(part.nq, p.nq - q0);
            now.queries = (const T *)p.queries + q0 * p.ld_queries;
            if (p.given > 0) { now.ids = p.ids + (int64_t)q0 * p.given; now.logp = p.logp + (int64_t)q0 * p.given; }
            now.lse = p.lse + q0;
            if (p.entropy) now.entropy = p.entropy + q0;
            if (p.k > 0) { now.alt_ids = p.alt_ids + (int64_t)q0 * p.k; now.alt_logp = p.alt_logp + (int64_t)q0 * p.k; }
            s.query_tiles = (now.nq + kTileN - 1) / kTileN;
            if constexpr (sizeof(T) == 4) AVQ_TRY((tiles_run<f16_t, true>(now, s, q0 > 0, st)));
            else AVQ_TRY((tiles_run<T, false>(now, s, q0 > 0, st)));
            // a few queries: as many threads a query as there can be
            const int parts = s.launches * s.parts * 2;
            AVQ_TRY((now.nq <= 256 ? finish_run<kByTiles, T, 1024>(now, s, parts, st) : finish_run<kByTiles, T, 512>(now, s, parts, st)));
        }
        return AVQ_OK;
    }
    const ProbScratch s = prob_scratch(p, p.scratch);
    if (path == kByRow) {
        AVQ_TRY(row_sized<T>(p, s, st));
        return finish_run<kByRow, T, 1024>(p, s, s.groups, st);
    }
    const bool aligned = ((uintptr_t)p.points % 16) == 0 && (p.ld_points * sizeof(T)) % 16 == 0;
    AVQ_TRY(aligned ? (stream_sized<T, true>(p, s, st)) : (stream_sized<T, false>(p, s, st)));
    return finish_run<kByStream, T, 1024>(p, s, s.groups, st);
}

int launch_log_probs(const ProbParams &p, hipStream_t st)
{
    if (p.nq == 0) return AVQ_OK;
    if (p.type == AVQ_F32) return log_probs_typed<float>(p, st);
    return p.type == AVQ_BF16 ? log_probs_typed<bf16_t>(p, st) : log_probs_typed<f16_t>(p, st);
}

} // namespace avq
