// Tiles of matrix products on the 16-bit matrix instructions (32 x 32 x 16), for operands laid out by rows_pack.hip or
// used as they are.
//
// fp32 operands are two f16 planes: v = (hi + lo) / s with s a power of two that brings the largest magnitude to 2^14 .. 2^15,
// hi = f16(v s), lo = f16(v s - hi). hi hi' + hi lo' + lo hi' differs from v v' s s' by less than 1.5 * 2^-23 of it (values
// down to 2^-28 of the largest; below, by 2^-40 of the largest), which is what an fp32 product and its sum lose anyway, at a third
// of the 16-bit rate: five times the fp32 matrix instruction's.
//
// A workgroup of four waves forms 256 x 128 values, a wave 128 x 64 (4 x 2 matrix instructions, 128 accumulators), over steps
// of 32 of the inner dimension. A step's operands (24 KB) come by copies straight to LDS, two steps ahead in a ring of three; one
// barrier a step. Two workgroups share a compute unit, so that one's epilogue runs beside the other's matrix instructions.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "avq_internal.h"
#include "lds_copy.h"
#include "row_types.h"

namespace avq {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16v8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16v8 __attribute__((ext_vector_type(8)));
struct alignas(16) Quad { uint32_t w[4]; };

constexpr int kTileM = 256, kTileN = 128, kTileK = 32, kTileThreads = 256;
constexpr int kStageA = kTileM * kTileK * 2, kStageB = kTileN * kTileK * 2, kStageBytes = kStageA + kStageB, kStages = 3;
constexpr int kTileLds = kStages * kStageBytes;

// Rows of 16-bit elements: `rows` of them, ld elements apart, 16-byte aligned; plane: elements from the hi to the lo plane.
struct Rows16 { const uint16_t *p; int64_t ld, plane, rows; };

__device__ __forceinline__ f32x16 mma32(const Quad &a, const Quad &b, f32x16 c, bf16_t)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16v8, a), __builtin_bit_cast(bf16v8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(const Quad &a, const Quad &b, f32x16 c, f16_t)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16v8, a), __builtin_bit_cast(f16v8, b), c, 0, 0, 0);
}

// Where a value of acc[i][j][r] lies in the tile: row (of A) and column (of B).
__device__ __forceinline__ int acc_row(int i, int r) { return ((threadIdx.x >> 6) >> 1) * 128 + i * 32 + 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }
__device__ __forceinline__ int acc_col(int j) { return ((threadIdx.x >> 6) & 1) * 64 + j * 32 + (threadIdx.x & 31); }

// Waits for a step's copies (all but the `newer` youngest of this wave's) and for every wave to be done with the step before.
template <int NEWER> __device__ __forceinline__ void step_barrier()
{
    if (NEWER == 0) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(6) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
constexpr int kCopies = 6; // of a wave a step (the 6 above)

// The products that make up one: with fp32 operands hi hi', hi lo', lo hi', else the one there is.
__device__ __forceinline__ int plane_of_a(int term) { return term == 2; }
__device__ __forceinline__ int plane_of_b(int term) { return term == 1; }

// Copies of operands whose rows hold the inner dimension (C = A B^T). In LDS a row's 32 elements are four 16-byte chunks, chunk c
// of row r at c ^ (r / 4 % 4): sixteen rows' reads of one chunk touch every bank once.
struct RowCopies {
    const char *a[4], *b[2];
    __device__ __forceinline__ void seek(const Rows16 &A, int64_t a0, const Rows16 &B, int64_t b0)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int chunk = (lane & 3) ^ ((lane >> 4) & 3);
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = (const char *)(A.p + min(a0 + (wave * 4 + j) * 16 + (lane >> 2), A.rows - 1) * A.ld) + chunk * 16;
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = (const char *)(B.p + min(b0 + (wave * 2 + j) * 16 + (lane >> 2), B.rows - 1) * B.ld) + chunk * 16;
    }
    __device__ __forceinline__ void issue(const Rows16 &A, const Rows16 &B, int term, int step, char *stage) const
    {
        const int wave = threadIdx.x >> 6;
        const int64_t oa = (plane_of_a(term) ? A.plane * 2 : 0) + (int64_t)step * (kTileK * 2), ob = (plane_of_b(term) ? B.plane * 2 : 0) + (int64_t)step * (kTileK * 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) lds_copy16(a[j] + oa, stage + (wave * 4 + j) * 1024);
#pragma unroll
        for (int j = 0; j < 2; ++j) lds_copy16(b[j] + ob, stage + kStageA + (wave * 2 + j) * 1024);
    }
    // the products of half a step (16 of the inner dimension)
    template <class H> static __device__ __forceinline__ void multiply(const char *stage, int half, f32x16 (&acc)[4][2])
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int at = (lane & 31) * 64 + ((((lane >> 5) + half * 2) ^ ((lane >> 2) & 3)) * 16);
        Quad a[4], b[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = *(const Quad *)(stage + kStageA + ((wave & 1) * 64 + j * 32) * 64 + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *(const Quad *)(stage + ((wave >> 1) * 128 + i * 32) * 64 + at);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = mma32(a[i], b[j], acc[i][j], H{});
    }
};

// Copies of operands whose rows are the inner dimension (C = A^T B): 32 rows of 256 columns of A and 128 of B a step. A row's
// 16-byte chunk c lies at c ^ (4 (r % 4)); the reads transpose 4 x 16 elements for 16 lanes, from four rows at once, which so lie in
// different banks.
struct ColumnCopies {
    const char *a[4], *b[2];
    int64_t row; // of the first step
    __device__ __forceinline__ void seek(const Rows16 &A, int64_t a0, int64_t a_columns, const Rows16 &B, int64_t b0)
    {
        // (columns of A past its last come from its last: nothing uses their products; B is as wide as its tiles)
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = (j * 2 + (lane >> 5)) & 3;
            a[j] = (const char *)(A.p + min(a0 + ((lane & 31) ^ (r * 4)) * 8, a_columns - 8));
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = (const char *)(B.p + b0 + ((lane & 15) ^ ((lane >> 4) * 4)) * 8);
    }
    __device__ __forceinline__ void issue(const Rows16 &A, const Rows16 &B, int term, int step, char *stage) const
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int64_t oa = plane_of_a(term) ? A.plane * 2 : 0, ob = plane_of_b(term) ? B.plane * 2 : 0;
        const int64_t first = row + (int64_t)step * kTileK;
#pragma unroll
        for (int j = 0; j < 4; ++j) lds_copy16(a[j] + oa + min(first + (wave * 4 + j) * 2 + (lane >> 5), A.rows - 1) * A.ld * 2, stage + (wave * 4 + j) * 1024);
#pragma unroll
        for (int j = 0; j < 2; ++j) lds_copy16(b[j] + ob + min(first + (wave * 2 + j) * 4 + (lane >> 4), B.rows - 1) * B.ld * 2, stage + kStageA + (wave * 2 + j) * 1024);
    }
    static __device__ __forceinline__ Quad read(const char *p, int row_bytes)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * row_bytes));
        Quad q;
        __builtin_memcpy(&q.w[0], &lo, 8);
        __builtin_memcpy(&q.w[2], &hi, 8);
        return q;
    }
    template <class H> static __device__ __forceinline__ void multiply(const char *stage, int half, f32x16 (&acc)[4][2])
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int i16 = lane & 15, g = lane >> 4, r = i16 >> 2; // row of the four, which the chunk's place goes by
        const int row_at = half * 16 + 8 * (g >> 1) + r, in_chunk = (2 * (g & 1) + ((i16 & 3) >> 1)) * 16 + (i16 & 1) * 8;
        Quad a[4], b[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = read(stage + kStageA + row_at * (kTileN * 2) + ((((wave & 1) * 2 + j) ^ r) * 64) + in_chunk, kTileN * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = read(stage + row_at * (kTileM * 2) + ((((wave >> 1) * 4 + i) ^ r) * 64) + in_chunk, kTileM * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = mma32(a[i], b[j], acc[i][j], H{});
    }
};

// `tiles` tiles one after the other, the copies running ahead over their borders. halves: 16s of the inner dimension.
// seek(i, copies): turns to tile i; epilogue(i, acc): takes its values. MEMORY: the epilogue loads or stores.
template <class H, int TERMS, bool MEMORY, class Copies, class Seek, class Epilogue>
__device__ __forceinline__ void run_tiles(const Rows16 &A, const Rows16 &B, int halves, int tiles, char *lds, Seek seek, Epilogue epilogue)
{
    if (tiles <= 0) return;
    const int steps = (halves + 1) / 2;
    Copies copies;
    int tile = 0, term = 0, step = 0, stage = 0; // of the next copies
    bool more = true;
    seek(0, copies);
    auto issue = [&]() {
        copies.issue(A, B, term, step, lds + stage * kStageBytes);
        stage = stage + 1 == kStages ? 0 : stage + 1;
        if (++step == steps) {
            step = 0;
            if (TERMS == 1 || ++term == TERMS) {
                term = 0;
                if (++tile == tiles) more = false;
                else seek(tile, copies);
            }
        }
    };
    issue();
    if (more) issue();
    const int total_steps = steps * TERMS;
    int at = 0;
    for (int t = 0; t < tiles; ++t) {
        f32x16 acc[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
        int s_in_term = 0;
        for (int s = 0; s < total_steps; ++s) {
            // the last step of all has no younger copies; after an epilogue with memory operations all are waited for
            const bool last = t + 1 == tiles && s + 1 == total_steps;
            if (last || (MEMORY && s == 0)) step_barrier<0>();
            else step_barrier<kCopies>();
            if (more) issue();
            const char *here = lds + at * kStageBytes;
            at = at + 1 == kStages ? 0 : at + 1;
            Copies::template multiply<H>(here, 0, acc);
            if (2 * s_in_term + 1 < halves) Copies::template multiply<H>(here, 1, acc);
            if (++s_in_term == steps) s_in_term = 0;
        }
        epilogue(t, acc);
    }
}

// Workgroups of one launch, and which of them share a part of the rows: those with the same part and all `others` tiles of the
// other operand lie on one XCD (workgroups go round the eight), so that the part's rows are read into one L2. parts: a multiple of 8.
struct Place { int part, other; };
__device__ __forceinline__ Place place_of(int block, int others)
{
    const int xcd = block & 7, local = block >> 3;
    return Place{(local / others) * 8 + xcd, local % others};
}
inline int parts_for(int64_t tiles, int others, int most_groups)
{
    const int64_t want = std::max<int64_t>(8, (int64_t)most_groups / others / 8 * 8);
    return (int)std::min<int64_t>(want, (tiles + 7) / 8 * 8);
}
// the tiles of part p: [first, first + count)
__host__ __device__ inline void part_tiles(int64_t tiles, int parts, int p, int64_t *first, int *count)
{
    const int64_t lo = tiles * p / parts, hi = tiles * (p + 1) / parts;
    *first = lo;
    *count = (int)(hi - lo);
}

// ---- rows_pack.hip -------------------------------------------------------------------------
// Largest finite magnitudes, as bits of non-negative floats (0: nothing yet).
struct Largest { uint32_t points, queries, upstream, pad; };

// the power of two that brings a largest magnitude to 2^14 .. 2^15 (1 where there is none)
__device__ __forceinline__ float range_scale(uint32_t largest_bits)
{
    if (largest_bits == 0) return 1.0f;
    int e = (int)(largest_bits >> 23) - 127;
    e = 14 - e;
    e = e > 100 ? 100 : e < -113 ? -113 : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

int launch_clear_largest(Largest *to, hipStream_t st);
// max over finite elements into *to
int launch_largest(const float *x, int64_t rows, int d, int64_t ld, uint32_t *to, hipStream_t st);
// Rows as 16-bit elements padded with zeros to `width` (a multiple of 8) elements, rows_out >= rows of them (zeros past the last).
// fp32: hi and lo plane, scaled by range_scale(*largest), or, largest == NULL, each row by its own, whose inverse goes to inv[row].
// negate: with the other sign (16-bit types, and rows with scales of their own).
int launch_pack_rows(const void *x, int type, int64_t rows, int d, int64_t ld, int64_t rows_out, int width, uint16_t *out, int64_t plane, const uint32_t *largest, float *inv,
                     bool negate, hipStream_t st);
// The transpose: out[c][t] = x[t][c] for c < columns_out (zeros past d), t < width (zeros past rows).
int launch_pack_transposed(const void *x, int type, int64_t rows, int d, int64_t ld, int columns_out, int width, uint16_t *out, int64_t plane, const uint32_t *largest,
                           hipStream_t st);

} // namespace avq
