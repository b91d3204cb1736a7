// Tiles of matrix products on the 16-bit matrix instructions (32 x 32 x 16), for operands laid out by rows_pack.hip or
// used as they are.
//
// fp32 operands (SPLIT) are two f16 values each: v = (hi + lo) / s with s a power of two that brings the largest magnitude to
// 2^14 .. 2^15, hi = f16(v s), lo = f16(v s - hi). hi hi' + hi lo' + lo hi' differs from v v' s s' by less than 1.5 * 2^-23 of it (values
// down to 2^-28 of the largest; below, by 2^-40 of the largest), which is what an fp32 product and its sum lose anyway, at a third
// of the 16-bit rate: five times the fp32 matrix instruction's. A row holds 16 hi, then their 16 lo, and so on.
//
// A workgroup of four waves forms 256 x 128 values, a wave 128 x 64 (4 x 2 matrix instructions, 128 accumulators), over steps
// of 32 of the inner dimension (SPLIT: 16, 24 matrix instructions rather than 16). A step's operands (24 KB, 64 bytes a row) come by
// copies straight to LDS, two steps ahead in a ring of three; one barrier a step. Two workgroups share a compute unit, so that
// one's epilogue runs beside the other's matrix instructions.
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

constexpr int kTileM = 256, kTileN = 128, kStepBytes = 64 /* of a row */, kTileThreads = 256;
constexpr int kStageA = kTileM * kStepBytes, kStageB = kTileN * kStepBytes, kStageBytes = kStageA + kStageB, kStages = 3;
constexpr int kTileLds = kStages * kStageBytes;

// Rows of 16-bit elements (SPLIT: of pairs of them): `rows` of them, `row` elements apart, 16-byte aligned; a step's 32 elements lie
// `step` elements after the step's before. Rows as a caller has them: step = 32. Packed ones: row = 32, so that the rows of a
// step lie side by side and copies read whole lines (a step of 64 bytes a row is half a line, and the copies of the products over
// rows, which read 512 bytes at a time, reached 1,020 TFLOP/s where those of 64 bytes reached 770).
struct Rows16 { const uint16_t *p; int64_t row, step, rows; };
constexpr int64_t kMaxRow16 = (int64_t)1 << 22; // (256 rows' places are 32-bit offsets)
constexpr int kStepElems16 = 32;

// The step that element c of a row belongs to, and its place there; SPLIT: of its hi, 16 elements before its lo.
template <bool SPLIT> __host__ __device__ inline int64_t step16(int64_t c) { return SPLIT ? c >> 4 : c >> 5; }
template <bool SPLIT> __host__ __device__ inline int in_step16(int64_t c) { return (int)(SPLIT ? c & 15 : c & 31); }
// The steps that an inner dimension of d takes.
template <bool SPLIT> __host__ __device__ inline int steps_of(int64_t d) { return (int)((d + (SPLIT ? 15 : 31)) / (SPLIT ? 16 : 32)); }

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

// Copies of operands whose rows hold the inner dimension (C = A B^T). In LDS a row's step is four 16-byte chunks, chunk c
// of row r at c ^ (r / 4 % 4): sixteen rows' reads of one chunk touch every bank once.
struct RowCopies {
    const char *pa, *pb; // the tile's first rows
    uint32_t a[4], b[2]; // this lane's places from there
    __device__ __forceinline__ void seek(const Rows16 &A, int64_t a0, const Rows16 &B, int64_t b0)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const uint32_t chunk = (uint32_t)((lane & 3) ^ ((lane >> 4) & 3)) * 16;
        const int last_a = (int)min(A.rows - 1 - a0, (int64_t)kTileM), last_b = (int)min(B.rows - 1 - b0, (int64_t)kTileN);
        pa = (const char *)(A.p + a0 * A.row);
        pb = (const char *)(B.p + b0 * B.row);
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = (uint32_t)min((wave * 4 + j) * 16 + (lane >> 2), last_a) * (uint32_t)(A.row * 2) + chunk;
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = (uint32_t)min((wave * 2 + j) * 16 + (lane >> 2), last_b) * (uint32_t)(B.row * 2) + chunk;
    }
    __device__ __forceinline__ void issue(const Rows16 &A, const Rows16 &B, int step, uint32_t stage) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const char *fa = pa + step * A.step * 2, *fb = pb + step * B.step * 2;
#pragma unroll
        for (int j = 0; j < 4; ++j) lds_copy16_from(fa, a[j], stage + (wave * 4 + j) * 1024);
#pragma unroll
        for (int j = 0; j < 2; ++j) lds_copy16_from(fb, b[j], stage + kStageA + (wave * 2 + j) * 1024);
    }
    // operands of 16 of the inner dimension: the step's first or second half (SPLIT: its hi or lo)
    static __device__ __forceinline__ void read(const char *stage, int half, Quad (&a)[4], Quad (&b)[2])
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int at = (lane & 31) * 64 + ((((lane >> 5) + half * 2) ^ ((lane >> 2) & 3)) * 16);
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = *(const Quad *)(stage + kStageA + ((wave & 1) * 64 + j * 32) * 64 + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *(const Quad *)(stage + ((wave >> 1) * 128 + i * 32) * 64 + at);
    }
};

// Copies of operands whose rows are the inner dimension (C = A^T B): 32 rows (SPLIT: 16 of pairs) of 256 columns of A and 128 of B a
// step. The reads transpose 4 x 16 elements for 16 lanes: 32 lanes read two pieces of 32 bytes, 32 (SPLIT: 64) apart, of four rows. So
// that these lie in different banks, a row's 16-byte chunk c lies at c ^ turn(row % 4).
template <bool SPLIT> struct ColumnCopies {
    static constexpr int kRows = SPLIT ? 16 : 32, kRowA = kStageA / kRows, kRowB = kStageB / kRows; // of a step; bytes of a row in LDS
    static constexpr int kChunksA = kRowA / 16, kChunksB = kRowB / 16;
    static __device__ __forceinline__ int turn(int r) { return SPLIT ? (r & 1) * 2 + (r >> 1) * 8 : r * 4; }
    const char *pa, *pb; // the tile's first columns
    uint32_t a[4], b[2]; // this lane's columns from there
    int64_t row;         // of the first step
    __device__ __forceinline__ void seek(const Rows16 &A, int64_t a0, int64_t a_columns, const Rows16 &B, int64_t b0)
    {
        // (columns of A past its last come from its last: nothing uses their products; B is as wide as its tiles)
        const int lane = threadIdx.x & 63;
        const int last = (int)min((step16<SPLIT>(a_columns) - step16<SPLIT>(a0)) * 4 - 1, (int64_t)kChunksA);
        pa = (const char *)(A.p + step16<SPLIT>(a0) * A.step);
        pb = (const char *)(B.p + step16<SPLIT>(b0) * B.step);
        auto at = [](int chunk, const Rows16 &r) { return (uint32_t)(chunk >> 2) * (uint32_t)(r.step * 2) + (uint32_t)(chunk & 3) * 16; };
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = at(min((lane % kChunksA) ^ turn((j * (64 / kChunksA) + lane / kChunksA + (SPLIT ? (threadIdx.x >> 6) * 4 : 0)) & 3), last), A);
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = at((lane % kChunksB) ^ turn((j * (64 / kChunksB) + lane / kChunksB) & 3), B);
    }
    __device__ __forceinline__ void issue(const Rows16 &A, const Rows16 &B, int step, uint32_t stage) const
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // (a step's rows past an operand's last, of which a whole step may consist, are its last row)
        const int64_t first = row + (int64_t)step * kRows, first_a = min(first, A.rows - 1), first_b = min(first, B.rows - 1);
        const char *fa = pa + first_a * A.row * 2, *fb = pb + first_b * B.row * 2;
        const int last_a = (int)min(A.rows - 1 - first_a, (int64_t)kRows), last_b = (int)min(B.rows - 1 - first_b, (int64_t)kRows);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            lds_copy16_from(fa, (uint32_t)min((wave * 4 + j) * (64 / kChunksA) + lane / kChunksA, last_a) * (uint32_t)(A.row * 2) + a[j], stage + (wave * 4 + j) * 1024);
#pragma unroll
        for (int j = 0; j < 2; ++j)
            lds_copy16_from(fb, (uint32_t)min((wave * 2 + j) * (64 / kChunksB) + lane / kChunksB, last_b) * (uint32_t)(B.row * 2) + b[j], stage + kStageA + (wave * 2 + j) * 1024);
    }
    static __device__ __forceinline__ Quad read_turned(const char *p, int row_bytes)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * row_bytes));
        Quad q;
        __builtin_memcpy(&q.w[0], &lo, 8);
        __builtin_memcpy(&q.w[2], &hi, 8);
        return q;
    }
    static __device__ __forceinline__ void read(const char *stage, int half, Quad (&a)[4], Quad (&b)[2])
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int i16 = lane & 15, g = lane >> 4, r = i16 >> 2; // r: row of the four
        const int row_at = (SPLIT ? 0 : half * 16) + 8 * (g >> 1) + r;
        // the chunk of columns 32 m + 16 (g & 1) + 4 (i16 & 3) onwards, and the place in it
        auto at = [&](int m) { return ((SPLIT ? m * 8 + (g & 1) * 4 + half * 2 + ((i16 & 3) >> 1) : m * 4 + (g & 1) * 2 + ((i16 & 3) >> 1)) ^ turn(r)) * 16 + (i16 & 1) * 8; };
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = read_turned(stage + kStageA + row_at * kRowB + at((wave & 1) * 2 + j), kRowB);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = read_turned(stage + row_at * kRowA + at((wave >> 1) * 4 + i), kRowA);
    }
};

template <class H> __device__ __forceinline__ void multiply(const Quad (&a)[4], const Quad (&b)[2], f32x16 (&acc)[4][2])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = mma32(a[i], b[j], acc[i][j], H{});
}

// `tiles` tiles of `steps` steps one after the other, the copies running ahead over their borders. seek(i, copies): turns to tile i;
// epilogue(i, acc): takes its values. MEMORY: the epilogue loads or stores.
template <class H, bool SPLIT, bool MEMORY, class Copies, class Seek, class Epilogue>
__device__ __forceinline__ void run_tiles(const Rows16 &A, const Rows16 &B, int steps, int tiles, char *lds, Seek seek, Epilogue epilogue)
{
    if (tiles <= 0) return;
    Copies copies;
    int tile = 0, step = 0, stage = 0; // of the next copies
    bool more = true;
    seek(0, copies);
    const uint32_t lds_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds);
    auto issue = [&]() __attribute__((always_inline)) {
        copies.issue(A, B, step, lds_at + stage * kStageBytes);
        stage = stage + 1 == kStages ? 0 : stage + 1;
        if (++step == steps) {
            step = 0;
            if (++tile == tiles) more = false;
            else seek(tile, copies);
        }
    };
    issue();
    if (more) issue();
    int at = 0;
    for (int t = 0; t < tiles; ++t) {
        f32x16 acc[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
        for (int s = 0; s < steps; ++s) {
            // the last step of all has no younger copies; after an epilogue with memory operations all are waited for
            if ((t + 1 == tiles && s + 1 == steps) || (MEMORY && s == 0)) step_barrier<0>();
            else step_barrier<kCopies>();
            if (more) issue();
            const char *here = lds + at * kStageBytes;
            at = at + 1 == kStages ? 0 : at + 1;
            Quad a[2][4], b[2][2];
            Copies::read(here, 0, a[0], b[0]);
            Copies::read(here, 1, a[1], b[1]);
            multiply<H>(a[0], b[0], acc);
            if (SPLIT) {
                multiply<H>(a[0], b[1], acc);
                multiply<H>(a[1], b[0], acc);
            } else {
                multiply<H>(a[1], b[1], acc);
            }
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
// Packed rows: out[step][row of `total`][32], `steps` steps, zeros past a row's end. fp32: pairs, scaled by range_scale(*largest), or,
// largest == NULL, each row by its own, whose inverse goes to inv[row]. negate: with the other sign.
int launch_pack_rows(const void *x, int type, int64_t rows, int d, int64_t ld, int steps, int64_t total, uint16_t *out, const uint32_t *largest, float *inv, bool negate,
                     hipStream_t st);
// The transpose packed: row c < d of d holds x[t][c], zeros past the last t.
int launch_pack_transposed(const void *x, int type, int64_t rows, int d, int64_t ld, int steps, uint16_t *out, const uint32_t *largest, hipStream_t st);

} // namespace avq
