// Tiles of matrix products on the 16-bit matrix instructions (32 x 32 x 16), for operands laid out by rows_pack.hip or
// used as they are.
//
// fp32 operands (SPLIT) are two f16 values each: v = (hi + lo) / s with s a power of two that brings the largest magnitude (of a row, or
// of all rows) to 2^14 .. 2^15, hi = f16(v s), lo = f16(v s - hi). hi hi' + hi lo' + lo hi' differs from v v' s s' by at most 2^-21 of it
// (lo lo', and the rounding of either lo) where v and v' are 2^-16 of their largest or more; below, lo is a multiple of 2^-24, and v has an
// error of 2^-39 of the largest. Sums of fp32 products lose as much, at a third of the 16-bit rate: five times the fp32
// matrix instruction's. A row holds 16 hi, then their 16 lo, and so on.
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

// Rows of 16-bit elements (SPLIT: of pairs of them): `rows` of them, in blocks of 16 elements (32 bytes), 16-byte aligned: block b of
// row r at p + b block + r row. A step is two blocks: 32 elements, or (SPLIT) the hi of 16 and their lo. Rows as a caller has them:
// block = 16. Packed ones: row = 16, so that the rows of a block lie side by side, and copies read, and stores write, whole lines;
// SPLIT ones always, others where they are not a caller's rows (or a copy of them, padded).
struct Rows16 { const uint16_t *p; int64_t row, block, rows; };
constexpr int64_t kMaxRow16 = (int64_t)1 << 22; // (256 rows' places are 32-bit offsets)
// Blocks lie apart by a little more than their rows: by a power of two, all of a row's blocks would be on few memory channels.
constexpr int kBlockGap = 72; // rows
inline Rows16 packed_rows(const uint16_t *p, int64_t rows) { return Rows16{p, 16, (rows + kBlockGap) * 16, rows}; }
inline size_t packed_bytes(int64_t rows, int steps) { return (size_t)(rows + kBlockGap) * steps * kStepBytes; }

// The block that element c of a row belongs to; SPLIT: of its hi, the lo's is the next.
template <bool SPLIT> __host__ __device__ inline int64_t block16(int64_t c) { return SPLIT ? (c >> 4) * 2 : c >> 4; }
// The steps that an inner dimension of d takes.
template <bool SPLIT> __host__ __device__ inline int steps_of(int64_t d) { return (int)((d + (SPLIT ? 15 : 31)) / (SPLIT ? 16 : 32)); }
// G's and the transposed queries' order of 16 queries: a lane of the product that makes G has queries 8 b + 4 h + e of a block, and
// stores them side by side, at 8 h + 4 b + e. (Its own inverse.)
__host__ __device__ inline int turned16(int i) { return ((i >> 2) & 1) * 8 + (i >> 3 & 1) * 4 + (i & 3); }

__device__ __forceinline__ void split_f16(float v, uint16_t *hi, uint16_t *lo)
{
    const _Float16 h = (_Float16)v;
    *hi = __builtin_bit_cast(uint16_t, h);
    *lo = __builtin_bit_cast(uint16_t, (_Float16)(v - (float)h));
}

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

// Copies of operands whose rows hold the inner dimension (C = A B^T). Lanes side by side read what lies side by side. In LDS a step of
// a caller's rows is 64 bytes a row, of which the 16-byte chunk c lies at c ^ (row / 4 % 4); of packed rows two blocks of 32 bytes a row,
// chunk c of a block at c ^ (row / 8 % 2). Either way sixteen rows' reads of one chunk touch every bank once.
template <bool PACKED, int ROWS> struct RowOperand {
    static constexpr int kEach = ROWS * kStepBytes / 1024 / 4; // copies of a wave
    const char *p;        // the tile's first row
    uint32_t at[kEach];   // this lane's places from there
    __device__ __forceinline__ void seek(const Rows16 &R, int64_t r0)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int last = (int)min(R.rows - 1 - r0, (int64_t)ROWS);
        p = (const char *)(R.p + r0 * R.row);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int i = wave * kEach + j;
            const int row = PACKED ? i % (ROWS / 32) * 32 + (lane >> 1) : i * 16 + (lane >> 2);
            const int chunk = PACKED ? i / (ROWS / 32) * 2 + ((lane & 1) ^ ((lane >> 4) & 1)) : (lane & 3) ^ ((lane >> 4) & 3);
            at[j] = (uint32_t)min(row, last) * (uint32_t)(R.row * 2) + (uint32_t)(chunk >> 1) * (uint32_t)(R.block * 2) + (chunk & 1) * 16;
        }
    }
    __device__ __forceinline__ void issue(const Rows16 &R, int step, uint32_t lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const char *from = p + step * R.block * 4;
#pragma unroll
        for (int j = 0; j < kEach; ++j) lds_copy16_from(from, at[j], lds + (wave * kEach + j) * 1024);
    }
    // row0 + (lane & 31) of 32 rows, the step's first or second half (SPLIT: hi or lo)
    static __device__ __forceinline__ Quad read(const char *lds, int row0, int half)
    {
        const int lane = threadIdx.x & 63;
        if (PACKED) return *(const Quad *)(lds + half * (ROWS * 32) + (row0 + (lane & 31)) * 32 + ((lane >> 5) ^ ((lane >> 3) & 1)) * 16);
        return *(const Quad *)(lds + (row0 + (lane & 31)) * 64 + ((((lane >> 5) + half * 2) ^ ((lane >> 2) & 3)) * 16));
    }
};

template <bool PACKED_A, bool PACKED_B> struct RowCopies {
    typedef RowOperand<PACKED_A, kTileM> OfA;
    typedef RowOperand<PACKED_B, kTileN> OfB;
    OfA a;
    OfB b;
    __device__ __forceinline__ void seek(const Rows16 &A, int64_t a0, const Rows16 &B, int64_t b0) { a.seek(A, a0); b.seek(B, b0); }
    __device__ __forceinline__ void issue(const Rows16 &A, const Rows16 &B, int step, uint32_t stage) const { a.issue(A, step, stage); b.issue(B, step, stage + kStageA); }
    // operands of 16 of the inner dimension
    static __device__ __forceinline__ void read(const char *stage, int half, Quad (&qa)[4], Quad (&qb)[2])
    {
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int j = 0; j < 2; ++j) qb[j] = OfB::read(stage + kStageA, (wave & 1) * 64 + j * 32, half);
#pragma unroll
        for (int i = 0; i < 4; ++i) qa[i] = OfA::read(stage, (wave >> 1) * 128 + i * 32, half);
    }
};

// Copies of operands whose rows are the inner dimension (C = A^T B): 32 rows (SPLIT: 16 of pairs) of 256 columns of A and 128 of B a
// step. Reads transpose 4 x 16 elements for 16 lanes: 32 lanes read 32 bytes of four rows in two blocks of columns. Packed rows lie in
// LDS as they do in memory, [block][row][32 bytes], rows of every other block of columns turned by four, so that the two blocks' reads
// touch different banks; a caller's rows (B where not SPLIT) [row][256 bytes], chunk c at c ^ (4 (row % 4)), so that the four rows' do.
template <bool SPLIT> struct ColumnCopies {
    static constexpr int kRows = SPLIT ? 16 : 32, kBlock = kRows * 32; // of a step; bytes of a block in LDS
    const char *pa, *pb; // the tile's first columns
    uint32_t a[4], b[2]; // this lane's columns from there
    int64_t row;         // of the first step
    __device__ __forceinline__ void seek(const Rows16 &A, int64_t a0, int64_t a_columns, const Rows16 &B, int64_t b0)
    {
        // (columns of A past its last come from its last: nothing uses their products; B is as wide as its tiles)
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int last = (int)min(block16<SPLIT>(a_columns) - block16<SPLIT>(a0) - 1, (int64_t)kStageA);
        pa = (const char *)(A.p + block16<SPLIT>(a0) * A.block);
        pb = (const char *)(B.p + block16<SPLIT>(b0) * B.block);
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = (uint32_t)min(SPLIT ? (wave * 4 + j) * 2 + (lane >> 5) : wave * 4 + j, last) * (uint32_t)(A.block * 2) + (lane & 1) * 16;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (SPLIT) b[j] = (uint32_t)((wave * 2 + j) * 2 + (lane >> 5)) * (uint32_t)(B.block * 2) + (lane & 1) * 16;
            else b[j] = (uint32_t)((lane & 15) ^ ((lane >> 4) * 4)) * 16; // (B.block == 16)
        }
    }
    // the row that a lane of the j-th copy has, of packed rows
    static __device__ __forceinline__ int packed_row(int lane, int j) { return ((lane >> 1) & (kRows - 1)) ^ ((j & 1) * 4); }
    __device__ __forceinline__ void issue(const Rows16 &A, const Rows16 &B, int step, uint32_t stage) const
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // (a step's rows past an operand's last, of which a whole step may consist, are its last row)
        const int64_t first = row + (int64_t)step * kRows, first_a = min(first, A.rows - 1), first_b = min(first, B.rows - 1);
        const char *fa = pa + first_a * A.row * 2, *fb = pb + first_b * B.row * 2;
        const int last_a = (int)min(A.rows - 1 - first_a, (int64_t)kRows), last_b = (int)min(B.rows - 1 - first_b, (int64_t)kRows);
#pragma unroll
        for (int j = 0; j < 4; ++j) lds_copy16_from(fa, (uint32_t)min(packed_row(lane, j), last_a) * (uint32_t)(A.row * 2) + a[j], stage + (wave * 4 + j) * 1024);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = SPLIT ? packed_row(lane, j) : (wave * 2 + j) * 4 + (lane >> 4);
            lds_copy16_from(fb, (uint32_t)min(r, last_b) * (uint32_t)(B.row * 2) + b[j], stage + kStageA + (wave * 2 + j) * 1024);
        }
    }
    // four rows at p and the four after them, at q, of which a lane gets its column
    static __device__ __forceinline__ Quad read_turned(const char *p, const char *q)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)q);
        Quad v;
        __builtin_memcpy(&v.w[0], &lo, 8);
        __builtin_memcpy(&v.w[2], &hi, 8);
        return v;
    }
    static __device__ __forceinline__ void read(const char *stage, int half, Quad (&qa)[4], Quad (&qb)[2])
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int i16 = lane & 15, g = lane >> 4, r = i16 >> 2; // r: row of the four
        const int first = (SPLIT ? 0 : half * 16) + 8 * (g >> 1);
        // of packed rows: columns 32 m + 16 (g & 1) + 4 (i16 & 3) onwards
        auto packed = [&](const char *lds, int m) __attribute__((always_inline)) {
            const int block = SPLIT ? (m * 2 + (g & 1)) * 2 + half : m * 2 + (g & 1);
            const char *rows = lds + block * kBlock + first * 32 + (i16 & 3) * 8;
            return read_turned(rows + (r + 4 * (g & 1)) * 32, rows + (r + 4 - 4 * (g & 1)) * 32);
        };
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (SPLIT) {
                qb[j] = packed(stage + kStageA, (wave & 1) * 2 + j);
            } else {
                const char *p = stage + kStageA + (first + r) * 256 + ((((wave & 1) * 2 + j) ^ r) * 64) + (2 * (g & 1) + ((i16 & 3) >> 1)) * 16 + (i16 & 1) * 8;
                qb[j] = read_turned(p, p + 4 * 256);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) qa[i] = packed(stage, (wave >> 1) * 4 + i);
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
// Ranges, as bits of non-negative floats (0, for the least infinity: nothing yet): of the rows' inverses, of the largest magnitudes that
// queries have over their factor in G; the largest bound of a query's G; and how many rows are odd.
struct Ranges { uint32_t inverse, least_inverse, weighted, least_weighted, upstream, odd; };

// the power of two that brings a largest magnitude to 2^14 .. 2^15 (1 where there is none)
__device__ __forceinline__ float range_scale(uint32_t largest_bits)
{
    if (largest_bits == 0) return 1.0f;
    int e = (int)(largest_bits >> 23) - 127;
    e = 14 - e;
    e = e > 97 ? 97 : e < -113 ? -113 : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Where rows have scales s of their own, what is kept is the inverse: kRowUnit / s for the table's rows, 1 / (kRowUnit s) for queries.
// A sum of products of two rows times the table's inverse is then the product of the row with a query of magnitudes up to 1/2, which
// stays in range for rows of any size; times the query's inverse it is the product itself. The kTileM rows of a tile have one scale
// where their largest magnitudes lie within kTileSpread of one another (rows of nothing but zeros aside), so that a tile of ordinary rows
// needs no factor a row: 8 % of a pass of 2,048 queries over 1,183,514 x 100.
constexpr float kRowUnit = 0x1p-16f, kTileSpread = 0x1p8f;
__device__ __forceinline__ float scale_of_inverse(float inv) { return kRowUnit / inv; }

// Odd rows hold an infinity or NaN. A pair has neither, so they are laid out as zeros with an infinite inverse, and their products taken as
// -infinity, which is what a mask means; queries for which one of them is something else (an infinity times 0 or of the other sign, NaN)
// are marked, and have no sum that is a number. A query that is not finite itself has zeros, and NaN for an inverse.
struct OddRows { uint32_t *count, *rows, *seen; }; // how many, which (in any order), [queries] whether marked

int launch_clear_ranges(Ranges *to, hipStream_t st);
// The same where a product adds rows up, so that they need one scale: inv[row] is the table's where its rows' largest magnitudes lie within
// kTableSpread of one another (pairs then hold the least of them to 2^-24), and the row's own where they do not; odd rows are counted.
constexpr float kTableSpread = 0x1p16f;
__device__ __forceinline__ bool rows_apart(const Ranges *ranges) { return __uint_as_float(ranges->inverse) > kTableSpread * __uint_as_float(ranges->least_inverse); }
int launch_common_inverses(const float *x, int64_t rows, int d, int64_t ld, float *inv, Ranges *ranges, hipStream_t st);
// inv[row] = kRowUnit / s of each row, and tile_inv[tile] that of the tile's rows where they have one, else 0
int launch_row_inverses(const float *x, int64_t rows, int d, int64_t ld, float *inv, float *tile_inv, const OddRows &odd, hipStream_t st);
// marks the queries (negate: with the other sign) whose product with an odd row is not -infinity
int launch_odd_rows(const float *x, int d, int64_t ld, const float *q, int nq, int64_t ld_q, bool negate, const OddRows &odd, hipStream_t st);
// Rows laid out as `to` says (to.p: where), `steps` steps of them, zeros past a row's end. fp32: pairs, by scales of which inv[row] is the
// inverse. negate: with the other sign.
int launch_pack_rows(const void *x, int type, int64_t rows, int d, int64_t ld, int steps, const Rows16 &to, const float *inv, bool negate, hipStream_t st);
// fp32 queries: pairs, each row by its own scale, whose inverse goes to inv[row]. Also begins what `odd` has: no rows, no marks.
int launch_pack_queries(const float *q, int64_t rows, int d, int64_t ld, int steps, const Rows16 &to, float *inv, const OddRows &odd, bool negate, hipStream_t st);
// The transpose packed: row c < d of d holds x[t][c] factor[t] (factor == NULL: x[t][c]), 16 t in the order of turned16, zeros past the
// last t and where the factor is 0.
int launch_pack_transposed(const void *x, int type, int64_t rows, int d, int64_t ld, int steps, const Rows16 &to, const float *factor, hipStream_t st);

} // namespace avq
