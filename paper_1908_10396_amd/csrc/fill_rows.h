// Clearing the rows of a table by workgroups that a launch has beyond its own: launches of mostly latency leave nearly all of the memory's
// time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "row_types.h"

namespace avq {

// Rows [lo, hi) of the table to be cleared by the workgroups of a launch beyond its own ones (ld, row_bytes: in bytes).
struct FillJob { char *out; int64_t lo, hi, ld, row_bytes; };

// bytes [from, to) of an address, multiples of two bytes, by the threads t of n
__device__ __forceinline__ void clear_bytes(char *from, char *to, int64_t t, int64_t n)
{
    char *head = min(to, (char *)(((uintptr_t)from + 15) & ~(uintptr_t)15)), *tail = max(head, (char *)((uintptr_t)to & ~(uintptr_t)15));
    typedef Pack<uint32_t, 4> Word;
    const int64_t words = (tail - head) / 16;
    int64_t i = t;
    for (; i + 3 * n < words; i += 4 * n)
#pragma unroll
        for (int u = 0; u < 4; ++u) *(Word *)(head + (i + u * n) * 16) = Word{};
    for (; i < words; i += n) *(Word *)(head + i * 16) = Word{};
    if (t < 8 && from + 2 * t < head) *(uint16_t *)(from + 2 * t) = 0;
    if (t < 8 && tail + 2 * t < to) *(uint16_t *)(tail + 2 * t) = 0;
}

// Dense rows are one long row, a piece of it a workgroup: many short workgroups, four stores a thread, write 5.8 to 6.1 TB/s, 2,048
// that stride over all of it 4.5 to 4.7 (0.42 to 1.37 GB).
constexpr int kFillPiece = 16 << 10, kFillGroups = 2048;

inline int fill_groups(const FillJob &f)
{
    const int64_t bytes = (f.hi - f.lo) * f.ld;
    if (bytes <= 0) return 0;
    return (int)std::min<int64_t>(f.ld == f.row_bytes ? (bytes + kFillPiece - 1) / kFillPiece : kFillGroups, 1 << 20);
}

__device__ __forceinline__ void fill_rows(const FillJob &f, int group, int groups)
{
    if (f.ld == f.row_bytes) {
        char *end = f.out + f.hi * f.ld;
        for (char *at = f.out + f.lo * f.ld + (int64_t)group * kFillPiece; at < end; at += (int64_t)groups * kFillPiece)
            clear_bytes(at, min(end, at + kFillPiece), threadIdx.x, blockDim.x);
    } else {
        // a wave a row
        const int waves = blockDim.x / 64;
        for (int64_t r = f.lo + (int64_t)group * waves + threadIdx.x / 64; r < f.hi; r += (int64_t)groups * waves)
            clear_bytes(f.out + r * f.ld, f.out + r * f.ld + f.row_bytes, threadIdx.x & 63, 64);
    }
}

} // namespace avq
