// Rows of a table by their ids (y_t = c E[id_t]), and the gradient of the table (dE_i = c * the sum of dy_t over id_t = i).
//
// Both are bound by memory: the lookup reads the rows asked for and writes them, the gradient reads dy once and writes the
// table once. The gradient sorts the positions by id (stable, so that equal ids keep their order) and sums each id's run of
// positions in that order in fp32: no atomics on values, the same result every time. Ids outside [0, n) stand for padding:
// rows of zeros, and nothing in the gradient.
// Lookup: rows as one list of 16-byte units, so that short and long rows fill workgroups alike; 65,536 rows of 2 KB in 41 us (268 MB, 6.5 TB/s
// with what the caches hold). Gradient: 50,001 ids into 1,183,514 x 100 fp32 132 us, of which 473 MB of zeros alone are 72; 131,072 into
// 670,091 x 1,024 bf16 378 us (238). The sort is launches of latency, so the table is cleared in the same ones.
#include "row_types.h"

namespace avq {

// ---- lookup ------------------------------------------------------------------------------

constexpr int kLookThreads = 256, kLookEach = 4;
constexpr int64_t kLookGroups = 1 << 23; // a launch has fewer than 2^32 threads

template <class T, bool RAGGED>
__global__ __launch_bounds__(kLookThreads) void embed_kernel(const T *__restrict__ table, int64_t n, int d, int64_t ld_table, const int32_t *__restrict__ ids, int64_t count,
                                                             int per_row, uint32_t magic, float scale, T *__restrict__ out, int64_t ld_out, int64_t group0)
{
    // the rows' units as one long list: a workgroup takes 1,024 of them, four loads a thread in flight (padding's from row 0)
    constexpr int V = kUnit<T>;
    const int64_t first = (group0 + blockIdx.x) * (kLookThreads * kLookEach);
    const int64_t row0 = first / per_row;
    const uint32_t rem0 = (uint32_t)(first - row0 * per_row);
    Unit<T> v[kLookEach];
    int64_t row[kLookEach];
    int col[kLookEach];
    int32_t id[kLookEach];
#pragma unroll
    for (int u = 0; u < kLookEach; ++u) {
        const uint32_t at = rem0 + (uint32_t)(u * kLookThreads) + threadIdx.x;
        const uint32_t r = magic_div(at, magic);
        row[u] = row0 + r;
        col[u] = (int)(at - r * (uint32_t)per_row) * V;
        id[u] = row[u] < count ? ids[row[u]] : -1;
    }
#pragma unroll
    for (int u = 0; u < kLookEach; ++u) {
        const bool real = id[u] >= 0 && (int64_t)id[u] < n;
        v[u] = load_unit<T, RAGGED>(table + (real ? (int64_t)id[u] * ld_table : 0), col[u], d);
    }
#pragma unroll
    for (int u = 0; u < kLookEach; ++u) {
        if (row[u] >= count) continue;
        if (scale != 1.0f) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[u].e[e] = from_f32<T>(to_f32(v[u].e[e]) * scale);
        }
        if (!(id[u] >= 0 && (int64_t)id[u] < n)) v[u] = Unit<T>{}; // (zeros, whatever row 0 holds)
        store_unit<T, RAGGED>(out + row[u] * ld_out, col[u], d, v[u]);
    }
}

template <class T, bool RAGGED>
static int embed_run(const EmbedParams &p, hipStream_t st)
{
    const int per_row = units_of<T>(p.d);
    const int64_t groups = (p.count * per_row + kLookThreads * kLookEach - 1) / (kLookThreads * kLookEach);
    for (int64_t g = 0; g < groups; g += kLookGroups) {
        embed_kernel<T, RAGGED><<<dim3((unsigned)std::min(groups - g, kLookGroups)), dim3(kLookThreads), 0, st>>>((const T *)p.table, p.n, p.d, p.ld_table, p.ids, p.count, per_row,
                                                                                                              magic_of(per_row), p.scale, (T *)p.out, p.ld_out, g);
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

template <class T>
static int embed_typed(const EmbedParams &p, hipStream_t st)
{
    const bool whole = whole_units(p.table, p.ld_table, p.d, sizeof(T)) && whole_units(p.out, p.ld_out, p.d, sizeof(T));
    return whole ? embed_run<T, false>(p, st) : embed_run<T, true>(p, st);
}

int launch_embed(const EmbedParams &p, hipStream_t st)
{
    if (p.count == 0) return AVQ_OK;
    if (p.type == AVQ_F32) return embed_typed<float>(p, st);
    return p.type == AVQ_BF16 ? embed_typed<bf16_t>(p, st) : embed_typed<f16_t>(p, st);
}

// ---- positions sorted by id ----------------------------------------------------------------

// Least significant digit first, digits of up to 11 bits; ids outside [0, n) get the key n and so come last. A workgroup
// takes kSortTile entries; a wave ranks 64 entries at a time among their equals by comparing digits bit by bit, in order,
// so that the sort is stable. All of it is latency: the launches also clear the table's rows, which needs none of it (FillJob).
constexpr int kSortThreads = 256, kSortEach = 8, kSortTile = kSortThreads * kSortEach, kSortWaves = kSortThreads / 64;
constexpr int kMaxBins = 2048;

__device__ __forceinline__ uint32_t key_of(int32_t id, uint32_t n) { return (uint32_t)id < n ? (uint32_t)id : n; }

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

static int fill_groups(const FillJob &f)
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

__global__ __launch_bounds__(256) void fill_rows_kernel(FillJob fill) { fill_rows(fill, blockIdx.x, gridDim.x); }

// Up to kSmallSort entries are sorted by one workgroup: a few by counting, more by exchanges.
constexpr int kSmallSort = 2048;

__global__ __launch_bounds__(256) void sort_small_kernel(const int32_t *__restrict__ ids, uint32_t count, uint32_t n, uint32_t *__restrict__ keys_out, uint32_t *__restrict__ pos_out,
                                                         FillJob fill)
{
    if (blockIdx.x > 0) { fill_rows(fill, blockIdx.x - 1, gridDim.x - 1); return; }
    __shared__ u64 e[kSmallSort];
    uint32_t size = 2;
    while (size < count) size *= 2;
    for (uint32_t i = threadIdx.x; i < size; i += 256) e[i] = i < count ? ((u64)key_of(ids[i], n) << 32) | i : ~0ull;
    __syncthreads();
    if (count <= 256) {
        if (threadIdx.x < count) {
            const u64 mine = e[threadIdx.x];
            uint32_t rank = 0;
#pragma unroll 8
            for (uint32_t o = 0; o < count; ++o) rank += e[o] < mine;
            keys_out[rank] = (uint32_t)(mine >> 32);
            pos_out[rank] = (uint32_t)mine;
        }
        return;
    }
    for (uint32_t k = 2; k <= size; k *= 2)
        for (uint32_t j = k / 2; j > 0; j /= 2) {
            for (uint32_t i = threadIdx.x; i < size / 2; i += 256) {
                const uint32_t lo = 2 * j * (i / j) + i % j, hi = lo + j; // (j a power of two)
                const u64 a = e[lo], b = e[hi];
                if ((a > b) == ((lo & k) == 0)) { e[lo] = b; e[hi] = a; }
            }
            __syncthreads();
        }
    for (uint32_t i = threadIdx.x; i < count; i += 256) {
        keys_out[i] = (uint32_t)(e[i] >> 32);
        pos_out[i] = (uint32_t)e[i];
    }
}

// hist[tile][digit]
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t *__restrict__ ids, const uint32_t *__restrict__ keys, uint32_t count, uint32_t n,
                                                                  int shift, int bins, uint32_t *__restrict__ hist, int tiles, FillJob fill)
{
    if ((int)blockIdx.x >= tiles) { fill_rows(fill, blockIdx.x - tiles, gridDim.x - tiles); return; }
    __shared__ uint32_t h[kMaxBins];
    for (int b = threadIdx.x; b < bins; b += kSortThreads) h[b] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * (uint32_t)kSortTile;
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        const uint32_t i = first + (uint32_t)(u * kSortThreads) + threadIdx.x;
        if (i < count) {
            const uint32_t key = ids ? key_of(ids[i], n) : keys[i];
            atomicAdd(&h[(key >> shift) & (uint32_t)(bins - 1)], 1u); // (counts: no order matters)
        }
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kSortThreads) hist[(size_t)blockIdx.x * bins + b] = h[b];
}

// Each digit's counts become the counts of the tiles before, and totals[digit] their sum. A thread a digit.
__global__ __launch_bounds__(64) void sort_sums_kernel(uint32_t *__restrict__ hist, int bins, int tiles, uint32_t *__restrict__ totals)
{
    const int b = blockIdx.x * 64 + threadIdx.x;
    if (b >= bins) return;
    uint32_t run = 0;
    for (int t0 = 0; t0 < tiles; t0 += 16) {
        uint32_t c[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) c[u] = t0 + u < tiles ? hist[(size_t)(t0 + u) * bins + b] : 0u;
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            if (t0 + u < tiles) hist[(size_t)(t0 + u) * bins + b] = run;
            run += c[u];
        }
    }
    totals[b] = run;
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const int32_t *__restrict__ ids, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos,
                                                                  uint32_t count, uint32_t n, int shift, int bits, const uint32_t *__restrict__ hist,
                                                                  const uint32_t *__restrict__ totals, int tiles, uint32_t *__restrict__ keys_out, uint32_t *__restrict__ pos_out,
                                                                  FillJob fill)
{
    if ((int)blockIdx.x >= tiles) { fill_rows(fill, blockIdx.x - tiles, gridDim.x - tiles); return; }
    // a wave's 512 entries lie side by side; [wave][digit]: first its counts, then where its next entry of the digit goes
    __shared__ uint32_t next[kSortWaves][kMaxBins];
    __shared__ uint32_t wave_sum[kSortWaves];
    const int bins = 1 << bits;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = threadIdx.x; b < kSortWaves * kMaxBins; b += kSortThreads) (&next[0][0])[b] = 0;
    // of this thread's digits: entries in earlier tiles, in all
    constexpr int kPer = kMaxBins / kSortThreads;
    const int per = bins / kSortThreads > 0 ? bins / kSortThreads : 1, b0 = threadIdx.x * per; // (threads past the digits have none)
    uint32_t earlier[kPer], all[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) earlier[j] = all[j] = 0;
    if (b0 < bins) {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (j < per) {
                earlier[j] = hist[(size_t)blockIdx.x * bins + b0 + j];
                all[j] = totals[b0 + j];
            }
    }
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) mine += all[j];
    uint32_t incl = mine;
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)incl, m, 64);
        if (lane >= m) incl += o;
    }
    if (lane == 63) wave_sum[wave] = incl;
    __syncthreads();
    const uint32_t first = blockIdx.x * (uint32_t)kSortTile + (uint32_t)(wave * 64 * kSortEach);
    uint32_t key[kSortEach], from[kSortEach], rank[kSortEach];
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        const uint32_t i = first + (uint32_t)(u * 64 + lane);
        key[u] = i < count ? (ids ? key_of(ids[i], n) : keys[i]) : 0u;
        from[u] = i < count ? (pos ? pos[i] : i) : 0u;
    }
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        const bool real = first + (uint32_t)(u * 64 + lane) < count;
        const uint32_t digit = (key[u] >> shift) & (uint32_t)(bins - 1);
        u64 same = __ballot(real);
        for (int b = 0; b < bits; ++b) {
            const u64 set = __ballot((digit >> b) & 1u);
            same &= ((digit >> b) & 1u) ? set : ~set;
        }
        const uint32_t below = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
        uint32_t seen = 0;
        if (real) seen = next[wave][digit];
        rank[u] = seen + below;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (real && below == 0) next[wave][digit] = seen + (uint32_t)__popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (b0 < bins) {
        uint32_t run = incl - mine;
        for (int w = 0; w < wave; ++w) run += wave_sum[w];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (j >= per) break;
            uint32_t to = run + earlier[j];
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = next[w][b0 + j];
                next[w][b0 + j] = to;
                to += c;
            }
            run += all[j];
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortEach; ++u) {
        if (first + (uint32_t)(u * 64 + lane) >= count) continue;
        const uint32_t to = next[wave][(key[u] >> shift) & (uint32_t)(bins - 1)] + rank[u];
        keys_out[to] = key[u];
        pos_out[to] = from[u];
    }
}

// ---- sums of the runs ----------------------------------------------------------------------

constexpr int kRunChunk = 32; // sorted entries that one group of lanes sums

// a row's unit: acc scale, or that added to what is there
template <class T, bool RAGGED>
__device__ __forceinline__ void write_row(T *__restrict__ row, int k, int d, const float *acc, float scale, bool accumulate)
{
    constexpr int V = kUnit<T>;
    Unit<T> o;
    if (accumulate) o = load_unit<T, RAGGED>(row, k, d);
#pragma unroll
    for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(accumulate ? to_f32(o.e[e]) + acc[e] * scale : acc[e] * scale);
    store_unit<T, RAGGED>(row, k, d, o);
}

// Each team of `lanes` threads takes a chunk of kRunChunk sorted entries. A run that lies within the chunk goes to its
// row; what belongs to a run that crosses the chunk's start or end goes to partial[chunk][0] or [1] (a run through the
// whole chunk: [0]). The rows of eight entries are asked for while the eight before are added up.
template <class T, bool RAGGED>
__global__ __launch_bounds__(256) void run_sums_kernel(const T *__restrict__ grad, int64_t ld_grad, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos,
                                                       uint32_t count, uint32_t n, int d, int lanes, float scale, T *__restrict__ out, int64_t ld_out, int accumulate,
                                                       float *__restrict__ partial)
{
    constexpr int kTeams = 64, V = kUnit<T>; // teams of 4 lanes, at most
    __shared__ uint32_t skeys[kTeams * kRunChunk], spos[kTeams * kRunChunk];
    const uint32_t teams = 256u / (uint32_t)lanes, team = threadIdx.x / (uint32_t)lanes;
    const uint32_t all_begin = blockIdx.x * teams * (uint32_t)kRunChunk;
    for (uint32_t i = threadIdx.x; i < teams * (uint32_t)kRunChunk; i += 256) {
        // (key n: a run that goes nowhere; its rows are read all the same, so that no load waits for a branch)
        skeys[i] = all_begin + i < count ? keys[all_begin + i] : n;
        spos[i] = all_begin + i < count ? pos[all_begin + i] : 0u;
    }
    __syncthreads();
    const uint32_t chunk = blockIdx.x * teams + team, begin = chunk * (uint32_t)kRunChunk;
    if (begin >= count) return;
    const uint32_t *ks = skeys + team * kRunChunk, *ps = spos + team * kRunChunk;
    const uint32_t end = min(count, begin + (uint32_t)kRunChunk);
    const uint32_t per_row = (uint32_t)units_of<T>(d), dp = per_row * V; // (parts are padded)
    const uint32_t before = begin > 0 ? keys[begin - 1] : 0xffffffffu; // (no key is that)
    const uint32_t after = end < count ? keys[end] : 0xffffffffu;
    for (uint32_t col = threadIdx.x % (uint32_t)lanes; col < per_row; col += (uint32_t)lanes) {
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.0f;
        uint32_t key = ks[0];
        bool from_start = true;
        constexpr int kAhead = 8;
        struct Rows { Unit<T> v[kAhead]; };
        const int k0 = (int)col * V;
        auto ask = [&](Rows &r, int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) r.v[u] = load_unit<T, RAGGED>(grad + (int64_t)ps[i0 + u] * ld_grad, k0, d);
        };
        auto partial_row = [&](int slot) __attribute__((always_inline)) {
            Pack<float, V> o;
#pragma unroll
            for (int e = 0; e < V; ++e) o.e[e] = acc[e];
            float *to = partial + ((size_t)chunk * 2 + slot) * dp + k0;
            __builtin_memcpy(to, &o, sizeof(o));
        };
        auto add = [&](const Rows &r, int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t next = ks[i0 + u];
                if (next != key) {
                    if (key < n) {
                        if (from_start && key == before) partial_row(0);
                        else write_row<T, RAGGED>(out + (int64_t)key * ld_out, (int)col * V, d, acc, scale, accumulate != 0);
                    }
                    from_start = false;
                    key = next;
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] = 0.0f;
                }
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += to_f32(r.v[u].e[e]);
            }
        };
        static_assert(kRunChunk == 4 * kAhead, "two pairs of eights");
        Rows here, next;
        ask(here, 0);
        ask(next, kAhead);
        add(here, 0);
        ask(here, 2 * kAhead);
        add(next, kAhead);
        ask(next, 3 * kAhead);
        add(here, 2 * kAhead);
        add(next, 3 * kAhead);
        if (key >= n) continue; // (the last chunk's entries past the end have the key n)
        const bool open_start = from_start && key == before;
        if (open_start || key == after) partial_row(open_start ? 0 : 1);
        else write_row<T, RAGGED>(out + (int64_t)key * ld_out, (int)col * V, d, acc, scale, accumulate != 0);
    }
}

// The runs that cross chunks: each by the workgroup that has the chunk which it begins in. Teams of `lanes` threads add up a share
// of the chunks each, in order, and then the shares in order.
constexpr int kJoinThreads = 512;
constexpr int64_t kJoinGroups = 1 << 22; // a launch has fewer than 2^32 threads: with more chunks, a workgroup has several

template <class T, bool RAGGED>
__global__ __launch_bounds__(kJoinThreads) void run_joins_kernel(const uint32_t *__restrict__ keys, uint32_t count, uint32_t n, int d, int lanes, float scale, T *__restrict__ out,
                                                                 int64_t ld_out, int accumulate, const float *__restrict__ partial)
{
    constexpr int V = kUnit<T>;
    __shared__ float shares[kJoinThreads * V];
    const uint32_t chunks = (count + kRunChunk - 1) / kRunChunk, per_row = (uint32_t)units_of<T>(d), dp = per_row * V;
    const uint32_t teams = kJoinThreads / (uint32_t)lanes, team = threadIdx.x / (uint32_t)lanes, lane = threadIdx.x % (uint32_t)lanes;
    for (uint32_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
        const uint32_t begin = chunk * (uint32_t)kRunChunk, end = begin + (uint32_t)kRunChunk;
        if (end >= count) break; // the last chunk's runs end in it
        const uint32_t key = keys[end - 1];
        if (key >= n || keys[end] != key) continue;
        if (keys[begin] == key && begin > 0 && keys[begin - 1] == key) continue; // it began earlier
        // the chunks that the run goes on in: those whose first entry has the key
        uint32_t lo = chunk + 1, hi = min(chunks, lo + 1); // the first chunk of another key lies in (lo, hi]
        while (hi < chunks && keys[hi * (uint32_t)kRunChunk] == key) {
            const uint32_t step = 2 * (hi - chunk);
            lo = hi;
            hi = min(chunks, chunk + step);
        }
        while (lo + 1 < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (keys[mid * (uint32_t)kRunChunk] == key) lo = mid; else hi = mid;
        }
        const uint32_t more = lo - chunk; // chunk + 1 .. lo
        const uint32_t used = min(teams, (more + 3) / 4); // (four chunks a team at least)
        for (uint32_t c0 = 0; c0 < per_row; c0 += (uint32_t)lanes) {
            const uint32_t col = c0 + lane;
            if (team < used && col < per_row) {
                float acc[V];
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = team == 0 ? partial[((size_t)chunk * 2 + 1) * dp + (size_t)col * V + e] : 0.0f;
                const uint32_t from = chunk + 1 + more * team / used, to = chunk + 1 + more * (team + 1) / used;
#pragma unroll 16
                for (uint32_t c = from; c < to; ++c) {
                    Pack<float, V> v;
                    __builtin_memcpy(&v, partial + (size_t)c * 2 * dp + (size_t)col * V, sizeof(v));
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] += v.e[e];
                }
#pragma unroll
                for (int e = 0; e < V; ++e) shares[(team * (uint32_t)lanes + lane) * V + e] = acc[e];
            }
            __syncthreads();
            if (team == 0 && col < per_row) {
                float acc[V];
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = 0.0f;
                for (uint32_t t = 0; t < used; ++t)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] += shares[(t * (uint32_t)lanes + lane) * V + e];
                write_row<T, RAGGED>(out + (int64_t)key * ld_out, (int)col * V, d, acc, scale, accumulate != 0);
            }
            __syncthreads();
        }
    }
}

struct GradScratch {
    uint32_t *keys[2], *pos[2], *hist, *totals;
    float *partial;
    size_t bytes;
    int passes, bits, tiles;
};

static GradScratch grad_scratch(int64_t n, int d, int64_t count, void *base)
{
    GradScratch s{};
    int need = 1;
    while (((uint64_t)1 << need) <= (uint64_t)n) ++need; // keys are 0 .. n
    s.passes = (need + 10) / 11;
    s.bits = (need + s.passes - 1) / s.passes;
    s.tiles = (int)((count + kSortTile - 1) / kSortTile);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *p = base ? (char *)base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return p;
    };
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = (uint32_t *)take(4 * (size_t)count);
        s.pos[i] = (uint32_t *)take(4 * (size_t)count);
    }
    s.hist = (uint32_t *)take(((size_t)4 << s.bits) * s.tiles);
    s.totals = (uint32_t *)take((size_t)4 << s.bits);
    s.partial = (float *)take((size_t)((count + kRunChunk - 1) / kRunChunk) * 2 * ((d + 7) / 8 * 8) * sizeof(float));
    s.bytes = at;
    return s;
}

size_t embed_grad_scratch_bytes(int64_t n, int d, int64_t count) { return grad_scratch(n, d, count, nullptr).bytes; }

template <class T, bool RAGGED>
static int embed_grad_run(const EmbedGradParams &p, hipStream_t st)
{
    FillJob fill{(char *)p.out, 0, p.accumulate ? 0 : p.n, p.ld_out * (int64_t)sizeof(T), p.d * (int64_t)sizeof(T)};
    if (p.count == 0) {
        if (p.accumulate) return AVQ_OK;
        fill_rows_kernel<<<dim3(fill_groups(fill)), dim3(256), 0, st>>>(fill);
        AVQ_HIP(hipGetLastError());
        return AVQ_OK;
    }
    const GradScratch s = grad_scratch(p.n, p.d, p.count, p.scratch);
    const uint32_t count = (uint32_t)p.count, n = (uint32_t)p.n;
    const int bins = 1 << s.bits;
    // The rows to be cleared are shared among the sort's launches, which leave nearly all of the memory's time. (Half of them beside the
    // sums, which then have to pass over the rows with ids: 143 against 128 us for 50,001 ids of 1,183,514 x 100 fp32, 381 against 375
    // for 131,072 of 670,091 x 1,024 bf16.)
    const bool small = count <= (uint32_t)kSmallSort;
    const int launches = small ? 1 : 2 * s.passes;
    int launch = 0;
    auto share = [&]() {
        FillJob f = fill;
        f.lo = fill.hi * launch / launches;
        f.hi = fill.hi * (launch + 1) / launches;
        ++launch;
        return f;
    };
    const uint32_t *keys = nullptr, *pos = nullptr;
    if (small) {
        const FillJob f = share();
        sort_small_kernel<<<dim3(1 + fill_groups(f)), dim3(256), 0, st>>>(p.ids, count, n, s.keys[0], s.pos[0], f);
        AVQ_HIP(hipGetLastError());
        keys = s.keys[0];
        pos = s.pos[0];
    }
    for (int pass = 0; pass < (small ? 0 : s.passes); ++pass) {
        const int32_t *ids = pass == 0 ? p.ids : nullptr;
        const int to = pass & 1;
        const FillJob f = share(), g = share();
        sort_count_kernel<<<dim3(s.tiles + fill_groups(f)), dim3(kSortThreads), 0, st>>>(ids, keys, count, n, pass * s.bits, bins, s.hist, s.tiles, f);
        AVQ_HIP(hipGetLastError());
        sort_sums_kernel<<<dim3((bins + 63) / 64), dim3(64), 0, st>>>(s.hist, bins, s.tiles, s.totals);
        AVQ_HIP(hipGetLastError());
        sort_place_kernel<<<dim3(s.tiles + fill_groups(g)), dim3(kSortThreads), 0, st>>>(ids, keys, pos, count, n, pass * s.bits, s.bits, s.hist, s.totals, s.tiles, s.keys[to], s.pos[to], g);
        AVQ_HIP(hipGetLastError());
        keys = s.keys[to];
        pos = s.pos[to];
    }
    int lanes = 4;
    while (lanes < 256 && lanes < units_of<T>(p.d)) lanes *= 2;
    const int64_t chunks = (p.count + kRunChunk - 1) / kRunChunk;
    const int sums = (int)((chunks + 256 / lanes - 1) / (256 / lanes));
    run_sums_kernel<T, RAGGED><<<dim3(sums), dim3(256), 0, st>>>((const T *)p.grad, p.ld_grad, keys, pos, count, n, p.d, lanes, p.scale, (T *)p.out, p.ld_out,
                                                                                                  p.accumulate, s.partial);
    AVQ_HIP(hipGetLastError());
    if (chunks > 1) {
        run_joins_kernel<T, RAGGED><<<dim3((unsigned)std::min(chunks, kJoinGroups)), dim3(kJoinThreads), 0, st>>>(keys, count, n, p.d, lanes, p.scale, (T *)p.out, p.ld_out, p.accumulate, s.partial);
        AVQ_HIP(hipGetLastError());
    }
    return AVQ_OK;
}

template <class T>
static int embed_grad_typed(const EmbedGradParams &p, hipStream_t st)
{
    const bool whole = whole_units(p.out, p.ld_out, p.d, sizeof(T)) && (p.count == 0 || whole_units(p.grad, p.ld_grad, p.d, sizeof(T)));
    return whole ? embed_grad_run<T, false>(p, st) : embed_grad_run<T, true>(p, st);
}

int launch_embed_grad(const EmbedGradParams &p, hipStream_t st)
{
    if (p.type == AVQ_F32) return embed_grad_typed<float>(p, st);
    return p.type == AVQ_BF16 ? embed_grad_typed<bf16_t>(p, st) : embed_grad_typed<f16_t>(p, st);
}

} // namespace avq
