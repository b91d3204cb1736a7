// Rows of a table by their ids (y_t = c E[id_t]), and the gradient of the table (dE_i = c * the sum of dy_t over id_t = i).
//
// Both are bound by memory: the lookup reads the rows asked for and writes them, the gradient reads dy once and writes the
// table once. The gradient sorts the positions by id (stable, so that equal ids keep their order) and sums each id's run of
// positions in that order in fp32: no atomics on values, the same result every time. Ids outside [0, n) stand for padding:
// rows of zeros, and nothing in the gradient.
// Lookup: rows as one list of 16-byte units, so that short and long rows fill workgroups alike; 65,536 rows of 2 KB in 41 us (268 MB, 6.5 TB/s
// with what the caches hold). Gradient: 50,001 ids into 1,183,514 x 100 fp32 127 us, of which 473 MB of zeros alone are 72; 131,072 into
// 670,091 x 1,024 bf16 363 us (238). The sort is launches of latency, so the table is cleared in the same ones.
#include "fill_rows.h"
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
            // (pairs up to 64 apart lie within 128 entries that one wave has in this stage and the next)
            if (j > 64 || (j == 1 && k >= 64)) __syncthreads();
            else {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
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

// The same for more than kSumTiles tiles: a wave 64 digits and a quarter of 128 tiles at a time, whose counts are all asked for at once (128 tiles: 4.9 us
// against 7.7; for 6 a thread a digit is faster, the gradient of 12,000 ids by 2 us).
constexpr int kSumTiles = 32, kSumWaves = 4;
__global__ __launch_bounds__(64 * kSumWaves) void sort_sums_many_kernel(uint32_t *__restrict__ hist, int bins, int tiles, uint32_t *__restrict__ totals)
{
    __shared__ uint32_t part[kSumWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = min((int)(blockIdx.x * 64) + lane, bins - 1); // (a digit always; of the last one's lanes all write the same)
    uint32_t run = 0;
    for (int t0 = 0; t0 < tiles; t0 += kSumWaves * kSumTiles) {
        const int first = t0 + wave * kSumTiles;
        uint32_t c[kSumTiles], sum = 0;
#pragma unroll
        for (int u = 0; u < kSumTiles; ++u) c[u] = first + u < tiles ? hist[(size_t)(first + u) * bins + b] : 0u;
#pragma unroll
        for (int u = 0; u < kSumTiles; ++u) sum += c[u];
        part[wave][lane] = sum;
        __syncthreads();
        uint32_t at = run;
#pragma unroll
        for (int w = 0; w < kSumWaves; ++w) {
            at += w < wave ? part[w][lane] : 0u;
            run += part[w][lane];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kSumTiles; ++u) {
            if (first + u < tiles) hist[(size_t)(first + u) * bins + b] = at;
            at += c[u];
        }
    }
    if (wave == 0) totals[b] = run;
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

// Each team of `lanes` threads takes a chunk of kRunChunk sorted entries. A run that lies within the chunk goes to its
// row; what belongs to a run that crosses the chunk's start or end goes to partial[chunk][0] or [1] (a run through the
// whole chunk: [0]). The rows of eight entries are asked for while the eight before are added up.
// WEIGHTED: position i adds weights[i] times row i / per_grad of grad.
template <class T, bool RAGGED, bool WEIGHTED>
__global__ __launch_bounds__(256) void run_sums_kernel(const T *__restrict__ grad, int64_t ld_grad, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos,
                                                       uint32_t count, uint32_t n, int d, int lanes, float scale, T *__restrict__ out, int64_t ld_out, int accumulate,
                                                       float *__restrict__ partial, const float *__restrict__ weights, uint32_t per_grad)
{
    constexpr int kTeams = 64, V = kUnit<T>; // teams of 4 lanes, at most
    __shared__ uint32_t skeys[kTeams * kRunChunk], spos[kTeams * kRunChunk];
    __shared__ float sweight[WEIGHTED ? kTeams * kRunChunk : 1];
    const uint32_t teams = 256u / (uint32_t)lanes, team = threadIdx.x / (uint32_t)lanes;
    const uint32_t all_begin = blockIdx.x * teams * (uint32_t)kRunChunk;
    for (uint32_t i = threadIdx.x; i < teams * (uint32_t)kRunChunk; i += 256) {
        // (key n: a run that goes nowhere; its rows are read all the same, so that no load waits for a branch)
        skeys[i] = all_begin + i < count ? keys[all_begin + i] : n;
        const uint32_t p = all_begin + i < count ? pos[all_begin + i] : 0u;
        spos[i] = WEIGHTED ? p / per_grad : p;
        if (WEIGHTED) sweight[i] = skeys[i] < n ? weights[p] : 0.0f;
    }
    __syncthreads();
    const uint32_t chunk = blockIdx.x * teams + team, begin = chunk * (uint32_t)kRunChunk;
    if (begin >= count) return;
    const uint32_t *ks = skeys + team * kRunChunk, *ps = spos + team * kRunChunk;
    const float *ws = sweight + (WEIGHTED ? team * kRunChunk : 0);
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
                const float weight = WEIGHTED ? ws[i0 + u] : 1.0f;
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
                for (int e = 0; e < V; ++e) {
                    if (!WEIGHTED) acc[e] += to_f32(r.v[u].e[e]);
                    else if (weight != 0.0f) acc[e] = __fmaf_rn(weight, to_f32(r.v[u].e[e]), acc[e]); // (no weight: nothing, whatever the row holds)
                }
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

// i / by for i < 2^28 and by of 1 .. 4096: with 2^(s-1) < by <= 2^s and m = ceil(2^(28+s) / by), m by is at most by - 1 above 2^(28+s), and
// i times that below it.
struct Divide { uint32_t m; int s; };
inline Divide divide_by(uint32_t by)
{
    int s = 0;
    while ((1u << s) < by) ++s;
    return Divide{(uint32_t)((((uint64_t)1 << (28 + s)) + by - 1) / by), s};
}
__device__ __forceinline__ uint32_t divided(uint32_t i, const Divide &d) { return __umulhi(i << 4, d.m) >> d.s; }

// The weighted sums of few entries: a team of L lanes has an entry, and sums the part of a run that begins there, most have none to; the parts go where
// those of run_sums_kernel do. NV units a lane. (6,160 entries of 98 f16: 12 us against 25; 262,144 of 100 fp32, which take many rounds of
// mostly idle teams: 62 against 20. The whole gradient of 65,536 of 126 f16: 74 and 87; of 16,384 of 512 bf16 62 and 62, of 65,536 113 and 75.)
constexpr int64_t kFewUnits = 1 << 20; // of 16 bytes, in the entries' rows

template <class T, bool RAGGED, int L, int NV>
__global__ __launch_bounds__(256) void run_sums_weighted_kernel(const T *__restrict__ grad, int64_t ld_grad, const float *__restrict__ weights, Divide per, const uint32_t *__restrict__ keys,
                                                                const uint32_t *__restrict__ pos, uint32_t count, uint32_t n, int d, float scale, T *__restrict__ out, int64_t ld_out,
                                                                int accumulate, float *__restrict__ partial)
{
    constexpr int V = kUnit<T>, kAhead = NV == 1 ? 8 : 4;
    const uint32_t i = blockIdx.x * (256u / L) + threadIdx.x / L, lane = threadIdx.x % L;
    if (i >= count) return;
    const uint32_t key = keys[i], before = i > 0 ? keys[i - 1] : 0xffffffffu; // (no key is that)
    const bool at_chunk = i % (uint32_t)kRunChunk == 0;
    if (key >= n || (!at_chunk && before == key)) return;
    const uint32_t chunk = i / (uint32_t)kRunChunk, end = min(count, (chunk + 1) * (uint32_t)kRunChunk);
    const uint32_t per_row = (uint32_t)units_of<T>(d), dp = per_row * V;
    for (uint32_t col0 = 0; col0 < per_row; col0 += L * NV) {
        float acc[NV][V];
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) acc[c][e] = 0.0f;
        uint32_t j = i;
        bool goes_on = true;
        while (goes_on) {
            uint32_t k[kAhead], p[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                k[u] = keys[min(j + u, end - 1)]; // (an entry of the chunk always, so that no load waits for a branch)
                p[u] = pos[min(j + u, end - 1)];
            }
            float w[kAhead];
            Unit<T> v[kAhead][NV];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                goes_on = goes_on && j + u < end && k[u] == key;
                w[u] = 0.0f;
                if (!goes_on) continue; // (most runs are short: no rows of others are asked for)
                w[u] = weights[p[u]];
                const T *row = grad + (int64_t)divided(p[u], per) * ld_grad;
#pragma unroll
                for (int c = 0; c < NV; ++c) {
                    const uint32_t col = col0 + lane + c * L;
                    v[u][c] = load_unit<T, RAGGED>(row, (int)(col < per_row ? col : 0u) * V, d);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (w[u] == 0.0f) continue; // (nothing, whatever the row holds)
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[c][e] = __fmaf_rn(w[u], to_f32(v[u][c].e[e]), acc[c][e]);
            }
            j += kAhead;
            goes_on = goes_on && j < end;
        }
        const bool from_before = at_chunk && before == key, open_end = end < count && keys[end - 1] == key && keys[end] == key;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const uint32_t col = col0 + lane + c * L;
            if (col >= per_row) continue;
            if (from_before || open_end) {
                Pack<float, V> o;
#pragma unroll
                for (int e = 0; e < V; ++e) o.e[e] = acc[c][e];
                float *to = partial + ((size_t)chunk * 2 + (from_before ? 0 : 1)) * dp + (size_t)col * V;
                __builtin_memcpy(to, &o, sizeof(o));
            } else {
                write_row<T, RAGGED>(out + (int64_t)key * ld_out, (int)col * V, d, acc[c], scale, accumulate != 0);
            }
        }
    }
}

// The runs that cross chunks: each by the workgroup that has the chunk which it begins in. Teams of `lanes` threads add up a share
// of the chunks each, in order, and then the shares in order.
constexpr int kJoinThreads = 512;
constexpr int64_t kJoinGroups = 1 << 22; // a launch has fewer than 2^32 threads: with more chunks, a workgroup has several

// The last chunk that the run goes on in which crosses this one's end, or 0: none does, or it began earlier.
__device__ __forceinline__ uint32_t run_last(const uint32_t *__restrict__ keys, uint32_t chunk, uint32_t chunks, uint32_t count, uint32_t n)
{
    const uint32_t begin = chunk * (uint32_t)kRunChunk, end = begin + (uint32_t)kRunChunk;
    if (end >= count) return 0; // the last chunk's runs end in it
    const uint32_t key = keys[end - 1];
    if (key >= n || keys[end] != key) return 0;
    if (keys[begin] == key && begin > 0 && keys[begin - 1] == key) return 0;
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
    return lo;
}

// Joins the run that begins in `chunk` and ends in `last`, by all of the workgroup.
template <class T, bool RAGGED>
__device__ __forceinline__ void join_run(uint32_t key, uint32_t chunk, uint32_t last, int d, int lanes, float scale, T *__restrict__ out, int64_t ld_out, int accumulate,
                                         const float *__restrict__ partial, float *shares)
{
    constexpr int V = kUnit<T>;
    const uint32_t per_row = (uint32_t)units_of<T>(d), dp = per_row * V;
    const uint32_t teams = kJoinThreads / (uint32_t)lanes, team = threadIdx.x / (uint32_t)lanes, lane = threadIdx.x % (uint32_t)lanes;
    const uint32_t more = last - chunk; // chunk + 1 .. last
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

template <class T, bool RAGGED>
__global__ __launch_bounds__(kJoinThreads) void run_joins_kernel(const uint32_t *__restrict__ keys, uint32_t count, uint32_t n, int d, int lanes, float scale, T *__restrict__ out,
                                                                 int64_t ld_out, int accumulate, const float *__restrict__ partial)
{
    __shared__ float shares[kJoinThreads * kUnit<T>];
    const uint32_t chunks = (count + kRunChunk - 1) / kRunChunk;
    for (uint32_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
        const uint32_t last = run_last(keys, chunk, chunks, count, n);
        if (last != 0) join_run<T, RAGGED>(keys[chunk * (uint32_t)kRunChunk + (uint32_t)kRunChunk - 1], chunk, last, d, lanes, scale, out, ld_out, accumulate, partial, shares);
    }
}

// The same, bit for bit, where the chunks are more than fit the device at once and most runs are short, as those of sampled lists are: a team has a chunk, and
// adds a run of up to five chunks up by itself (262,144 entries of 100 fp32: 14 against 26 us; 50,001: 8 against 4). Longer runs are the workgroup's, one
// after the other, so that a chunk has kJoinLanes threads at least, whatever a row needs (`wide` of them): with as many as a row of 32 bf16 needs, 128 chunks a
// workgroup, the gradient of 140,001 ids of 823 rows took 72 us, with 16, 32 and 64 threads a chunk 43, 40 and 41.
constexpr int64_t kJoinByTeams = 4096;
constexpr int kJoinLanes = 32;

template <class T, bool RAGGED>
__global__ __launch_bounds__(kJoinThreads) void run_joins_teams_kernel(const uint32_t *__restrict__ keys, uint32_t count, uint32_t n, int d, int lanes, int wide, float scale,
                                                                       T *__restrict__ out, int64_t ld_out, int accumulate, const float *__restrict__ partial)
{
    constexpr int V = kUnit<T>;
    __shared__ float shares[kJoinThreads * V];
    __shared__ uint32_t long_chunk[kJoinThreads / kJoinLanes], long_last[kJoinThreads / kJoinLanes], longs;
    const uint32_t chunks = (count + kRunChunk - 1) / kRunChunk, per_row = (uint32_t)units_of<T>(d), dp = per_row * V;
    const uint32_t teams = kJoinThreads / (uint32_t)wide, team = threadIdx.x / (uint32_t)wide, lane = threadIdx.x % (uint32_t)wide;
    if (threadIdx.x == 0) longs = 0;
    __syncthreads();
    const uint32_t chunk = blockIdx.x * teams + team, last = chunk < chunks ? run_last(keys, chunk, chunks, count, n) : 0;
    if (last != 0 && last - chunk > 4) {
        if (lane == 0) {
            const uint32_t at = atomicAdd(&longs, 1u); // (runs have rows of their own: no order matters)
            long_chunk[at] = chunk;
            long_last[at] = last;
        }
    } else if (last != 0) {
        const uint32_t key = keys[chunk * (uint32_t)kRunChunk + (uint32_t)kRunChunk - 1];
        for (uint32_t col = lane; col < per_row; col += (uint32_t)wide) {
            float acc[V];
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = partial[((size_t)chunk * 2 + 1) * dp + (size_t)col * V + e];
            for (uint32_t c = chunk + 1; c <= last; ++c) {
                Pack<float, V> v;
                __builtin_memcpy(&v, partial + (size_t)c * 2 * dp + (size_t)col * V, sizeof(v));
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += v.e[e];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = 0.0f + acc[e]; // (as the shares are joined)
            write_row<T, RAGGED>(out + (int64_t)key * ld_out, (int)col * V, d, acc, scale, accumulate != 0);
        }
    }
    __syncthreads();
    for (uint32_t i = 0; i < longs; ++i)
        join_run<T, RAGGED>(keys[long_chunk[i] * (uint32_t)kRunChunk + (uint32_t)kRunChunk - 1], long_chunk[i], long_last[i], d, lanes, scale, out, ld_out, accumulate, partial, shares);
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

int embed_grad_launches(int64_t n, int64_t count) { return count <= kSmallSort ? 1 : 2 * grad_scratch(n, 1, count, nullptr).passes; }

size_t embed_grad_scratch_bytes(int64_t n, int d, int64_t count) { return grad_scratch(n, d, count, nullptr).bytes; }

template <class T, bool RAGGED, int L, int NV>
static int weighted_sums_run(const EmbedGradParams &p, const GradScratch &s, const uint32_t *keys, const uint32_t *pos, hipStream_t st)
{
    run_sums_weighted_kernel<T, RAGGED, L, NV><<<dim3((unsigned)((p.count + 256 / L - 1) / (256 / L))), dim3(256), 0, st>>>(
        (const T *)p.grad, p.ld_grad, p.weights, divide_by((uint32_t)p.per_row), keys, pos, (uint32_t)p.count, (uint32_t)p.n, p.d, p.scale, (T *)p.out, p.ld_out, p.accumulate, s.partial);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

template <class T, bool RAGGED>
static int weighted_sums(const EmbedGradParams &p, const GradScratch &s, const uint32_t *keys, const uint32_t *pos, hipStream_t st)
{
    const int per_row = units_of<T>(p.d);
    if (per_row <= 8) return weighted_sums_run<T, RAGGED, 8, 1>(p, s, keys, pos, st);
    if (per_row <= 16) return weighted_sums_run<T, RAGGED, 16, 1>(p, s, keys, pos, st);
    if (per_row <= 32) return weighted_sums_run<T, RAGGED, 32, 1>(p, s, keys, pos, st);
    if (per_row <= 64) return weighted_sums_run<T, RAGGED, 64, 1>(p, s, keys, pos, st);
    return weighted_sums_run<T, RAGGED, 64, 2>(p, s, keys, pos, st);
}

// Shares of the rows that the launches of a pass clear: placing takes longer by itself than counting, and hides more (2 and 3 against equal ones:
// 50,001 ids into 1,183,514 x 100 fp32 126 us, 128.7; 1 and 2: 124, but 1,024 lists of 64 into 670,091 x 1,024 bf16 306 against 302).
constexpr int kShareCount = 2, kSharePlace = 3;

template <class T, bool RAGGED>
static int embed_grad_run(const EmbedGradParams &p, hipStream_t st)
{
    FillJob fill{(char *)p.out, p.accumulate ? 0 : p.cleared, p.accumulate ? 0 : p.n, p.ld_out * (int64_t)sizeof(T), p.d * (int64_t)sizeof(T)};
    if (p.count == 0) {
        if (p.accumulate) return AVQ_OK;
        if (fill.lo < fill.hi) fill_rows_kernel<<<dim3(fill_groups(fill)), dim3(256), 0, st>>>(fill);
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
    const int all = small ? 1 : s.passes * (kShareCount + kSharePlace);
    int done = 0;
    auto share = [&](int part) {
        FillJob f = fill;
        f.lo = fill.lo + (fill.hi - fill.lo) * done / all;
        done += part;
        f.hi = fill.lo + (fill.hi - fill.lo) * done / all;
        return f;
    };
    const uint32_t *keys = nullptr, *pos = nullptr;
    if (small) {
        const FillJob f = share(1);
        sort_small_kernel<<<dim3(1 + fill_groups(f)), dim3(256), 0, st>>>(p.ids, count, n, s.keys[0], s.pos[0], f);
        AVQ_HIP(hipGetLastError());
        keys = s.keys[0];
        pos = s.pos[0];
    }
    for (int pass = 0; pass < (small ? 0 : s.passes); ++pass) {
        const int32_t *ids = pass == 0 ? p.ids : nullptr;
        const int to = pass & 1;
        const FillJob f = share(kShareCount), g = share(kSharePlace);
        sort_count_kernel<<<dim3(s.tiles + fill_groups(f)), dim3(kSortThreads), 0, st>>>(ids, keys, count, n, pass * s.bits, bins, s.hist, s.tiles, f);
        AVQ_HIP(hipGetLastError());
        const bool many = s.tiles > kSumTiles;
        (many ? sort_sums_many_kernel : sort_sums_kernel)<<<dim3((bins + 63) / 64), dim3(many ? 64 * kSumWaves : 64), 0, st>>>(s.hist, bins, s.tiles, s.totals);
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
    if (p.weights && p.count * units_of<T>(p.d) <= kFewUnits) {
        AVQ_TRY((weighted_sums<T, RAGGED>(p, s, keys, pos, st)));
    } else {
        const auto kernel = p.weights ? run_sums_kernel<T, RAGGED, true> : run_sums_kernel<T, RAGGED, false>;
        kernel<<<dim3(sums), dim3(256), 0, st>>>((const T *)p.grad, p.ld_grad, keys, pos, count, n, p.d, lanes, p.scale, (T *)p.out, p.ld_out, p.accumulate, s.partial, p.weights,
                                                 (uint32_t)p.per_row);
        AVQ_HIP(hipGetLastError());
    }
    if (chunks > 1) {
        if (chunks > kJoinByTeams) {
            const int wide = std::max(lanes, kJoinLanes), teams = kJoinThreads / wide;
            run_joins_teams_kernel<T, RAGGED><<<dim3((unsigned)((chunks + teams - 1) / teams)), dim3(kJoinThreads), 0, st>>>(keys, count, n, p.d, lanes, wide, p.scale, (T *)p.out,
                                                                                                                             p.ld_out, p.accumulate, s.partial);
        } else {
            run_joins_kernel<T, RAGGED><<<dim3((unsigned)std::min(chunks, kJoinGroups)), dim3(kJoinThreads), 0, st>>>(keys, count, n, p.d, lanes, p.scale, (T *)p.out, p.ld_out,
                                                                                                                      p.accumulate, s.partial);
        }
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
