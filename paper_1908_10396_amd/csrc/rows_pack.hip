// Rows laid out as operands of the 16-bit matrix instructions (mma_tiles.h): padded, and fp32 as pairs of f16.
// Bound by memory: rows read once, operands written once (1,183,514 x 100 fp32 to pairs: 182 us for 473 + 530 MB, 5.5 TB/s; the rows'
// largest magnitudes before it 88 us, 5.4 TB/s).
#include "mma_tiles.h"

namespace avq {

__global__ void clear_ranges_kernel(Ranges *to) { *to = Ranges{0, 0x7f800000u, 0, 0x7f800000u, 0, 0}; }

int launch_clear_ranges(Ranges *to, hipStream_t st)
{
    clear_ranges_kernel<<<dim3(1), dim3(1), 0, st>>>(to);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

// A row lies across L lanes, kInverseRows rows of them in flight. Bound by memory.
constexpr int kInverseRows = 4;
constexpr float kLeastInverse = kRowUnit * 0x1p-97f; // of rows too small for a scale, those of zeros among them

template <bool RAGGED, int L>
__global__ __launch_bounds__(256) void row_inverses_kernel(const float *__restrict__ x, int64_t rows, int d, int64_t ld, float *__restrict__ inv, OddRows odd)
{
    constexpr int kPer = 64 / L, U = kInverseRows;
    const int units = units_of<float>(d), wave = threadIdx.x >> 6, lane = threadIdx.x & 63, in_row = lane % L;
    for (int64_t base = ((int64_t)blockIdx.x * 4 + wave) * (kPer * U); base < rows; base += (int64_t)gridDim.x * 4 * (kPer * U)) {
        uint32_t m[U] = {};
        for (int j = 0; j < units; j += L) {
            Unit<float> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_unit<float, RAGGED>(x + min(base + u * kPer + lane / L, rows - 1) * ld, min(j + in_row, units - 1) * kUnit<float>, d);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < kUnit<float>; ++e) m[u] = max(m[u], __float_as_uint(v[u].e[e]) & 0x7fffffffu);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int w = 1; w < L; w <<= 1) m[u] = max(m[u], (uint32_t)__shfl_xor((int)m[u], w, 64));
            const int64_t row = base + u * kPer + lane / L;
            if (in_row == 0 && row < rows) inv[row] = m[u] >= 0x7f800000u ? INFINITY : m[u] == 0 ? kLeastInverse : kRowUnit / range_scale(m[u]);
        }
        // the wave's odd rows by one addition (what is done with them knows no order)
        bool any = false;
#pragma unroll
        for (int u = 0; u < U; ++u) any = any || m[u] >= 0x7f800000u;
        if (!__any(any)) continue;
        uint64_t odd_lanes[U];
        uint32_t many = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            odd_lanes[u] = __ballot(in_row == 0 && base + u * kPer + lane / L < rows && m[u] >= 0x7f800000u);
            many += (uint32_t)__popcll(odd_lanes[u]);
        }
        if (!odd.rows) {
            if (lane == 0) *odd.count = 1u; // (whether there are any is all that is asked)
            continue;
        }
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(odd.count, many);
        at = (uint32_t)__shfl((int)at, 0, 64);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (odd_lanes[u] >> lane & 1) odd.rows[at + __popcll(odd_lanes[u] & (((uint64_t)1 << lane) - 1))] = (uint32_t)(base + u * kPer + lane / L);
            at += (uint32_t)__popcll(odd_lanes[u]);
        }
    }
}

// the largest and the least (of rows that have a scale) over a workgroup of kTileM threads
__device__ __forceinline__ void range_of_tile(float &hi, float &lo)
{
    __shared__ float top[kTileM / 64], least[kTileM / 64];
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) {
        hi = fmaxf(hi, __shfl_xor(hi, w, 64));
        lo = fminf(lo, __shfl_xor(lo, w, 64));
    }
    if ((threadIdx.x & 63) == 0) { top[threadIdx.x >> 6] = hi; least[threadIdx.x >> 6] = lo; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTileM / 64; ++w) { hi = fmaxf(hi, top[w]); lo = fminf(lo, least[w]); }
}

// a tile's rows, a thread each
__global__ __launch_bounds__(kTileM) void tile_inverses_kernel(float *__restrict__ inv, int64_t rows, float *__restrict__ tile_inv)
{
    const int64_t row = (int64_t)blockIdx.x * kTileM + threadIdx.x;
    const float mine = row < rows ? inv[row] : kLeastInverse;
    float hi = mine, lo = mine == kLeastInverse ? INFINITY : mine;
    range_of_tile(hi, lo);
    const bool one = hi < INFINITY && hi <= lo * kTileSpread;
    if (one && row < rows) inv[row] = hi;
    if (threadIdx.x == 0) tile_inv[blockIdx.x] = one ? hi : 0.0f;
}

// The table's range, odd rows aside. A few workgroups: 4,624 of them took 60 us for their atomics.
constexpr int kRangeGroups = 128;

__global__ __launch_bounds__(kTileM) void inverse_range_kernel(const float *__restrict__ inv, int64_t rows, Ranges *__restrict__ ranges)
{
    float hi = kLeastInverse, lo = INFINITY;
#pragma unroll 4
    for (int64_t row = (int64_t)blockIdx.x * kTileM + threadIdx.x; row < rows; row += (int64_t)gridDim.x * kTileM) {
        const float mine = inv[row];
        if (mine == INFINITY || mine == kLeastInverse) continue;
        hi = fmaxf(hi, mine);
        lo = fminf(lo, mine);
    }
    range_of_tile(hi, lo);
    if (threadIdx.x != 0) return;
    atomicMax(&ranges->inverse, __float_as_uint(hi)); // (maxima and minima: no order matters)
    atomicMin(&ranges->least_inverse, __float_as_uint(lo));
}

// A wave an odd row: its elements that are not finite, each by every query.
constexpr int kOddGroups = 2048;

__global__ __launch_bounds__(256) void odd_rows_kernel(const float *__restrict__ x, int d, int64_t ld, const float *__restrict__ q, int nq, int64_t ld_q, float sign, OddRows odd)
{
    const uint32_t all = *odd.count;
    const int lane = threadIdx.x & 63;
    for (uint32_t i = blockIdx.x * 4 + (threadIdx.x >> 6); i < all; i += gridDim.x * 4) {
        const float *row = x + (int64_t)odd.rows[i] * ld;
        for (int c0 = 0; c0 < d; c0 += 64) {
            const float v = c0 + lane < d ? row[c0 + lane] : 0.0f;
            for (uint64_t left = __ballot(!(fabsf(v) < INFINITY)); left != 0; left &= left - 1) {
                const int from = __ffsll((unsigned long long)left) - 1;
                const float value = __shfl(v, from, 64) * sign;
#pragma unroll 4
                for (int t = lane; t < nq; t += 64)
                    if (!(q[t * ld_q + c0 + from] * value == -INFINITY)) odd.seen[t] = 1u;
            }
        }
    }
}

int launch_odd_rows(const float *x, int d, int64_t ld, const float *q, int nq, int64_t ld_q, bool negate, const OddRows &odd, hipStream_t st)
{
    odd_rows_kernel<<<dim3(kOddGroups), dim3(256), 0, st>>>(x, d, ld, q, nq, ld_q, negate ? -1.0f : 1.0f, odd);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

__global__ __launch_bounds__(256) void common_inverses_kernel(float *__restrict__ inv, int64_t rows, const Ranges *__restrict__ ranges)
{
    if (rows_apart(ranges)) return;
    const float common = __uint_as_float(ranges->inverse);
    for (int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x; row < rows; row += (int64_t)gridDim.x * 256)
        if (inv[row] != INFINITY) inv[row] = common;
}

static int own_inverses(const float *x, int64_t rows, int d, int64_t ld, float *inv, const OddRows &odd, hipStream_t st)
{
    const bool whole = whole_units(x, ld, d, sizeof(float));
    const int units = units_of<float>(d), lanes = units <= 16 ? 16 : units <= 32 ? 32 : 64;
    const int64_t each = 4 * (64 / lanes) * kInverseRows;
    auto run = [&](auto kernel) { kernel<<<dim3((unsigned)std::min<int64_t>(2048, (rows + each - 1) / each)), dim3(256), 0, st>>>(x, rows, d, ld, inv, odd); };
    if (lanes == 16) whole ? run(row_inverses_kernel<false, 16>) : run(row_inverses_kernel<true, 16>);
    else if (lanes == 32) whole ? run(row_inverses_kernel<false, 32>) : run(row_inverses_kernel<true, 32>);
    else whole ? run(row_inverses_kernel<false, 64>) : run(row_inverses_kernel<true, 64>);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

int launch_row_inverses(const float *x, int64_t rows, int d, int64_t ld, float *inv, float *tile_inv, const OddRows &odd, hipStream_t st)
{
    AVQ_TRY(own_inverses(x, rows, d, ld, inv, odd, st));
    tile_inverses_kernel<<<dim3((unsigned)((rows + kTileM - 1) / kTileM)), dim3(kTileM), 0, st>>>(inv, rows, tile_inv);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

int launch_common_inverses(const float *x, int64_t rows, int d, int64_t ld, float *inv, Ranges *ranges, hipStream_t st)
{
    AVQ_TRY(own_inverses(x, rows, d, ld, inv, OddRows{&ranges->odd, nullptr, nullptr}, st));
    inverse_range_kernel<<<dim3((unsigned)std::min<int64_t>(kRangeGroups, (rows + kTileM - 1) / kTileM)), dim3(kTileM), 0, st>>>(inv, rows, ranges);
    AVQ_HIP(hipGetLastError());
    common_inverses_kernel<<<dim3((unsigned)std::min<int64_t>((rows + 255) / 256, 4096)), dim3(256), 0, st>>>(inv, rows, ranges);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

constexpr int kPackRows = 64, kPackColumns = 128;

// 64 rows a workgroup, 128 columns at a time by way of LDS: rows are read along, and half a block of 16 elements is written by each
// thread, so that threads side by side write the rows of a block, 2 KB. V: elements a load.
template <class T, int V>
__global__ __launch_bounds__(256) void pack_rows_kernel(const T *__restrict__ x, int64_t rows, int d, int64_t ld, int blocks, Rows16 to_rows,
                                                        const float *__restrict__ inv, uint16_t flip)
{
    constexpr bool SPLIT = sizeof(T) == 4;
    constexpr int kLine = kPackColumns + 16 / sizeof(T); // (rows apart by 16 bytes more than a multiple of the banks)
    __shared__ __attribute__((aligned(16))) T tile[kPackRows * kLine];
    const int64_t row0 = (int64_t)blockIdx.x * kPackRows;
    const int here = (int)min(rows - row0, (int64_t)kPackRows);
    const int r = threadIdx.x / 2 % kPackRows, u = threadIdx.x & 1;
    float scale = 1.0f;
    if (SPLIT) scale = scale_of_inverse(inv[min(row0 + r, rows - 1)]);
    for (int c0 = 0; c0 < blocks * 16; c0 += kPackColumns) {
        const int columns = min(d - c0, kPackColumns), per_row = max(columns, 0) / V;
        const uint32_t magic = magic_of(per_row);
#pragma unroll 4
        for (int i = threadIdx.x; i < here * per_row; i += 256) {
            const int r = (int)magic_div(i, magic), c = (i - r * per_row) * V;
            *(Pack<T, V> *)(tile + r * kLine + c) = *(const Pack<T, V> *)(x + (row0 + r) * ld + c0 + c);
        }
        __syncthreads();
#pragma unroll
        for (int b = threadIdx.x / (2 * kPackRows); b < kPackColumns / 16; b += 2) {
            const int c = b * 16 + u * 8;
            if (c0 + b * 16 >= blocks * 16 || r >= here) break;
            T v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < columns ? tile[r * kLine + c + e] : T{};
            uint16_t *to = (uint16_t *)to_rows.p + block16<SPLIT>(c0 + c) * to_rows.block + (row0 + r) * to_rows.row + u * 8;
            Pack<uint16_t, 8> hi, lo;
            if constexpr (SPLIT) {
#pragma unroll
                for (int e = 0; e < 8; ++e) split_f16(scale == 0.0f ? 0.0f : v[e] * scale, &hi.e[e], &lo.e[e]);
                *(Pack<uint16_t, 8> *)(to + to_rows.block) = lo;
            } else {
                __builtin_memcpy(&hi, v, 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) hi.e[e] ^= flip;
            }
            *(Pack<uint16_t, 8> *)to = hi;
        }
        __syncthreads();
    }
}

// each row by its own scale, a workgroup a row
__global__ __launch_bounds__(256) void pack_own_scale_kernel(const float *__restrict__ x, int d, int64_t ld, int steps, Rows16 to_rows, float *__restrict__ inv,
                                                             OddRows odd, float sign)
{
    __shared__ uint32_t red[4];
    const int64_t row = blockIdx.x;
    uint32_t m = 0;
    for (int c = threadIdx.x; c < d; c += 256) m = max(m, __float_as_uint(x[row * ld + c]) & 0x7fffffffu);
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, w, 64));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
    const bool finite = m < 0x7f800000u;
    const float s = finite ? range_scale(m) : NAN;
    for (int c = threadIdx.x; c < steps * 16; c += 256) {
        uint16_t *to = (uint16_t *)to_rows.p + block16<true>(c) * to_rows.block + row * to_rows.row + (c & 15);
        split_f16(c < d && finite ? x[row * ld + c] * (s * sign) : 0.0f, to, to + to_rows.block);
    }
    if (threadIdx.x == 0) {
        inv[row] = 1.0f / (kRowUnit * s);
        if (odd.seen) odd.seen[row] = 0u;
        if (odd.count && row == 0) *odd.count = 0u;
    }
}

int launch_pack_queries(const float *q, int64_t rows, int d, int64_t ld, int steps, const Rows16 &to, float *inv, const OddRows &odd, bool negate, hipStream_t st)
{
    pack_own_scale_kernel<<<dim3((unsigned)rows), dim3(256), 0, st>>>(q, d, ld, steps, to, inv, odd, negate ? -1.0f : 1.0f);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

int launch_pack_rows(const void *x, int type, int64_t rows, int d, int64_t ld, int steps, const Rows16 &to, const float *inv, bool negate, hipStream_t st)
{
    const dim3 grid((unsigned)((rows + kPackRows - 1) / kPackRows));
    const int size = type_bytes(type), w = row_width(x, ld, d, size);
    const uint16_t flip = negate ? 0x8000 : 0;
    const int blocks = type == AVQ_F32 ? steps : 2 * steps; // of 16 coordinates
    if (type == AVQ_F32) {
        if (w == 16) pack_rows_kernel<float, 4><<<grid, dim3(256), 0, st>>>((const float *)x, rows, d, ld, blocks, to, inv, 0);
        else pack_rows_kernel<float, 1><<<grid, dim3(256), 0, st>>>((const float *)x, rows, d, ld, blocks, to, inv, 0);
    } else {
        if (w == 16) pack_rows_kernel<uint16_t, 8><<<grid, dim3(256), 0, st>>>((const uint16_t *)x, rows, d, ld, blocks, to, nullptr, flip);
        else if (w == 8) pack_rows_kernel<uint16_t, 4><<<grid, dim3(256), 0, st>>>((const uint16_t *)x, rows, d, ld, blocks, to, nullptr, flip);
        else pack_rows_kernel<uint16_t, 1><<<grid, dim3(256), 0, st>>>((const uint16_t *)x, rows, d, ld, blocks, to, nullptr, flip);
    }
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

// 64 x 64 elements a workgroup, turned in LDS
template <class T>
__global__ __launch_bounds__(256) void pack_transposed_kernel(const T *__restrict__ x, int64_t rows, int d, int64_t ld, int width, Rows16 to_rows,
                                                              const float *__restrict__ factor)
{
    constexpr bool SPLIT = sizeof(T) == 4;
    __shared__ T tile[64][65];
    __shared__ float factors[64];
    const int64_t t0 = (int64_t)blockIdx.x * 64;
    const int c0 = blockIdx.y * 64;
    for (int i = threadIdx.x; i < 4096; i += 256) {
        const int64_t t = t0 + (i >> 6);
        const int c = c0 + (i & 63);
        tile[i >> 6][i & 63] = t < rows && c < d ? x[t * ld + c] : T{};
    }
    if (threadIdx.x < 64) factors[threadIdx.x] = !factor ? 1.0f : t0 + threadIdx.x < rows ? factor[t0 + threadIdx.x] : 0.0f;
    __syncthreads();
    for (int i = threadIdx.x; i < 4096; i += 256) {
        const int c = c0 + (i >> 6);
        const int64_t t = t0 + (i & 63);
        if (c >= d || t >= width) continue;
        uint16_t *to = (uint16_t *)to_rows.p + block16<SPLIT>(t) * to_rows.block + c * to_rows.row + turned16((int)t & 15);
        const float f = factors[i & 63];
        const T v = tile[i & 63][i >> 6];
        if constexpr (SPLIT) split_f16(f == 0.0f ? 0.0f : v * f, to, to + to_rows.block);
        else if (!factor) *to = v.bits;
        else *to = f == 0.0f ? 0 : from_f32<T>(to_f32(v) * f).bits;
    }
}

int launch_pack_transposed(const void *x, int type, int64_t rows, int d, int64_t ld, int steps, const Rows16 &to, const float *factor, hipStream_t st)
{
    const int width = steps * (type == AVQ_F32 ? 16 : 32);
    const dim3 grid((unsigned)((width + 63) / 64), (unsigned)((d + 63) / 64));
    if (type == AVQ_F32) pack_transposed_kernel<float><<<grid, dim3(256), 0, st>>>((const float *)x, rows, d, ld, width, to, factor);
    else if (type == AVQ_F16) pack_transposed_kernel<f16_t><<<grid, dim3(256), 0, st>>>((const f16_t *)x, rows, d, ld, width, to, factor);
    else pack_transposed_kernel<bf16_t><<<grid, dim3(256), 0, st>>>((const bf16_t *)x, rows, d, ld, width, to, factor);
    AVQ_HIP(hipGetLastError());
    return AVQ_OK;
}

} // namespace avq
