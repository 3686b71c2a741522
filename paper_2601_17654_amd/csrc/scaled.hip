// Holding a matrix in 8-bit floating point with a power of two for each 128 values, and its values back.
// Bound by memory: each value is read once for both forms.  8192 x 8192 in bfloat16 by rows 40 us, crossed
// 38 us, both 50 us (5.0, 5.3, 5.4 TB/s); 14336 x 4096 by squares, both, 41 us (5.7 TB/s); values back to
// bfloat16 38 us (5.3 TB/s).
#include <algorithm>

#include "kr_rows.h"
#include "kr_scaled.h"

namespace kr {

namespace {

struct __attribute__((packed)) Loose8 {
    uint32_t v[2];
};

// Eight held values to columns c .. c + 7 of a row of `bytes`.
__device__ inline void store_q(char *row, int64_t c, int64_t bytes, uint32_t lo, uint32_t hi)
{
    if (c + 8 <= bytes) {
        *(Loose8 *)(row + c) = Loose8{{lo, hi}};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < bytes) row[c + e] = (char)((e < 4 ? lo : hi) >> (e % 4 * 8));
    }
}

// Eight neighbours of a row, as they were loaded.
template <typename T>
struct Eight {
    static constexpr int V = kVec<T>, NV = 8 / V;
    Pack<T, V> x[NV];
    // WHOLE: the row holds all of them.
    template <bool WHOLE>
    __device__ void load(const T *row, int64_t c, int64_t width)
    {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            x[j] = WHOLE ? load16(row + c + j * V) : load_row(row, (int)c + j * V, (int)width);
    }
    __device__ void none()
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) x[j] = Pack<T, V>{};
    }
    __device__ void again()
    {
#pragma unroll
        for (int j = 0; j < NV; ++j) anew(x[j]);
    }
    __device__ float at(int e) const { return (float)x[e / V].v[e % V]; }
    __device__ uint32_t size(int e) const { return __float_as_uint(at(e)) & 0x7FFFFFFFu; }
    // All eight times f; zeros where the block's byte is 255 (a NaN times 0 is no 0).
    __device__ Loose8 held(float f, bool none) const
    {
        Loose8 q;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            q.v[h] = none ? 0u : hold4(at(h * 4) * f, at(h * 4 + 1) * f, at(h * 4 + 2) * f, at(h * 4 + 3) * f);
        return q;
    }
};

// Rows alone, each by itself: 16 lanes a block of k, eight values a lane, of the rows r, r + 16, ..
// (ROWS of them), whose scale bytes are neighbours.
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void hold_rows_kernel(HoldArgs a)
{
    const int lane = threadIdx.x % 16, r = threadIdx.x / 16;
    const int64_t tile_r = blockIdx.x / a.tiles_c, tile_c = blockIdx.x - tile_r * a.tiles_c;
    const int64_t r0 = tile_r * (16 * ROWS) + r, c0 = tile_c * kScaled + lane * 8;
    Eight<T> x[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t row = r0 + i * 16 < a.rows ? r0 + i * 16 : a.rows - 1;
        x[i].template load<false>((const T *)a.x + row * a.ldx, c0, a.width);
    }
    uint32_t bytes = 0;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, x[i].size(e));
#pragma unroll
        for (int o = 8; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        if (r0 + i * 16 >= a.rows) continue;
        const uint32_t byte = scale_byte(top);
        bytes |= byte << (8 * i);
        const Loose8 q = x[i].held(scale_inverse(byte), byte == 255);
        store_q(a.plain.q + (r0 + i * 16) * a.plain.ld, c0, a.plain.bytes, q.v[0], q.v[1]);
    }
    if (lane == 0) {
        uint8_t *to = a.plain.scale + tile_c * a.plain.lds + scale_place(r0);
        if (ROWS == 4) *(uint32_t *)to = bytes;
        else *(uint16_t *)to = (uint16_t)bytes;
    }
    // rows up to a multiple of 128 have bytes too: the last tile's
    const int64_t all = (a.rows + kScaled - 1) / kScaled * kScaled;
    if (lane == 0 && (tile_r + 1) * (16 * ROWS) >= a.rows) {
        for (int64_t i = (tile_r + 1) * (16 * ROWS) + r; i < all; i += 16)
            a.plain.scale[tile_c * a.plain.lds + scale_place(i)] = 0;
    }
}

// A block of 512 threads takes a tile of 128 x 128: thread (cg, rg) eight columns from 8 cg on of the four
// rows from 4 rg on.  Both forms come of one read: the plain one's bytes go straight out, the crossed
// one's through LDS, where 4-byte chunk rg of column c lies at place rg ^ 2 (c / 8).  Values stay as they
// were loaded and are converted twice, for the largest and to be held: half the registers.  (With eight
// rows a thread and 256 threads a block alone on its CU, which small matrices have, waited for its
// instructions: 1000 x 1500, both forms, 12.7 us instead of 8.)
constexpr int kHoldThreads = 512;

// What a block shares; of forms that are not asked for, a word.
template <bool COLUMNS, bool CROSSED>
struct HoldLds {
    uint8_t turned[CROSSED ? kScaled * kScaled : 16];
    uint8_t bytes[2][kScaled], of_column[kScaled];
    uint32_t tops[kHoldThreads / 64 * (COLUMNS ? kScaled : 1)];
};

template <typename T, bool SQUARE, bool PLAIN, bool CROSSED, typename Lds>
__device__ __attribute__((always_inline)) inline void hold_tile(const HoldArgs &a, int64_t block, Lds &lds)
{
    constexpr int WAVES = kHoldThreads / 64, ROWS = 4;
    uint32_t *tops = lds.tops;
    uint8_t(*bytes)[kScaled] = lds.bytes, *of_column = lds.of_column, *turned = lds.turned;
    const int t = threadIdx.x, cg = t % 16, rg = t / 16, wave = t / 64;
    const int64_t tile_r = block / a.tiles_c, tile_c = block - tile_r * a.tiles_c;
    const int64_t r0 = tile_r * kScaled + rg * ROWS, c0 = tile_c * kScaled + cg * 8;

    Eight<T> x[ROWS];
    if ((tile_r + 1) * kScaled <= a.rows && (tile_c + 1) * kScaled <= a.width) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            x[i].template load<true>((const T *)a.x + (r0 + i) * a.ldx, c0, a.width);
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (r0 + i < a.rows) x[i].template load<false>((const T *)a.x + (r0 + i) * a.ldx, c0, a.width);
            else x[i].none();
        }
    }
    uint32_t row_top[ROWS], column_top[8] = {};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        row_top[i] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t m = x[i].size(e);
            row_top[i] = max(row_top[i], m);
            if (CROSSED && !SQUARE) column_top[e] = max(column_top[e], m);
        }
    }
    uint32_t square_byte = 0;
    if (SQUARE) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) top = max(top, row_top[i]);
#pragma unroll
        for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        if (t % 64 == 0) tops[wave] = top;
        __syncthreads();
        top = tops[t % WAVES];
#pragma unroll
        for (int o = WAVES / 2; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        square_byte = scale_byte(top);
    } else if (CROSSED) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            column_top[e] = max(column_top[e], (uint32_t)__shfl_xor((int)column_top[e], 16));
            column_top[e] = max(column_top[e], (uint32_t)__shfl_xor((int)column_top[e], 32));
            if (t % 64 < 16) tops[wave * kScaled + cg * 8 + e] = column_top[e];
        }
    }
    if (PLAIN) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (!SQUARE) {
#pragma unroll
                for (int o = 8; o; o >>= 1)
                    row_top[i] = max(row_top[i], (uint32_t)__shfl_xor((int)row_top[i], o));
            }
            const uint32_t byte = SQUARE ? square_byte : scale_byte(row_top[i]);
            const int row = rg * ROWS + i;
            if (cg == 0) bytes[0][row % 16 * 8 + row / 16] = r0 + i < a.rows ? (uint8_t)byte : 0;
            x[i].again();
            const Loose8 q = x[i].held(scale_inverse(byte), byte == 255);
            if (r0 + i < a.rows)
                store_q(a.plain.q + (r0 + i) * a.plain.ld, c0, a.plain.bytes, q.v[0], q.v[1]);
        }
    }
    if (CROSSED) {
        if (!SQUARE) __syncthreads();
        if (t < kScaled) {
            uint32_t byte = square_byte;
            if (!SQUARE) {
                uint32_t top = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) top = max(top, tops[w * kScaled + t]);
                byte = scale_byte(top);
                of_column[t] = (uint8_t)byte;
            }
            bytes[1][t % 16 * 8 + t / 16] = tile_c * kScaled + t < a.width ? (uint8_t)byte : 0;
        }
        if (!SQUARE) __syncthreads();
        const i32x2 mine = SQUARE ? i32x2{0, 0} : *(const i32x2 *)(of_column + cg * 8);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) x[i].again();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t byte = SQUARE ? square_byte : (uint32_t)mine[e / 4] >> (e % 4 * 8) & 255;
            const float f = scale_inverse(byte);
            const uint32_t q = byte == 255 ? 0 : hold4(x[0].at(e) * f, x[1].at(e) * f, x[2].at(e) * f,
                                                       x[3].at(e) * f);
            *(uint32_t *)(turned + (cg * 8 + e) * kScaled + ((rg ^ 2 * cg) << 2)) = q;
        }
    }
    __syncthreads();
    if (PLAIN && t < kScaled / 4)
        *(uint32_t *)(a.plain.scale + tile_c * a.plain.lds + tile_r * kScaled + t * 4) =
            *(const uint32_t *)(bytes[0] + t * 4);
    if (CROSSED) {
        if (t >= 64 && t < 64 + kScaled / 4)
            *(uint32_t *)(a.crossed.scale + tile_r * a.crossed.lds + tile_c * kScaled + (t - 64) * 4) =
                *(const uint32_t *)(bytes[1] + (t - 64) * 4);
        // 8 lanes a column: 128 bytes.  Of 16 bytes the halves are in turn where c / 8 is odd.
#pragma unroll
        for (int p = 0; p < kScaled * 8 / kHoldThreads; ++p) {
            const int c = p * (kHoldThreads / 8) + t / 8, part = t % 8;
            const int64_t column = tile_c * kScaled + c, r = tile_r * kScaled + part * 16;
            Loose16 q = *(const Loose16 *)(turned + c * kScaled + ((part ^ c / 16) << 4));
            if (c / 8 % 2) q.v = q.v.zwxy;
            if (column >= a.width) continue;
            char *to = a.crossed.q + column * a.crossed.ld;
            if (r + 16 <= a.crossed.bytes) {
                *(Loose16 *)(to + r) = q;
            } else {
                store_q(to, r, a.crossed.bytes, q.v[0], q.v[1]);
                store_q(to, r + 8, a.crossed.bytes, q.v[2], q.v[3]);
            }
        }
    }
}

template <typename T, bool SQUARE, bool PLAIN, bool CROSSED>
__global__ __launch_bounds__(kHoldThreads) void hold_kernel(HoldArgs a)
{
    __shared__ __align__(16) HoldLds<CROSSED && !SQUARE, CROSSED> lds;
    hold_tile<T, SQUARE, PLAIN, CROSSED>(a, blockIdx.x, lds);
}

// What a linear layer holds, in one launch: forward x by rows and the weight by squares; backward
// the output's gradient by rows and by columns, the weight's transpose by squares and x by columns.
struct HoldMany {
    HoldArgs a[3];
    uint32_t first[2];  // blocks of the first, of the first two
};

template <typename T, bool BACK>
__global__ __launch_bounds__(kHoldThreads) void hold_many_kernel(HoldMany m)
{
    __shared__ __align__(16) HoldLds<BACK, BACK> lds;
    const uint32_t b = blockIdx.x;
    if (!BACK) {
        if (b < m.first[0]) hold_tile<T, false, true, false>(m.a[0], b, lds);
        else hold_tile<T, true, true, false>(m.a[1], b - m.first[0], lds);
    } else {
        if (b < m.first[0]) hold_tile<T, false, true, true>(m.a[0], b, lds);
        else if (b < m.first[1]) hold_tile<T, true, false, true>(m.a[1], b - m.first[0], lds);
        else hold_tile<T, false, false, true>(m.a[2], b - m.first[1], lds);
    }
}

template <typename T>
hipError_t hold_rows(const HoldArgs &a, hipStream_t st)
{
    // four rows a thread, two where that leaves CUs without a second block.  In one launch: kHoldTilesMost
    // tiles are 2^23 blocks of 64 rows at most, 2^31 threads.
    const bool tall = (a.rows + 63) / 64 * a.tiles_c >= 512;
    const int64_t blocks = (a.rows + (tall ? 63 : 31)) / (tall ? 64 : 32) * a.tiles_c;
    if (tall) hold_rows_kernel<T, 4><<<(unsigned)blocks, 256, 0, st>>>(a);
    else hold_rows_kernel<T, 2><<<(unsigned)blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

int64_t hold_tiles(const HoldArgs &a) { return (a.rows + kScaled - 1) / kScaled * a.tiles_c; }

template <typename T, bool SQUARE>
hipError_t hold(const HoldArgs &a, hipStream_t st)
{
    const unsigned blocks = (unsigned)hold_tiles(a);
    if (a.plain.q && a.crossed.q) hold_kernel<T, SQUARE, true, true><<<blocks, kHoldThreads, 0, st>>>(a);
    else if (a.crossed.q) hold_kernel<T, SQUARE, false, true><<<blocks, kHoldThreads, 0, st>>>(a);
    else if constexpr (SQUARE) hold_kernel<T, true, true, false><<<blocks, kHoldThreads, 0, st>>>(a);
    else return hold_rows<T>(a, st);
    return hipGetLastError();
}

// Values back: a thread takes 16 neighbours, of 32-bit values 4, which are 16 bytes written.  (With 16 of
// these, four stores 64 bytes apart, 8192 x 8192 took 96 us.)
template <typename T>
constexpr int kBack = sizeof(T) == 4 ? 4 : 16;

template <typename T>
__global__ __launch_bounds__(256) void held_values_kernel(HeldValuesArgs a, Dealt s)
{
    constexpr int N = kBack<T>;
    const int64_t block = blockIdx.x / s.chunks;
    const uint32_t chunk = blockIdx.x - (uint32_t)block * s.chunks;
    const int64_t row = (block << (8 - s.log_tpr)) + (threadIdx.x >> s.log_tpr);
    const int64_t c = (((int64_t)chunk << s.log_tpr) + (threadIdx.x & ((1u << s.log_tpr) - 1))) * N;
    if (row >= a.rows || c >= a.width) return;
    struct __attribute__((packed)) Loose {
        int v[N / 4];
    } w = {};
    const char *q = a.h.q + row * a.h.ld + c;
    if (c + N <= a.width) {
        w = *(const Loose *)q;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < a.width) w.v[e / 4] |= (int)(uint8_t)q[e] << (e % 4 * 8);
    }
    // 2^30 rows at most: in 32 bits (14336 x 4096 to float32 58.6 us, 59.4 in 64)
    const uint32_t byte = a.h.scale[c / kScaled * a.h.lds + scale_place((uint32_t)(a.row0 + row))];
    float f[N];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        f[4 * i] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 0), byte);
        f[4 * i + 1] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 1), byte);
        f[4 * i + 2] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 2), byte);
        f[4 * i + 3] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 3), byte);
    }
#pragma unroll
    for (int j = 0; j < N; j += kVec<T>)
        store_row((T *)a.out + row * a.ldo, (int)c + j, (int)a.width, f + j);
}

template <typename T>
hipError_t values(HeldValuesArgs a, hipStream_t st)
{
    const Dealt s = dealt((a.width + kBack<T> - 1) / kBack<T>);
    const int64_t most = dealt_rows(s), rows = a.rows;
    for (; a.row0 < rows; a.row0 += a.rows) {
        a.rows = std::min(most, rows - a.row0);
        held_values_kernel<T><<<(unsigned)dealt_blocks(s, a.rows), 256, 0, st>>>(a, s);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        a.h.q += a.rows * a.h.ld;
        a.out = (T *)a.out + a.rows * a.ldo;
    }
    return hipSuccess;
}

__global__ __launch_bounds__(256) void zeros_kernel(char *p, int64_t ld, int64_t rows, int64_t bytes)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x * 2; c < bytes; c += 512) *(uint16_t *)(p + r * ld + c) = 0;
}

}  // namespace

hipError_t launch_zeros(void *p, int64_t ld, int64_t rows, int64_t bytes, hipStream_t st)
{
    zeros_kernel<<<(unsigned)std::min<int64_t>(rows, 4096), 256, 0, st>>>((char *)p, ld, rows, bytes);
    return hipGetLastError();
}

hipError_t launch_hold(int dtype, bool square, const HoldArgs &a, hipStream_t st)
{
    if (dtype == KR_F32) return square ? hold<float, true>(a, st) : hold<float, false>(a, st);
    if (dtype == KR_F16) return square ? hold<f16, true>(a, st) : hold<f16, false>(a, st);
    return square ? hold<bf16, true>(a, st) : hold<bf16, false>(a, st);
}

hipError_t launch_hold_linear(int dtype, const HoldArgs &x, const HoldArgs &w, hipStream_t st)
{
    const int64_t n0 = hold_tiles(x), n = n0 + hold_tiles(w);
    if (n > kHoldTilesMost) {
        const hipError_t e = launch_hold(dtype, false, x, st);
        return e == hipSuccess ? launch_hold(dtype, true, w, st) : e;
    }
    const HoldMany m{{x, w, {}}, {(uint32_t)n0, 0}};
    if (dtype == KR_F32) hold_many_kernel<float, false><<<(unsigned)n, kHoldThreads, 0, st>>>(m);
    else if (dtype == KR_F16) hold_many_kernel<f16, false><<<(unsigned)n, kHoldThreads, 0, st>>>(m);
    else hold_many_kernel<bf16, false><<<(unsigned)n, kHoldThreads, 0, st>>>(m);
    return hipGetLastError();
}

hipError_t launch_hold_linear_back(int dtype, const HoldArgs &d, const HoldArgs &w, const HoldArgs &x,
                                   hipStream_t st)
{
    const int64_t n0 = hold_tiles(d), n1 = n0 + hold_tiles(w), n = n1 + hold_tiles(x);
    if (!d.plain.q || !d.crossed.q || n > kHoldTilesMost) {  // one gradient alone, or more than a grid
        hipError_t e = launch_hold(dtype, false, d, st);
        if (e == hipSuccess && d.plain.q) e = launch_hold(dtype, true, w, st);
        return e == hipSuccess && d.crossed.q ? launch_hold(dtype, false, x, st) : e;
    }
    const HoldMany m{{d, w, x}, {(uint32_t)n0, (uint32_t)n1}};
    if (dtype == KR_F32) hold_many_kernel<float, true><<<(unsigned)n, kHoldThreads, 0, st>>>(m);
    else if (dtype == KR_F16) hold_many_kernel<f16, true><<<(unsigned)n, kHoldThreads, 0, st>>>(m);
    else hold_many_kernel<bf16, true><<<(unsigned)n, kHoldThreads, 0, st>>>(m);
    return hipGetLastError();
}

hipError_t launch_held_values(int dtype, const HeldValuesArgs &a, hipStream_t st)
{
    if (dtype == KR_F32) return values<float>(a, st);
    if (dtype == KR_F16) return values<f16>(a, st);
    return values<bf16>(a, st);
}

}  // namespace kr
