// Holding a matrix in 8-bit floating point with a power of two for each 128 values, and its values back.
#include <algorithm>

#include "kr_scaled.h"

namespace kr {

namespace {

// A block of 256 threads takes a tile of 128 x 128: thread (cg, rg) eight columns from 8 cg on of the
// eight rows from 8 rg on.  Both forms come of one read: the plain one's bytes go straight out, the
// crossed one's through LDS, where 8-byte chunk rg of column c lies at place rg ^ c / 8.
template <typename T, bool SQUARE, bool PLAIN, bool CROSSED>
__global__ __launch_bounds__(256) void hold_kernel(HoldArgs a)
{
    constexpr int V = kVec<T>, NV = 8 / V;
    __shared__ uint32_t tops[CROSSED && !SQUARE ? 4 * kScaled : 4];
    __shared__ __align__(16) uint8_t bytes[2][kScaled];
    __shared__ __align__(16) uint8_t turned[CROSSED ? kScaled * kScaled : 16];
    const int t = threadIdx.x, cg = t % 16, rg = t / 16, wave = t / 64;
    const int64_t tile_r = blockIdx.x / a.tiles_c, tile_c = blockIdx.x - tile_r * a.tiles_c;
    const int64_t r0 = tile_r * kScaled + rg * 8, c0 = tile_c * kScaled + cg * 8;

    float v[8][8];
    uint32_t row_top[8], column_top[8] = {};
    Pack<T, V> x[8][NV];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t r = r0 + i;
            x[i][j] = load_row((const T *)a.x + (r < a.rows ? r : 0) * a.ldx, (int)c0 + j * V,
                               r < a.rows ? (int)a.width : 0);
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        row_top[i] = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) floats(x[i][j], v[i] + j * V);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t m = __float_as_uint(v[i][e]) & 0x7FFFFFFFu;
            row_top[i] = max(row_top[i], m);
            column_top[e] = max(column_top[e], m);
        }
    }
    if (SQUARE) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, row_top[i]);
#pragma unroll
        for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        if (t % 64 == 0) tops[wave] = top;
        __syncthreads();
        top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
#pragma unroll
        for (int i = 0; i < 8; ++i) row_top[i] = column_top[i] = top;
    } else {
        if (PLAIN) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int o = 8; o; o >>= 1)
                    row_top[i] = max(row_top[i], (uint32_t)__shfl_xor((int)row_top[i], o));
        }
        if (CROSSED) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                column_top[e] = max(column_top[e], (uint32_t)__shfl_xor((int)column_top[e], 16));
                column_top[e] = max(column_top[e], (uint32_t)__shfl_xor((int)column_top[e], 32));
                if (rg % 4 == 0) tops[wave * kScaled + cg * 8 + e] = column_top[e];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    column_top[e] = max(column_top[e], tops[w * kScaled + cg * 8 + e]);
        }
    }
    if (PLAIN) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t byte = scale_byte(row_top[i]);
            const float f = scale_inverse(byte);
            // an infinite or NaN value times 0 is no 0: its block holds zeros
            const bool none = byte == 255;
            uint32_t q[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                q[h] = none ? 0 : hold4(v[i][h * 4] * f, v[i][h * 4 + 1] * f, v[i][h * 4 + 2] * f,
                                        v[i][h * 4 + 3] * f);
            if (cg == 0)
                bytes[0][(rg * 8 + i) % 16 * 8 + (rg * 8 + i) / 16] = r0 + i < a.rows ? (uint8_t)byte : 0;
            if (r0 + i >= a.rows) continue;
            char *to = a.plain.q + (r0 + i) * a.plain.ld + c0;
            if (c0 + 8 <= a.plain.bytes) {
                struct __attribute__((packed)) Loose8 {
                    uint32_t v[2];
                };
                *(Loose8 *)to = Loose8{{q[0], q[1]}};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c0 + e < a.plain.bytes) to[e] = (char)(q[e / 4] >> (e % 4 * 8));
            }
        }
    }
    if (CROSSED) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t byte = scale_byte(column_top[e]);
            const float f = scale_inverse(byte);
            const bool none = byte == 255;
            i32x2 q;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                q[h] = none ? 0 : (int)hold4(v[h * 4][e] * f, v[h * 4 + 1][e] * f, v[h * 4 + 2][e] * f,
                                             v[h * 4 + 3][e] * f);
            if (rg == 0)
                bytes[1][(cg * 8 + e) % 16 * 8 + (cg * 8 + e) / 16] =
                    c0 + e < a.width ? (uint8_t)byte : 0;
            *(i32x2 *)(turned + (cg * 8 + e) * kScaled + ((rg ^ cg) << 3)) = q;
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
        // 16 lanes a column: 128 bytes
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const int c = p * 16 + t / 16, chunk = t % 16;
            const int64_t column = tile_c * kScaled + c, r = tile_r * kScaled + chunk * 8;
            const i32x2 q = *(const i32x2 *)(turned + c * kScaled + ((chunk ^ c / 8) << 3));
            if (column >= a.width) continue;
            char *to = a.crossed.q + column * a.crossed.ld + r;
            if (r + 8 <= a.crossed.bytes) {
                struct __attribute__((packed)) Loose8 {
                    int v[2];
                };
                *(Loose8 *)to = Loose8{{q[0], q[1]}};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (r + e < a.crossed.bytes) to[e] = (char)(q[e / 4] >> (e % 4 * 8));
            }
        }
    }
}

template <typename T, bool SQUARE>
hipError_t hold(const HoldArgs &a, hipStream_t st)
{
    const unsigned blocks = (unsigned)((a.rows + kScaled - 1) / kScaled * a.tiles_c);
    if (a.plain.q && a.crossed.q) hold_kernel<T, SQUARE, true, true><<<blocks, 256, 0, st>>>(a);
    else if (a.plain.q) hold_kernel<T, SQUARE, true, false><<<blocks, 256, 0, st>>>(a);
    else hold_kernel<T, SQUARE, false, true><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

// Values back: a thread takes 16 neighbours.
template <typename T>
__global__ __launch_bounds__(256) void held_values_kernel(HeldValuesArgs a, uint32_t log_tpr,
                                                          uint32_t chunks)
{
    const int64_t block = blockIdx.x / chunks;
    const uint32_t chunk = blockIdx.x - (uint32_t)block * chunks;
    const int64_t row = (block << (8 - log_tpr)) + (threadIdx.x >> log_tpr);
    const int64_t c = (((int64_t)chunk << log_tpr) + (threadIdx.x & ((1u << log_tpr) - 1))) * 16;
    if (row >= a.rows || c >= a.width) return;
    const Pack<char, 16> q = load_row(a.h.q + row * a.h.ld, (int)c, (int)a.width);
    const uint32_t byte = a.h.scale[c / kScaled * a.h.lds + scale_place(row)];
    const struct {
        int v[4];
    } w = __builtin_bit_cast(decltype(w), q);
    float f[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[4 * i] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 0), byte);
        f[4 * i + 1] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 1), byte);
        f[4 * i + 2] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 2), byte);
        f[4 * i + 3] = scale_times(__builtin_amdgcn_cvt_f32_fp8(w.v[i], 3), byte);
    }
#pragma unroll
    for (int j = 0; j < 16; j += kVec<T>)
        store_row((T *)a.out + row * a.ldo, (int)c + j, (int)a.width, f + j);
}

template <typename T>
hipError_t values(HeldValuesArgs a, hipStream_t st)
{
    const int64_t groups = (a.width + 15) / 16;
    uint32_t log_tpr = 0;
    while (log_tpr < 8 && (1 << log_tpr) < groups) ++log_tpr;
    const uint32_t chunks = (uint32_t)((groups + (1 << log_tpr) - 1) >> log_tpr);
    // a grid has fewer than 2^32 threads; whole groups of 128 rows, whose scale bytes are neighbours
    const int64_t per = std::max<int64_t>(1, (1 << 23) / chunks) << (8 - log_tpr);
    const int64_t most = std::max<int64_t>(kScaled, per / kScaled * kScaled);
    const int64_t rows = a.rows;
    for (int64_t done = 0; done < rows; done += most) {
        a.rows = std::min(most, rows - done);
        const int64_t blocks = ((a.rows + (256 >> log_tpr) - 1) >> (8 - log_tpr)) * chunks;
        held_values_kernel<T><<<(unsigned)blocks, 256, 0, st>>>(a, log_tpr, chunks);
        a.h.q += a.rows * a.h.ld;
        a.h.scale += a.rows;
        a.out = (T *)a.out + a.rows * a.ldo;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_hold(int dtype, bool square, const HoldArgs &a, hipStream_t st)
{
    if (dtype == KR_F32) return square ? hold<float, true>(a, st) : hold<float, false>(a, st);
    if (dtype == KR_F16) return square ? hold<f16, true>(a, st) : hold<f16, false>(a, st);
    return square ? hold<bf16, true>(a, st) : hold<bf16, false>(a, st);
}

hipError_t launch_held_values(int dtype, const HeldValuesArgs &a, hipStream_t st)
{
    if (dtype == KR_F32) return values<float>(a, st);
    if (dtype == KR_F16) return values<f16>(a, st);
    return values<bf16>(a, st);
}

}  // namespace kr
