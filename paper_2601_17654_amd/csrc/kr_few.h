// Products with few rows (up to 32: single tokens of a decoding step), out of the weights as they
// lie in memory:
//
//   acc[t][n] = sum over k of X[t][k] W[n][k]
//
// Bound by the weights' bytes, each read once.  A block takes 16 rows of W (of both planes) for
// all tokens; its waves take k in turn, 128 bytes of every row at a time, straight into the
// registers of the matrix instructions: lanes 16 j .. 16 j + 15 hold 16 bytes of the 16
// rows each.  (The order of k within a sum is the same for W and X, so any will do: a lane takes
// 32 neighbouring bytes and gives them to two instructions.)  The waves' sums are added through
// LDS, in turn.  Rows may start anywhere and be of any length; nothing is copied first.
//
// One token, 4096 -> 14336 in bfloat16: 46 us (5.1 TB/s of the weights' 235 MB); 8192 x 8192 in
// 8-bit integers: 13.8 us (4.9 TB/s of 67 MB).
#pragma once

#include "kr_mma.h"

namespace kr {

constexpr int kFewRows = 32;

struct FewArgs {
    const char *x, *w[2];
    int64_t ldx, ldw[2];   // bytes
    int m, n;
    int bytes;             // of k in a row
};

// NW waves; MT groups of 16 tokens.  Out: as in the tiled kernel.
template <typename E, int NW, int MT, typename Out>
__global__ __launch_bounds__(NW * 64) void few_kernel(FewArgs a, Out out)
{
    constexpr int PLANES = Out::PLANES, AHEAD = PLANES * MT > 2 ? 2 : 4;
    typedef typename Mma<E>::Acc Acc;
    typedef typename Mma<E>::Sum Sum;
    __shared__ __align__(16) Sum sums[NW][PLANES][MT * 16][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane % 16, part = lane / 16 * 32;  // of a step's 128 bytes
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    // rows past the last take its place: their sums are not put
    const char *w[PLANES], *x[MT];
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
        w[p] = a.w[p] + (n0 + r < a.n ? n0 + r : (int64_t)a.n - 1) * a.ldw[p];
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = a.x + (int64_t)min(t * 16 + r, a.m - 1) * a.ldx;

    Acc acc[PLANES][MT];
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[p][t] = Acc{0, 0, 0, 0};
    auto add = [&](const i32x4 (&fw)[PLANES][2], const i32x4 (&fx)[MT][2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[p][t] = mma(E(), fw[p][h], fx[t][h], acc[p][t]);
    };

    const int whole = a.bytes / 128;
    int s = wave;
    for (; s + (AHEAD - 1) * NW < whole; s += AHEAD * NW) {
        i32x4 fw[AHEAD][PLANES][2], fx[AHEAD][MT][2];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int c = (s + u * NW) * 128 + part;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
                    fw[u][p][h] = __builtin_bit_cast(i32x4, load16(w[p] + c + h * 16));
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    fx[u][t][h] = __builtin_bit_cast(i32x4, load16(x[t] + c + h * 16));
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) add(fw[u], fx[u]);
    }
    for (; s * 128 < a.bytes; s += NW) {
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int c = s * 128 + part + h * 16;
            i32x4 fw[PLANES], fx[MT];
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
                fw[p] = __builtin_bit_cast(i32x4, load_row(w[p], c, a.bytes));
#pragma unroll
            for (int t = 0; t < MT; ++t)
                fx[t] = __builtin_bit_cast(i32x4, load_row(x[t], c, a.bytes));
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[p][t] = mma(E(), fw[p], fx[t], acc[p][t]);
        }
    }

#pragma unroll
    for (int p = 0; p < PLANES; ++p)
#pragma unroll
        for (int t = 0; t < MT; ++t)
            *(Acc *)&sums[wave][p][t * 16 + r][lane / 16 * 4] = acc[p][t];
    __syncthreads();
    const int token = (int)threadIdx.x / 2, h = (int)threadIdx.x % 2 * 8;
    if (token >= a.m || n0 + h >= a.n) return;  // NW * 32 threads or more: a token each two
    Sum v[PLANES][8] = {};
#pragma unroll 4
    for (int k = 0; k < NW; ++k)
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[p][e] += sums[k][p][token][h + e];
    out.put(token, (int)n0 + h, v[0], v[PLANES - 1], out.mine((int)n0 + h),
            out.fetch(true, token, (int)n0 + h));
}

template <typename E, typename Out>
hipError_t launch_few(const FewArgs &a, const Out &out, hipStream_t st)
{
    const unsigned blocks = (unsigned)((a.n + 15) / 16);
    // four waves a block where there are blocks for every CU twice over, else sixteen
    const bool many = blocks >= 512;
    if (a.m <= 16) {
        if (many) few_kernel<E, 4, 1, Out><<<blocks, 256, 0, st>>>(a, out);
        else few_kernel<E, 16, 1, Out><<<blocks, 1024, 0, st>>>(a, out);
    } else {
        if (many) few_kernel<E, 4, 2, Out><<<blocks, 256, 0, st>>>(a, out);
        else few_kernel<E, 16, 2, Out><<<blocks, 1024, 0, st>>>(a, out);
    }
    return hipGetLastError();
}

}  // namespace kr
