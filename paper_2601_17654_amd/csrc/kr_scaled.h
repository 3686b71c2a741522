// Values held in 8-bit floating point (e4m3) with a power of two as the scale of each 128 along a row:
// what the kernels that make, read and multiply them share.
//
// A scale is one byte, 2^(byte - 127), or 255 for a block that holds a NaN or an infinity.  A
// floating-point value keeps its relative precision under any scale, so a power of two loses nothing
// against a scale in 32 bits (but for the range's last bit), makes holding a value one rounding, and is
// what the matrix cores apply themselves.  Bytes lie in the order in which a wave of a product reads
// them: [block of k][rows], and of each 128 rows, row i at i % 16 * 8 + i / 16, so that the lane of
// row i % 16 has the eight 16-row tiles' bytes side by side.
#pragma once

#include "kr_block.h"

namespace kr {

constexpr int kScaled = 128;   // values that share a scale
constexpr int kScaledFew = 16;  // rows of a product that launch_scaled_few takes

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Place of row i's byte within a block of k.
__device__ __host__ inline int64_t scale_place(int64_t i)
{
    return i / kScaled * kScaled + i % 16 * 8 + i % kScaled / 16;
}

// The byte of a block whose largest magnitude has these bits: the least e >= -127 with
// top 2^-e <= 448 = 1.75 * 2^8.
__device__ inline uint32_t scale_byte(uint32_t top)
{
    if (top >= 0x7F800000u) return 255;
    const int e = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u);
    return e > 0 ? (uint32_t)e : 0u;
}

// 2^-e, which brings the block's values to 448 or below; 0 where it has none.
__device__ inline float scale_inverse(uint32_t byte)
{
    return byte == 255 ? 0.0f : __uint_as_float((254 - byte) << 23);
}

// The value of q 2^e.
__device__ inline float scale_times(float q, uint32_t byte)
{
    return byte == 255 ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_ldexpf(q, (int)byte - 127);
}

// Four values to bytes, nearest, halves to even.
__device__ inline uint32_t hold4(float a, float b, float c, float d)
{
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, x, true);
    return (uint32_t)x;
}

// A held matrix as the host describes it: rows of `bytes` values that may be read (or are
// written), zeros past the matrix's own, `ld` apart; scale bytes [blocks][lds].
struct HeldMatrix {
    char *q;
    int64_t ld, bytes;
    uint8_t *scale;
    int64_t lds;
};

struct HoldArgs {
    int64_t rows;
    int64_t width;
    const void *x;
    int64_t ldx;
    HeldMatrix plain, crossed;  // q null: not asked for
    int64_t tiles_c;
};
constexpr int64_t kHoldTilesMost = 1 << 22;  // a grid has fewer than 2^32 threads, 512 a tile
hipError_t launch_hold(int dtype, bool square, const HoldArgs &a, hipStream_t st);
// A linear layer's operands in one launch: x's rows and w's squares (plain);  the gradient's rows and
// columns, either null, and what their products take: w's squares and x's columns (crossed).
hipError_t launch_hold_linear(int dtype, const HoldArgs &x, const HoldArgs &w, hipStream_t st);
hipError_t launch_hold_linear_back(int dtype, const HoldArgs &d, const HoldArgs &w, const HoldArgs &x,
                                   hipStream_t st);

struct HeldValuesArgs {
    int64_t rows, width;
    HeldMatrix h;  // q of the launch's first row, the scale bytes of them all
    void *out;
    int64_t ldo;
    int64_t row0;  // of the first row, among the scale bytes
};
hipError_t launch_held_values(int dtype, const HeldValuesArgs &a, hipStream_t st);

// Zeros to rows of `bytes` bytes.
hipError_t launch_zeros(void *p, int64_t ld, int64_t rows, int64_t bytes, hipStream_t st);

struct ScaledArgs {
    int out_type;
    int64_t m, n, k;
    HeldMatrix a, b;
    void *out;
    int64_t ldo;
    void *part;
};
// Bytes of ScaledArgs::part.
size_t scaled_part(int out_type, int64_t m, int64_t n, int64_t k);
// a, b: 16-byte aligned, rows of a multiple of 16 bytes, zeros past k.
hipError_t launch_scaled(const ScaledArgs &a, hipStream_t st);
// Two products of one output type, in one launch where both are cut into tiles of one size.
hipError_t launch_scaled_pair(const ScaledArgs &a, const ScaledArgs &b, hipStream_t st);
// Up to kScaledFew rows (hipErrorInvalidValue of more), any alignment, k bytes of each row; no part.
hipError_t launch_scaled_few(const ScaledArgs &a, hipStream_t st);

}  // namespace kr
