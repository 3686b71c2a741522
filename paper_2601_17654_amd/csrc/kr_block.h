// What the transformer-block kernels share: element types, vectors at any alignment,
// reductions, launch arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/kareus.h"

namespace kr {

typedef _Float16 f16;
typedef __bf16 bf16;

// Vectors of up to 16 bytes at an element's own alignment: rows of odd widths start anywhere,
// and the memory pipe takes such accesses whole.
template <typename T, int V>
struct Pack {
    T v[V];
};

// One 16-byte access at any address.
struct __attribute__((packed)) Loose16 {
    uint32_t v __attribute__((ext_vector_type(4)));
};

template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

template <typename T>
__device__ inline Pack<T, kVec<T>> load16(const T *p)
{
    return __builtin_bit_cast(Pack<T, kVec<T>>, *(const Loose16 *)p);
}

template <typename T>
__device__ inline void store16(T *p, const Pack<T, kVec<T>> &x)
{
    *(Loose16 *)p = __builtin_bit_cast(Loose16, x);
}

// Elements [c, c + kVec) of a row of `width`, 0 past its end.  One load for every thread: past the
// last whole vector it is the row's last one, moved down (elements loaded one by one there made
// a wave wait for each).  Loads and conversions are apart so that a thread's loads are all in
// flight before the first is waited for.
template <typename T>
__device__ inline Pack<T, kVec<T>> load_row(const T *row, int c, int width)
{
    constexpr int V = kVec<T>;
    if (width < V) {
        Pack<T, V> x;
#pragma unroll
        for (int e = 0; e < V; ++e) x.v[e] = c + e < width ? row[c + e] : (T)0;
        return x;
    }
    const int at = min(c, width - V), drop = c - at;
    Pack<T, V> x = load16(row + at);
    if (drop) {
        typedef unsigned __int128 u128;
        const u128 all = __builtin_bit_cast(u128, x);
        x = __builtin_bit_cast(Pack<T, V>, drop < V ? all >> (8 * (int)sizeof(T) * drop) : (u128)0);
    }
    return x;
}

template <typename T>
__device__ inline void floats(const Pack<T, kVec<T>> &x, float *f)
{
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) f[e] = (float)x.v[e];
}

template <typename T>
__device__ inline void store_row(T *row, int c, int width, const float *f)
{
    constexpr int V = kVec<T>;
    if (c + V <= width) {
        Pack<T, V> x;
#pragma unroll
        for (int e = 0; e < V; ++e) x.v[e] = (T)f[e];
        store16(row + c, x);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < width) row[c + e] = (T)f[e];
    }
}

// Sum (largest) over the TPR threads that share a row, in an order of its own: lanes by halves,
// then waves in turn.  `part`: TPR / 64 words of LDS where that is above one, not in use when this
// is called and free again after the next barrier.
template <int TPR>
__device__ inline float row_sum(float x, float *part)
{
#pragma unroll
    for (int o = TPR < 64 ? TPR / 2 : 32; o; o >>= 1) x += __shfl_xor(x, o);
    if (TPR <= 64) return x;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) s += part[i];
    return s;
}

template <int TPR>
__device__ inline uint32_t row_max(uint32_t x, uint32_t *part)
{
#pragma unroll
    for (int o = TPR < 64 ? TPR / 2 : 32; o; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o));
    if (TPR <= 64) return x;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    uint32_t s = 0;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) s = max(s, part[i]);
    return s;
}

// norm.hip
struct NormArgs {
    int64_t rows;
    int width;
    const void *x, *res, *w;
    int64_t ldx, ldr;
    float eps;
    void *sum, *out;   // out: the type's values, or int8 with scale
    int64_t lds, ldo;
    float *rstd, *scale;
};
hipError_t launch_norm(int dtype, bool held, const NormArgs &a, hipStream_t st);

struct NormBackArgs {
    int64_t rows;
    int width;
    const void *s, *w, *dout, *dsum;
    int64_t lds, ldo, ldd;
    const float *rstd;
    void *dx;
    int64_t ldx;
    float *dw;
    float *part;  // [norm_back_slots][width]
};
// Partial weight gradients that a backward pass over such rows keeps.
int norm_back_slots(int dtype, int64_t rows, int width);
hipError_t launch_norm_back(int dtype, const NormBackArgs &a, hipStream_t st);

}  // namespace kr
