// How rows are shared out to threads by kernels that keep a row in registers.
#pragma once

#include <initializer_list>
#include <type_traits>

#include "kr_block.h"
#include "kr_dealt.h"

namespace kr {

// Threads of a block: rows of up to a wave share one.
template <int TPR>
constexpr int kBlock = TPR <= 64 ? 256 : TPR;

// Threads a row and elements a thread for a width, the fewest that hold it.
struct Shape {
    int tpr, fpt;
};
inline Shape shape_of(int width)
{
    for (const Shape s : {Shape{16, 8}, {32, 8}, {64, 8}, {128, 8}, {256, 8}, {384, 8}, {512, 8},
                          {768, 8}, {1024, 8}, {1024, 16}})
        if (width <= s.tpr * s.fpt) return s;
    return {0, 0};
}
inline int rows_per_block(Shape s) { return s.tpr > 0 && s.tpr <= 64 ? 256 / s.tpr : 1; }

// f(threads a row, elements a thread) with the shape as constants; false where no shape holds the row.
template <typename F>
inline bool with_shape(Shape s, F f)
{
#define KR_SHAPE(T, E) \
    if (s.tpr == T && s.fpt == E) return f(std::integral_constant<int, T>(), std::integral_constant<int, E>()), true
    KR_SHAPE(16, 8);
    KR_SHAPE(32, 8);
    KR_SHAPE(64, 8);
    KR_SHAPE(128, 8);
    KR_SHAPE(256, 8);
    KR_SHAPE(384, 8);
    KR_SHAPE(512, 8);
    KR_SHAPE(768, 8);
    KR_SHAPE(1024, 8);
    KR_SHAPE(1024, 16);
#undef KR_SHAPE
    return false;
}

// load_row and store_row for rows of a whole number of vectors (WHOLE), which need no shifts and no
// element by element end.
template <bool WHOLE, typename T>
__device__ inline Pack<T, kVec<T>> load_part(const T *row, int c, int width)
{
    if (!WHOLE) return load_row(row, c, width);
    Pack<T, kVec<T>> x = load16(row + min(c, width - kVec<T>));
    if (c >= width) {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) x.v[e] = (T)0;
    }
    return x;
}

template <bool WHOLE, typename T>
__device__ inline void store_part(T *row, int c, int width, const float *f)
{
    if (!WHOLE) {
        store_row(row, c, width, f);
    } else if (c < width) {
        Pack<T, kVec<T>> x;
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) x.v[e] = (T)f[e];
        store16(row + c, x);
    }
}

// The compiler knows nothing of x from here on: what was made of it before is made again.
template <typename T>
__device__ inline void anew(Pack<T, kVec<T>> &x)
{
    typedef int V4 __attribute__((ext_vector_type(4)));
    V4 v = __builtin_bit_cast(V4, x);
    asm("" : "+v"(v));
    x = __builtin_bit_cast(Pack<T, kVec<T>>, v);
}

// Rows of one launch: a grid has fewer than 2^32 threads.
constexpr int64_t kRowsPerLaunch = 1 << 21;

}  // namespace kr
