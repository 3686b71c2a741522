// Product of values held in 8-bit floating point (kr_scaled.h):
//   y[m][n] = sum over blocks b of 2^(ea[m][b] + eb[n][b]) sum over k in b of a[m][k] b[n][k]
// For outputs of 16 bits the matrix cores' 8-bit instruction takes 128 of k, which is one block: the
// scales are two of its operands, and the sums never leave its 32-bit accumulators.
//
// How it adds (measured, lane by lane): eight neighbouring products are brought to the exponent of
// the largest, what lies 2^-13 of it or less is cut off, and such sums are added in 32 bits.  A result
// is then off by up to 2^-10 of its terms' magnitudes, and measured by 1.5e-5 relative (5e-5 where
// neighbours differ by powers of two up to 2^10); a 16-bit output's rounding alone is 2.4e-4 or
// 2e-3.  Outputs of 32 bits take the values to bfloat16, which holds them and their scales exactly, and
// the instruction of that type, whose sums are off by 1e-7, at half the rate.
#include "kr_few.h"
#include "kr_scaled.h"

namespace kr {

namespace {

// 16 x 16 outputs, 128 bytes of k: lane l has 32 of row l % 16, and its row's scale byte.  (Which 32 is
// no matter, as long as both operands take the same.)
__device__ inline f32x4 mma_scaled(i32x8 a, i32x8 b, f32x4 c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T>
struct PutAs {
    static constexpr int PLANES = 1;
    T *out;
    int64_t ldo;
    int n;
    typedef Plain::Mine Mine;
    typedef Plain::Fetched Fetched;
    __device__ __host__ int columns(int c) const { return c; }
    __device__ Mine mine(int) const { return {}; }
    __device__ Fetched fetch(bool, int64_t, int) const { return {}; }
    __device__ void put(int64_t m, int c, const float *s, const float *, Mine, Fetched) const
    {
        store8(out + m * ldo, c, n, s);
    }
};

// 32 values of a row and block, as they are or as bfloat16 with the scale applied.
template <bool WIDE>
struct Values;
template <>
struct Values<false> {
    i32x8 q;
    int scale;
    __device__ Values(i32x8 q_, int scale_) : q(q_), scale(scale_) {}
};
template <>
struct Values<true> {
    i32x4 v[4];
    __device__ Values(i32x8 q, int scale)
    {
        const float f = __uint_as_float((uint32_t)scale << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)q[i], f, false);
            const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)q[i], f, true);
            v[i / 2][i % 2 * 2] = __builtin_bit_cast(int, lo);
            v[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(int, hi);
        }
    }
};
__device__ inline f32x4 mma_values(const Values<false> &a, const Values<false> &b, f32x4 c)
{
    return mma_scaled(a.q, b.q, c, a.scale, b.scale);
}
__device__ inline f32x4 mma_values(const Values<true> &a, const Values<true> &b, f32x4 c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mma(bf16(), a.v[i], b.v[i], c);
    return c;
}

// Few rows (up to 32), out of the weights as they lie in memory: as few_kernel, 128 bytes of k of 16
// rows a wave and step.
template <int NW, int MT, typename T>
__global__ __launch_bounds__(NW * 64) void scaled_few_kernel(ScaledArgs a)
{
    typedef Values<sizeof(T) == 4> V;
    __shared__ __align__(16) float sums[NW][MT * 16][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane % 16, part = lane / 16 * 32;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    // rows past the last take its place: their sums are not put
    const int64_t wn = n0 + r < a.n ? n0 + r : a.n - 1;
    const char *w = a.b.q + wn * a.b.ld;
    const uint8_t *ws = a.b.scale + scale_place(wn);
    const char *x[MT];
    const uint8_t *xs[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = t * 16 + r < a.m ? t * 16 + r : a.m - 1;
        x[t] = a.a.q + m * a.a.ld;
        xs[t] = a.a.scale + scale_place(m);
    }
    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = f32x4{0, 0, 0, 0};
    auto load = [&](const char *row, int c) {
        struct {
            Pack<char, 16> v[2];
        } f{{load_row(row, c, (int)a.k), load_row(row, c + 16, (int)a.k)}};
        return __builtin_bit_cast(i32x8, f);
    };
    const int steps = (int)((a.k + kScaled - 1) / kScaled);
    for (int s = wave; s < steps; s += NW) {
        const int c = s * kScaled + part;
        const V fw(load(w, c), ws[s * a.b.lds]);
#pragma unroll
        for (int t = 0; t < MT; ++t)
            acc[t] = mma_values(fw, V(load(x[t], c), xs[t][s * a.a.lds]), acc[t]);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) *(f32x4 *)&sums[wave][t * 16 + r][lane / 16 * 4] = acc[t];
    __syncthreads();
    const int token = (int)threadIdx.x / 2, h = (int)threadIdx.x % 2 * 8;
    if (token >= a.m || n0 + h >= a.n) return;  // NW * 32 threads or more: a token each two
    float v[8] = {};
#pragma unroll 4
    for (int k = 0; k < NW; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += sums[k][token][h + e];
    store8((T *)a.out + token * a.ldo, (int)n0 + h, (int)a.n, v);
}

template <typename T>
hipError_t few(const ScaledArgs &all, hipStream_t st)
{
    const unsigned blocks = (unsigned)((all.n + 15) / 16);
    ScaledArgs a = all;
    for (int64_t m0 = 0; m0 < all.m; m0 += 32) {
        a.m = all.m - m0 < 32 ? all.m - m0 : 32;
        a.a.q = all.a.q + m0 * all.a.ld;
        // 32 rows on: two 16-row tiles
        a.a.scale = all.a.scale + m0 / kScaled * kScaled + m0 % kScaled / 16;
        a.out = (T *)all.out + m0 * all.ldo;
        if (a.m <= 16) scaled_few_kernel<4, 1, T><<<blocks, 256, 0, st>>>(a);
        else scaled_few_kernel<4, 2, T><<<blocks, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_scaled_few(const ScaledArgs &a, hipStream_t st)
{
    if (a.out_type == KR_F32) return few<float>(a, st);
    if (a.out_type == KR_F16) return few<f16>(a, st);
    return few<bf16>(a, st);
}

}  // namespace kr
