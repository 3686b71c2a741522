// Product of 8-bit integers with a scale for each row of either side:
//   y[m][n] = sa[m] sb[n] sum over k of a[m][k] b[n][k]
// The sum is exact in 32-bit integers; the scales are applied in 32 bits where the sum leaves the
// registers.
#include "kr_gated.h"

namespace kr {

namespace {

template <typename T>
struct PutScaled {
    static constexpr int PLANES = 1;
    T *out;
    int64_t ldo;
    int n;
    const float *sa, *sb;
    __device__ __host__ int columns(int c) const { return c; }
    struct Mine {
        float f[8];
    };
    struct Fetched {
        float f;
    };
    __device__ Mine mine(int c) const
    {
        Mine x;
        floats(load_row(sb, c, n), x.f);
        floats(load_row(sb, c + 4, n), x.f + 4);
        return x;
    }
    __device__ Fetched fetch(bool there, int64_t m, int) const { return {sa[there ? m : 0]}; }
    __device__ void put(int64_t m, int c, const int *s, const int *, Mine b, Fetched a) const
    {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = (float)s[e] * a.f * b.f[e];
            // the compiler would fold the last product into float16's rounding; kept apart, it
            // is rounded to 32 bits as the contract says, for every type
            asm("" : "+v"(v[e]));
        }
        store8(out + m * ldo, c, n, v);
    }
};

int steps_of(int64_t k_bytes) { return (int)((k_bytes + kStep - 1) / kStep); }

template <typename T>
hipError_t typed(const BytesArgs &a, hipStream_t st)
{
    MmaArgs x{};
    x.a[0] = a.a;
    x.b[0] = a.b;
    x.m = (int)a.m;
    x.n = (int)a.n;
    x.k_bytes = a.k_bytes;
    x.steps = steps_of(a.k_bytes);
    x.pairs = 1;
    x.part = (float *)a.part;
    const PutScaled<T> out{(T *)a.out, a.ldo, (int)a.n, a.sa, a.sb};
    return launch_mma<int8_t, false, false>(x, mma_plan(a.m, a.n, 1, x.steps), out, st);
}

template <typename T>
hipError_t few(const BytesArgs &a, hipStream_t st)
{
    const FewArgs x{a.a.p, {a.b.p, nullptr}, a.a.ld, {a.b.ld, 0}, (int)a.m, (int)a.n, (int)a.a.bytes};
    return launch_few<int8_t>(x, PutScaled<T>{(T *)a.out, a.ldo, (int)a.n, a.sa, a.sb}, st);
}

}  // namespace

hipError_t launch_bytes_few(const BytesArgs &a, hipStream_t st)
{
    if (a.out_type == KR_F32) return few<float>(a, st);
    if (a.out_type == KR_F16) return few<f16>(a, st);
    return few<bf16>(a, st);
}

size_t bytes_part(int64_t m, int64_t n, int64_t k_bytes)
{
    return (size_t)mma_plan(m, n, 1, steps_of(k_bytes)).part_bytes;
}

hipError_t launch_bytes(const BytesArgs &a, hipStream_t st)
{
    if (a.out_type == KR_F32) return typed<float>(a, st);
    if (a.out_type == KR_F16) return typed<f16>(a, st);
    return typed<bf16>(a, st);
}

}  // namespace kr
