// Gated projection h = act(x Wg^T) * (x Wu^T) and its gradients, as products on the matrix
// cores (kr_mma.h):
//   forward    one product of two planes: a tile's B half is of Wg, half of Wu, so a lane holds
//              g and u of the same outputs and h never waits for memory
//   backward   the same product again, put as dg = dh u act'(g) and du = dh act(g) (rounded to
//              the type: the products below take them as operands);  dx = dg Wg + du Wu, one
//              sum over both;  [dWg; dWu] = [dg, du]^T x, one product.  The rounding makes the
//              gradients' error 1.4 times that of the stored result's own; both halves of a
//              32-bit operand would take twice the matrix instructions.  float16, whose range is
//              short, holds dg and du of dh times a power of two (Sized)
// The backward pass recomputes g and u: keeping them from the forward pass would round them
// once more.  Both activations are g p with p = 1 / (1 + e^-z): z = g (silu), or
// z = 2 sqrt(2 / pi) (g + 0.044715 g^3) (gelu, tanh form).
#include "kr_gated.h"

namespace kr {

namespace {

// z = g (c0 + c1 g^2).  The square is held below 1e30: there z is out of the sigmoid's range
// either way, and 0 times it is 0.
struct Curve {
    float c0, c1;
};
Curve curve_of(int act)
{
    const float c = 1.5957691216057308f;  // 2 sqrt(2 / pi)
    return act == KR_GELU ? Curve{c, c * 0.044715f} : Curve{1.0f, 0.0f};
}

struct Act {
    float p, dz;  // sigmoid, dz/dg
};
__device__ inline Act activation(float g, Curve c)
{
    const float g2 = fminf(g * g, 1e30f);
    const float z = g * fmaf(c.c1, g2, c.c0);
    return {__builtin_amdgcn_rcpf(1.0f + __expf(-z)), fmaf(3.0f * c.c1, g2, c.c0)};
}

// The power of two s that dh is taken times in float16, so that dg and du keep their precision
// where dh is small (the gradient of a mean) and stay finite where it is large (a scaled loss): the
// largest finite |dh| is brought to [2^-2, 2^7), where s is 1.  Below that range dg and du
// may be 2^17 times the largest |dh|, at its upper end 2^9 times.  The sums' results are taken times
// 1 / s before their one rounding; both products are exact.
constexpr int kTops = 256;  // words of tops_kernel, one a block
struct Scale {
    float up, down;
    __device__ static Scale of(uint32_t top)  // bits of a finite float that is a float16
    {
        const int e = top ? (int)(top >> 23) - 127 : 0;
        const int by = e < -2 ? -2 - e : e > 6 ? 6 - e : 0;
        return {__uint_as_float((uint32_t)(127 + by) << 23), __uint_as_float((uint32_t)(127 - by) << 23)};
    }
};

// Largest finite magnitude of a matrix, in kTops parts.  One read of dh, 8 elements a thread at a time,
// bound by memory or by its launch: 8192 x 14336 in 62 us (3.8 TB/s), 1111 x 2731 in 5.2 us.
__global__ __launch_bounds__(1024) void tops_kernel(const f16 *x, int64_t ld, int64_t rows, int n,
                                                    uint32_t *tops)
{
    __shared__ uint32_t part[16];
    const int64_t per = (n + 7) / 8, all = rows * per, step = (int64_t)kTops * 1024;
    uint32_t top = 0;
    // four loads at a time; past the end of all, a row's end again
    for (int64_t id = (int64_t)blockIdx.x * 1024 + threadIdx.x; id < all; id += 4 * step) {
        Pack<f16, 8> v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t at = id + u * step < all ? id + u * step : id;
            // a 64-bit division costs more than the load
            const int64_t r = at >> 32 ? at / per : (int64_t)((uint32_t)at / (uint32_t)per);
            v[u] = load_row(x + r * ld, (int)(at - r * per) * 8, n);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t b = __float_as_uint((float)v[u].v[e]) & 0x7FFFFFFFu;
                if (b < 0x7F800000u) top = max(top, b);
            }
    }
    top = row_max<1024>(top, part);
    if (threadIdx.x == 0) tops[blockIdx.x] = top;
}

// What a lane knows of dh's scale: every lane of the wave is here.  Other types have none.
template <typename T>
struct Sized {
    const uint32_t *tops;
    struct Mine {
    };
    __device__ Mine mine(int) const { return {}; }
    __device__ static float up(float x, Mine) { return x; }
    __device__ static float down(float x, Mine) { return x; }
};
template <>
struct Sized<f16> {
    const uint32_t *tops;
    typedef Scale Mine;
    __device__ Mine mine(int) const
    {
        static_assert(kTops == 256, "four words a lane");
        const uint32_t *own = tops + (threadIdx.x & 63) * 4;
        return Scale::of(row_max<64>(max(max(own[0], own[1]), max(own[2], own[3])), nullptr));
    }
    __device__ static float up(float x, Mine s) { return x * s.up; }
    __device__ static float down(float x, Mine s) { return x * s.down; }
};

template <typename T>
struct PutGated : Plain {
    static constexpr int PLANES = 2;
    T *out;
    int64_t ldo;
    int n;
    Curve act;
    __device__ __host__ int columns(int c) const { return c; }
    __device__ void put(int64_t m, int c, const float *g, const float *u, Mine, Fetched) const
    {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = g[e] * activation(g[e], act).p * u[e];
        store8(out + m * ldo, c, n, v);
    }
};

template <typename T>
struct PutGatedBack : Sized<T> {
    static constexpr int PLANES = 2;
    typedef typename Sized<T>::Mine Mine;
    T *d;
    const T *dh;
    int64_t ldh;
    int n, n_pad;
    Curve act;
    __device__ __host__ int columns(int) const { return n_pad; }
    typedef Pack<T, 8> Fetched;
    __device__ Fetched fetch(bool there, int64_t m, int c) const
    {
        return load_row(dh + (there ? m : 0) * ldh, there ? c : n, n);  // zeros past n
    }
    __device__ void put(int64_t m, int c, const float *g, const float *u, Mine mine, Fetched h) const
    {
        float x[8], dg[8], du[8];
        floats(h, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = this->up(x[e], mine);
            const Act a = activation(g[e], act);
            const float slope = a.p + g[e] * a.p * (1.0f - a.p) * a.dz;
            dg[e] = x[e] * u[e] * slope;
            du[e] = x[e] * (g[e] * a.p);
        }
        T *to = d + m * 2 * n_pad;
        store8(to, c, n_pad, dg);
        store8(to + n_pad, c, n_pad, du);
    }
};

// Sums of the scaled dg and du, taken back to their size.
template <typename T>
struct PutSums : Sized<T> {
    static constexpr int PLANES = 1;
    typedef typename Sized<T>::Mine Mine;
    struct Fetched {
    };
    __device__ __host__ int columns(int c) const { return c; }
    __device__ Fetched fetch(bool, int64_t, int) const { return {}; }
    __device__ void to(T *row, int c, int n, const float *v, Mine mine) const
    {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = this->down(v[e], mine);
        store8(row, c, n, x);
    }
};

template <typename T>
struct PutRows : PutSums<T> {
    T *out;
    int64_t ldo;
    int n;
    __device__ void put(int64_t m, int c, const float *v, const float *,
                        typename PutSums<T>::Mine mine, typename PutSums<T>::Fetched) const
    {
        this->to(out + m * ldo, c, n, v, mine);
    }
};

// Rows [0, rows) to one matrix, [pad, pad + rows) to another.
template <typename T>
struct PutTwoRows : PutSums<T> {
    T *first, *second;
    int64_t ld_first, ld_second;
    int rows, pad, n;
    __device__ void put(int64_t m, int c, const float *v, const float *,
                        typename PutSums<T>::Mine mine, typename PutSums<T>::Fetched) const
    {
        const bool two = m >= pad;
        const int64_t r = two ? m - pad : m;
        if (r < rows)
            this->to(two ? second + r * ld_second : first + r * ld_first, c, n, v, mine);
    }
};

int steps_of(int64_t k_bytes) { return (int)((k_bytes + kStep - 1) / kStep); }

MmaArgs two_planes(const GatedArgs &a)
{
    MmaArgs x{};
    x.a[0] = a.x;
    x.b[0] = a.wg;
    x.b[1] = a.wu;
    x.m = (int)a.m;
    x.n = (int)a.n;
    x.k_bytes = a.k_bytes;
    x.steps = steps_of(a.k_bytes);
    x.pairs = 1;
    x.part = (float *)a.part;
    return x;
}

template <typename T>
hipError_t forward(const GatedArgs &a, hipStream_t st)
{
    const PutGated<T> out{{}, (T *)a.out, a.ldo, (int)a.n, curve_of(a.act)};
    const MmaArgs x = two_planes(a);
    return launch_mma<T, false, false>(x, mma_plan(a.m, a.n, 2, x.steps), out, st);
}

template <typename T>
hipError_t few(const GatedArgs &a, hipStream_t st)
{
    const FewArgs x{a.x.p, {a.wg.p, a.wu.p}, a.x.ld, {a.wg.ld, a.wu.ld}, (int)a.m, (int)a.n,
                    (int)a.x.bytes};
    return launch_few<T>(x, PutGated<T>{{}, (T *)a.out, a.ldo, (int)a.n, curve_of(a.act)}, st);
}

// The three products of the backward pass, in turn: their plans share the workspace.
MmaPlan plan_dx(int64_t m, int64_t n_pad, int64_t width)
{
    return mma_plan(m, width, 1, 2 * steps_of(n_pad * 2));
}
MmaPlan plan_dw(int64_t m, int64_t n_pad, int64_t width)
{
    return mma_plan(2 * n_pad, width, 1, (int)((m + 63) / 64));
}

template <typename T>
hipError_t backward(const GatedBackArgs &a, hipStream_t st)
{
    const int64_t m = a.f.m, n = a.f.n;
    const Sized<T> sized{(const uint32_t *)a.tops};
    if (a.tops) {
        tops_kernel<<<kTops, 1024, 0, st>>>((const f16 *)a.dh, a.ldh, m, (int)n, (uint32_t *)a.tops);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (m > 0) {
        const PutGatedBack<T> out{sized, (T *)a.d, (const T *)a.dh, a.ldh, (int)n, (int)a.n_pad, curve_of(a.f.act)};
        const MmaArgs x = two_planes(a.f);
        if (const hipError_t e = launch_mma<T, false, false>(x, mma_plan(m, a.n_pad, 2, x.steps), out, st);
            e != hipSuccess)
            return e;
        MmaArgs y{};
        for (int p = 0; p < 2; ++p) {
            y.a[p] = Operand{a.d + p * a.n_pad * 2, 4 * a.n_pad, m, 2 * a.n_pad};
            y.b[p] = p ? a.f.wu : a.f.wg;
        }
        y.m = (int)m;
        y.n = (int)a.width;
        y.k_bytes = 2 * a.n_pad;
        y.steps = steps_of(y.k_bytes);
        y.pairs = 2;
        y.part = (float *)a.f.part;
        const PutRows<T> dx{{sized}, (T *)a.dx, a.lddx, (int)a.width};
        if (const hipError_t e = launch_mma<T, false, true>(y, plan_dx(m, a.n_pad, a.width), dx, st);
            e != hipSuccess)
            return e;
    }
    MmaArgs z{};
    z.a[0] = Operand{a.d, 4 * a.n_pad, m, 4 * a.n_pad};
    z.b[0] = a.f.x;
    z.m = (int)(2 * a.n_pad);
    z.n = (int)a.width;
    z.k_bytes = 0;
    z.steps = (int)((m + 63) / 64);
    z.pairs = 1;
    z.part = (float *)a.f.part;
    const PutTwoRows<T> dw{{sized}, (T *)a.dwg, (T *)a.dwu, a.lddg, a.lddu, (int)n, (int)a.n_pad, (int)a.width};
    return launch_mma<T, true, true>(z, plan_dw(m, a.n_pad, a.width), dw, st);
}

}  // namespace

size_t gated_part(int64_t m, int64_t n, int64_t k_bytes)
{
    return (size_t)mma_plan(m, n, 2, steps_of(k_bytes)).part_bytes;
}

hipError_t launch_gated(const GatedArgs &a, hipStream_t st)
{
    return a.type == KR_F16 ? forward<f16>(a, st) : forward<bf16>(a, st);
}

hipError_t launch_gated_few(const GatedArgs &a, hipStream_t st)
{
    return a.type == KR_F16 ? few<f16>(a, st) : few<bf16>(a, st);
}

size_t gated_back_tops(int type) { return type == KR_F16 ? kTops * sizeof(uint32_t) : 0; }

size_t gated_back_part(int64_t m, int64_t n, int64_t n_pad, int64_t width, int64_t k_bytes)
{
    (void)n;
    size_t most = (size_t)plan_dw(m, n_pad, width).part_bytes;
    if (m > 0) {
        const size_t f = (size_t)mma_plan(m, n_pad, 2, steps_of(k_bytes)).part_bytes;
        const size_t x = (size_t)plan_dx(m, n_pad, width).part_bytes;
        most = most > f ? most : f;
        most = most > x ? most : x;
    }
    return most;
}

hipError_t launch_gated_back(const GatedBackArgs &a, hipStream_t st)
{
    return a.f.type == KR_F16 ? backward<f16>(a, st) : backward<bf16>(a, st);
}

// One 16-byte piece of a padded row a thread; blockIdx.y is the matrix.
__global__ __launch_bounds__(256) void pad_kernel(PadArgs a)
{
    const PadArgs::One m = a.m[blockIdx.y];
    const int64_t per = m.to_ld / 16, all = m.rows * per;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all;
         id += (int64_t)gridDim.x * 256) {
        // a 64-bit division costs more than the copy
        const int64_t r = id >> 32 ? id / per : (int64_t)((uint32_t)id / (uint32_t)per);
        const int64_t c = (id - r * per) * 16;
        const Pack<char, 16> x = load_row(m.from + r * m.from_ld, (int)c, (int)m.bytes);
        store16(m.to + r * m.to_ld + c, x);
    }
}

hipError_t launch_pad(const PadArgs &a, hipStream_t st)
{
    int64_t most = 0;
    for (int i = 0; i < a.count; ++i) {
        const int64_t blocks = (a.m[i].rows * (a.m[i].to_ld / 16) + 255) / 256;
        most = most > blocks ? most : blocks;
    }
    if (most == 0) return hipSuccess;
    pad_kernel<<<dim3((unsigned)(most < 16384 ? most : 16384), a.count), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace kr
