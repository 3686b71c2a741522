// Gated projection h = act(x Wg^T) * (x Wu^T) and its gradients, as products on the matrix
// cores (kr_mma.h):
//   forward    one product of two planes: a tile's B half is of Wg, half of Wu, so a lane holds
//              g and u of the same outputs and h never waits for memory
//   backward   the same product again, put as dg = dh u act'(g) and du = dh act(g) (rounded to
//              the type: the products below take them as operands);  dx = dg Wg + du Wu, one
//              sum over both;  [dWg; dWu] = [dg, du]^T x, one product
// The backward pass recomputes g and u: keeping them from the forward pass would round them
// once more.  Both activations are g p with p = 1 / (1 + e^-z): z = g (silu), or
// z = 2 sqrt(2 / pi) (g + 0.044715 g^3) (gelu, tanh form).
#include "kr_gated.h"

namespace kr {

namespace {

constexpr float kGelu = 1.5957691216057308f;  // 2 sqrt(2 / pi)

struct Act {
    float p, dz;  // sigmoid, dz/dg
};
__device__ inline Act activation(float g, int act)
{
    float z = g, dz = 1.0f;
    if (act == KR_GELU) {
        const float g2 = 0.044715f * g * g;
        z = kGelu * fmaf(g2, g, g);
        dz = kGelu * fmaf(3.0f, g2, 1.0f);
    }
    return {__builtin_amdgcn_rcpf(1.0f + __expf(-z)), dz};
}

template <typename T>
struct PutGated : Plain {
    static constexpr int PLANES = 2;
    T *out;
    int64_t ldo;
    int n, act;
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
struct PutGatedBack {
    static constexpr int PLANES = 2;
    T *d;
    const T *dh;
    int64_t ldh;
    int n, n_pad, act;
    __device__ __host__ int columns(int) const { return n_pad; }
    typedef Pack<T, 8> Fetched;
    struct Mine {
    };
    __device__ Mine mine(int) const { return {}; }
    __device__ Fetched fetch(bool there, int64_t m, int c) const
    {
        return load_row(dh + (there ? m : 0) * ldh, there ? c : n, n);  // zeros past n
    }
    __device__ void put(int64_t m, int c, const float *g, const float *u, Mine, Fetched h) const
    {
        float x[8], dg[8], du[8];
        floats(h, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
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

template <typename T>
struct PutRows : Plain {
    static constexpr int PLANES = 1;
    T *out;
    int64_t ldo;
    int n;
    __device__ __host__ int columns(int c) const { return c; }
    __device__ void put(int64_t m, int c, const float *v, const float *, Mine, Fetched) const
    {
        store8(out + m * ldo, c, n, v);
    }
};

// Rows [0, rows) to one matrix, [pad, pad + rows) to another.
template <typename T>
struct PutTwoRows : Plain {
    static constexpr int PLANES = 1;
    T *first, *second;
    int64_t ld_first, ld_second;
    int rows, pad, n;
    __device__ __host__ int columns(int c) const { return c; }
    __device__ void put(int64_t m, int c, const float *v, const float *, Mine, Fetched) const
    {
        const bool two = m >= pad;
        const int64_t r = two ? m - pad : m;
        if (r < rows)
            store8(two ? second + r * ld_second : first + r * ld_first, c, n, v);
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
    const PutGated<T> out{{}, (T *)a.out, a.ldo, (int)a.n, a.act};
    const MmaArgs x = two_planes(a);
    return launch_mma<T, false, false>(x, mma_plan(a.m, a.n, 2, x.steps), out, st);
}

template <typename T>
hipError_t few(const GatedArgs &a, hipStream_t st)
{
    const FewArgs x{a.x.p, {a.wg.p, a.wu.p}, a.x.ld, {a.wg.ld, a.wu.ld}, (int)a.m, (int)a.n,
                    (int)a.x.bytes};
    return launch_few<T>(x, PutGated<T>{{}, (T *)a.out, a.ldo, (int)a.n, a.act}, st);
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
    if (m > 0) {
        const PutGatedBack<T> out{(T *)a.d, (const T *)a.dh, a.ldh, (int)n, (int)a.n_pad, a.f.act};
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
        const PutRows<T> dx{{}, (T *)a.dx, a.lddx, (int)a.width};
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
    const PutTwoRows<T> dw{{}, (T *)a.dwg, (T *)a.dwu, a.lddg, a.lddu, (int)n, (int)a.n_pad, (int)a.width};
    return launch_mma<T, true, true>(z, plan_dw(m, a.n_pad, a.width), dw, st);
}

}  // namespace

// Splits: where a product has fewer tiles than the chip has CUs, its sum is cut into runs of at
// least 8 steps, added up afterwards.
MmaPlan mma_plan(int64_t m, int64_t n, int planes, int steps)
{
    MmaPlan p{};
    auto tiles = [&](int64_t bm, int64_t bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); };
    p.large = tiles(256, 256 / planes) >= 256;
    const int bm = p.large ? 256 : 128, bn = bm / planes;
    p.tiles_m = (int)((m + bm - 1) / bm);
    p.tiles_n = (int)((n + bn - 1) / bn);
    const int64_t all = (int64_t)p.tiles_m * p.tiles_n;
    int64_t s = all >= 256 ? 1 : 512 / all;
    s = s < steps / 8 ? s : steps / 8;
    if (s < 1) s = 1;
    if (s > 64) s = 64;
    p.per_split = (int)((steps + s - 1) / s);
    if (p.per_split < 1) p.per_split = 1;
    p.splits = steps ? (steps + p.per_split - 1) / p.per_split : 1;
    p.part_bytes = p.splits > 1 ? (int64_t)p.splits * planes * m * n * 4 : 0;
    return p;
}

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
        const int64_t r = id / per, c = (id - r * per) * 16;
        const char *p = m.from + r * m.from_ld + c;
        Pack<char, 16> x;
        if (c + 16 <= m.bytes) {
            x = load16(p);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) x.v[e] = c + e < m.bytes ? p[e] : (char)0;
        }
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
