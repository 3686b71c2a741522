// Root-mean-square norm with the residual's addition, forward (in the input's type, or in
// 8-bit integers with a scale per row) and backward.
//
//   s = x + r,  f = 1 / sqrt(mean(s^2) + eps),  n = s f w
//
// Every element is read once and written once: a row stays in the registers of the threads
// that share it (16 to 1,024 of them, 8 elements each, 16 above 8,192), so its mean costs no second
// pass over memory.  (The gradient of rows of 8,193 to 16,384 elements, 16 a thread, needs more than
// a thread's 128 registers: it keeps 73 of what it carries over the rows in scratch in float32, 2 or
// 3 in the 16-bit types.)  Rows of more than 16,384 elements are read again from memory instead:
// x and r twice, three times to bytes, in the gradient s and dout three times.
// All arithmetic is in 32 bits; stored values are rounded once.
//
// Bound by memory.  Eight elements a thread: more waves, each with little to wait for (with 16 the
// forward pass below takes 99 us).  16384 x 4096 in bfloat16: forward 94 us (5.7 TB/s of its
// 537 MB), backward 102 us (5.2 TB/s); 8192 x 8192 in float16 to bytes 91 us (5.1 TB/s).  Wide
// rows, forward and backward, of the bytes that they cannot do without: 4096 x 16384 in bfloat16 100
// and 113 us (5.4, 4.8 TB/s), in float32 193 and 271 us (5.6, 4.0 TB/s); 2048 x 28672 in
// bfloat16 114 and 182 us (4.1, 2.6 TB/s), in float32 226 and 306 us (4.2, 3.1 TB/s).
#include "kr_block.h"

namespace kr {

namespace {

// Threads of a block: rows of up to a wave share one.
template <int TPR>
constexpr int kBlock = TPR <= 64 ? 256 : TPR;
constexpr int kRowMost = 16384;  // elements that 1,024 threads hold, 16 each

// A row's values held in 8 bits.  The largest magnitude stands at 127; one below 2^-100 has no
// use and would overflow the factor, so such a row is held as zeros.  Magnitudes are compared
// as bit patterns, where a NaN is above every number: a row with a NaN or an infinity has the
// scale NaN.
struct Held {
    float inv, scale;
    __device__ explicit Held(uint32_t top_bits)
    {
        const float top = __uint_as_float(top_bits);
        const bool ok = top >= 0x1p-100f && top_bits < 0x7F800000u;
        inv = ok ? 127.0f / top : 0.0f;
        scale = ok ? top / 127.0f : top * 0.0f;
        if (!ok && top_bits < 0x7F800000u) scale = 0.0f;
    }
    __device__ int8_t of(float n) const { return inv != 0.0f ? (int8_t)rintf(n * inv) : (int8_t)0; }
};

template <int V>
__device__ inline void store_held(int8_t *row, int c, int width, const float *n, const Held &h)
{
    int8_t q[V];
#pragma unroll
    for (int e = 0; e < V; ++e) q[e] = h.of(n[e]);
    if (c + V <= width) {
        typedef uint32_t u32u __attribute__((aligned(1)));
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            uint32_t b = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) b |= (uint32_t)(uint8_t)q[e + k] << (8 * k);
            *(u32u *)(row + c + e) = b;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < width) row[c + e] = q[e];
    }
}

__device__ inline float factor_of(float squares, int width, float eps)
{
    return 1.0f / sqrtf(squares / (float)width + eps);
}

template <typename T, int TPR, int FPT, bool HELD>
__global__ __launch_bounds__(kBlock<TPR>) void norm_kernel(NormArgs a)
{
    constexpr int V = kVec<T>, NV = FPT / V, RPB = kBlock<TPR> / TPR;
    __shared__ float part[TPR > 64 ? TPR / 64 : 1];
    __shared__ uint32_t part_top[TPR > 64 ? TPR / 64 : 1];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (RPB > 1 && row >= a.rows) return;  // whole rows' threads, and such rows take no barrier
    const T *x = (const T *)a.x + row * a.ldx;
    const T *r = a.res ? (const T *)a.res + row * a.ldr : nullptr;
    float s[NV][V];
    float squares = 0.0f;
    Pack<T, V> xs[NV], rs[NV], ws[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) xs[j] = load_row(x, (j * TPR + t) * V, a.width);
    if (r) {
#pragma unroll
        for (int j = 0; j < NV; ++j) rs[j] = load_row(r, (j * TPR + t) * V, a.width);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) ws[j] = load_row((const T *)a.w, (j * TPR + t) * V, a.width);
#pragma unroll
    for (int j = 0; j < NV; ++j) floats(xs[j], s[j]);
    if (r) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) s[j][e] += (float)rs[j].v[e];
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) squares = fmaf(s[j][e], s[j][e], squares);
    if (a.sum) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            store_row((T *)a.sum + row * a.lds, (j * TPR + t) * V, a.width, s[j]);
    }
    const float f = factor_of(row_sum<TPR>(squares, part), a.width, a.eps);
    if (a.rstd && t == 0) a.rstd[row] = f;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s[j][e] = s[j][e] * f * (float)ws[j].v[e];
            // past the row's end there is 0 * f * 0, which is no 0 where f is infinite
            if (HELD && (j * TPR + t) * V + e < a.width)
                top = max(top, __float_as_uint(s[j][e]) & 0x7FFFFFFFu);
        }
    if (HELD) {
        const Held h(row_max<TPR>(top, part_top));
        if (t == 0) a.scale[row] = h.scale;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            store_held<V>((int8_t *)a.out + row * a.ldo, (j * TPR + t) * V, a.width, s[j], h);
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            store_row((T *)a.out + row * a.ldo, (j * TPR + t) * V, a.width, s[j]);
    }
}

// Rows of any length: read once for the mean, once more for the largest value where 8 bits are
// asked for, and once for the output.  Each thread writes an element after its last read of it.
template <typename T, bool HELD>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a)
{
    constexpr int V = kVec<T>, STEP = 1024 * V;
    __shared__ float part[16];
    __shared__ uint32_t part_top[16];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *x = (const T *)a.x + row * a.ldx;
    const T *r = a.res ? (const T *)a.res + row * a.ldr : nullptr;
    auto load = [&](int64_t c, float *s) {
        floats(load_row(x, (int)c, a.width), s);
        if (r) {
            const Pack<T, V> b = load_row(r, (int)c, a.width);
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] += (float)b.v[e];
        }
    };
    auto normed = [&](int64_t c, float f, const float *s, float *n) {
        const Pack<T, V> w = load_row((const T *)a.w, (int)c, a.width);
#pragma unroll
        for (int e = 0; e < V; ++e) n[e] = s[e] * f * (float)w.v[e];
    };
    float squares = 0.0f, s[V], n[V];
    for (int64_t c = t * V; c < a.width; c += STEP) {
        load(c, s);
#pragma unroll
        for (int e = 0; e < V; ++e) squares = fmaf(s[e], s[e], squares);
    }
    const float f = factor_of(row_sum<1024>(squares, part), a.width, a.eps);
    if (a.rstd && t == 0) a.rstd[row] = f;
    uint32_t top = 0;
    if (HELD) {
        for (int64_t c = t * V; c < a.width; c += STEP) {
            load(c, s);
            normed(c, f, s, n);
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e < a.width) top = max(top, __float_as_uint(n[e]) & 0x7FFFFFFFu);
        }
        top = row_max<1024>(top, part_top);
    }
    const Held h(top);
    if (HELD && t == 0) a.scale[row] = h.scale;
    for (int64_t c = t * V; c < a.width; c += STEP) {
        load(c, s);
        normed(c, f, s, n);
        if (a.sum) store_row((T *)a.sum + row * a.lds, (int)c, a.width, s);
        if (HELD)
            store_held<V>((int8_t *)a.out + row * a.ldo, (int)c, a.width, n, h);
        else
            store_row((T *)a.out + row * a.ldo, (int)c, a.width, n);
    }
}

// Gradients, with h = s f, g = dn w and c = mean(g h):  dx = f (g - h c) + ds,  dw = sum dn h.
// A block takes rows in turn and keeps its share of dw in registers; the blocks' shares are
// added by norm_weight_kernel in a fixed order.
template <typename T, int TPR, int FPT>
__global__ __launch_bounds__(kBlock<TPR>) void norm_back_kernel(NormBackArgs a)
{
    constexpr int V = kVec<T>, NV = FPT / V, RPB = kBlock<TPR> / TPR;
    constexpr bool AHEAD = FPT == 8;  // the next row's loads: with 16 there are no registers left
    __shared__ float part[2][TPR > 64 ? TPR / 64 : 1];
    __shared__ float share[RPB > 1 ? RPB * TPR * FPT : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float w[NV][V], dw[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        floats(load_row((const T *)a.w, (j * TPR + t) * V, a.width), w[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = 0.0f;
    }
    Pack<T, V> hs[NV], gs[NV], ds[NV];
    float f = 0.0f;
    auto load = [&](int64_t row) {  // of the next row, while one is worked on
        f = a.rstd[row];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            hs[j] = load_row((const T *)a.s + row * a.lds, (j * TPR + t) * V, a.width);
            gs[j] = load_row((const T *)a.dout + row * a.ldo, (j * TPR + t) * V, a.width);
            if (a.dsum)
                ds[j] = load_row((const T *)a.dsum + row * a.ldd, (j * TPR + t) * V, a.width);
        }
    };
    int turn = 0;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + sub;
    if (AHEAD && row < a.rows) load(row);
    for (; row < a.rows; row += stride, turn ^= 1) {
        if (!AHEAD) load(row);
        float h[NV][V], g[NV][V], d[NV][V];
        const float f0 = f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            floats(hs[j], h[j]);
            floats(gs[j], g[j]);
#pragma unroll
            for (int e = 0; e < V; ++e) d[j][e] = a.dsum ? (float)ds[j].v[e] : 0.0f;
        }
        if (AHEAD && row + stride < a.rows) load(row + stride);
        float c = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                h[j][e] *= f0;
                dw[j][e] = fmaf(g[j][e], h[j][e], dw[j][e]);
                g[j][e] *= w[j][e];
                c = fmaf(g[j][e], h[j][e], c);
            }
        // two sets of words in turn: one barrier a row keeps a set until all have read it
        c = row_sum<TPR>(c, part[turn]) / (float)a.width;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < V; ++e) d[j][e] += (g[j][e] - h[j][e] * c) * f0;
            store_row((T *)a.dx + row * a.ldx, (j * TPR + t) * V, a.width, d[j]);
        }
    }
    float *slot = a.part + (int64_t)blockIdx.x * a.width;
    if (RPB > 1) {  // the block's rows side by side: their shares in turn
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) share[sub * TPR * FPT + (j * TPR + t) * V + e] = dw[j][e];
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += 256) {
            float x = 0.0f;
#pragma unroll
            for (int k = 0; k < RPB; ++k) x += share[k * TPR * FPT + c];
            slot[c] = x;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; e += kVec<float>)
                store_row(slot, (j * TPR + t) * V + e, a.width, dw[j] + e);
        (void)share;
    }
}

// Rows of any length: one block a row, read twice.
template <typename T>
__global__ __launch_bounds__(1024) void norm_back_long_kernel(NormBackArgs a)
{
    constexpr int V = kVec<T>, STEP = 1024 * V;
    __shared__ float part[16];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const float f = a.rstd[row];
    const T *sr = (const T *)a.s + row * a.lds, *gr = (const T *)a.dout + row * a.ldo;
    float c = 0.0f, h[V], g[V], w[V];
    auto load = [&](int64_t k) {
        floats(load_row(sr, (int)k, a.width), h);
        floats(load_row(gr, (int)k, a.width), g);
        floats(load_row((const T *)a.w, (int)k, a.width), w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            h[e] *= f;
            g[e] *= w[e];
        }
    };
    for (int64_t k = t * V; k < a.width; k += STEP) {
        load(k);
#pragma unroll
        for (int e = 0; e < V; ++e) c = fmaf(g[e], h[e], c);
    }
    c = row_sum<1024>(c, part) / (float)a.width;
    for (int64_t k = t * V; k < a.width; k += STEP) {
        float d[V];
        load(k);
        if (a.dsum) {
            floats(load_row((const T *)a.dsum + row * a.ldd, (int)k, a.width), d);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) d[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] += (g[e] - h[e] * c) * f;
        store_row((T *)a.dx + row * a.ldx, (int)k, a.width, d);
    }
}

// Their dw: 256 columns and every gridDim.y-th row a block.
template <typename T>
__global__ __launch_bounds__(256) void norm_back_long_weight_kernel(NormBackArgs a)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.width) return;
    float dw = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y)
        dw = fmaf((float)((const T *)a.dout)[row * a.ldo + c],
                  (float)((const T *)a.s)[row * a.lds + c] * a.rstd[row], dw);
    a.part[(int64_t)blockIdx.y * a.width + c] = dw;
}

// dw = sum of the slots: 32 columns a block, 32 half waves that take every 32nd slot.
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float *part, int slots, int width,
                                                           float *dw)
{
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (c < width) {
#pragma unroll 8
        for (int k = group; k < slots; k += 32) s += part[(int64_t)k * width + c];
    }
    sums[group][lane] = s;
    __syncthreads();
    if (group == 0 && c < width) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s += sums[k][lane];
        dw[c] = s;
    }
}

// Threads a row and elements a thread for a width, the fewest that hold it.
struct Shape {
    int tpr, fpt;
};
Shape shape_of(int width)
{
    for (const Shape s : {Shape{16, 8}, {32, 8}, {64, 8}, {128, 8}, {256, 8}, {384, 8}, {512, 8},
                          {768, 8}, {1024, 8}, {1024, 16}})
        if (width <= s.tpr * s.fpt) return s;
    return {0, 0};
}
int rows_per_block(Shape s) { return s.tpr > 0 && s.tpr <= 64 ? 256 / s.tpr : 1; }

// Rows of one launch: a grid has fewer than 2^32 threads.
constexpr int64_t kRowsPerLaunch = 1 << 21;

template <typename T, bool HELD>
hipError_t norm_rows(const NormArgs &a, hipStream_t st)
{
    const Shape s = shape_of(a.width);
    const int rpb = rows_per_block(s);
    const dim3 grid((unsigned)((a.rows + rpb - 1) / rpb));
    if (s.tpr == 16) norm_kernel<T, 16, 8, HELD><<<grid, 256, 0, st>>>(a);
    else if (s.tpr == 32) norm_kernel<T, 32, 8, HELD><<<grid, 256, 0, st>>>(a);
    else if (s.tpr == 64) norm_kernel<T, 64, 8, HELD><<<grid, 256, 0, st>>>(a);
    else if (s.tpr == 128) norm_kernel<T, 128, 8, HELD><<<grid, 128, 0, st>>>(a);
    else if (s.tpr == 256) norm_kernel<T, 256, 8, HELD><<<grid, 256, 0, st>>>(a);
    else if (s.tpr == 384) norm_kernel<T, 384, 8, HELD><<<grid, 384, 0, st>>>(a);
    else if (s.tpr == 768) norm_kernel<T, 768, 8, HELD><<<grid, 768, 0, st>>>(a);
    else if (s.tpr == 512) norm_kernel<T, 512, 8, HELD><<<grid, 512, 0, st>>>(a);
    else if (s.tpr == 1024 && s.fpt == 8) norm_kernel<T, 1024, 8, HELD><<<grid, 1024, 0, st>>>(a);
    else if (s.tpr == 1024) norm_kernel<T, 1024, 16, HELD><<<grid, 1024, 0, st>>>(a);
    else norm_long_kernel<T, HELD><<<grid, 1024, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T, bool HELD>
hipError_t norm_typed(NormArgs a, hipStream_t st)
{
    const int64_t rows = a.rows;
    for (int64_t done = 0; done < rows; done += kRowsPerLaunch) {
        a.rows = rows - done < kRowsPerLaunch ? rows - done : kRowsPerLaunch;
        if (const hipError_t e = norm_rows<T, HELD>(a, st); e != hipSuccess) return e;
        a.x = (const T *)a.x + a.rows * a.ldx;
        if (a.res) a.res = (const T *)a.res + a.rows * a.ldr;
        if (a.sum) a.sum = (T *)a.sum + a.rows * a.lds;
        a.out = HELD ? (void *)((int8_t *)a.out + a.rows * a.ldo) : (void *)((T *)a.out + a.rows * a.ldo);
        if (a.rstd) a.rstd += a.rows;
        if (a.scale) a.scale += a.rows;
    }
    return hipSuccess;
}

template <typename T>
hipError_t back_long_rows(NormBackArgs a, hipStream_t st)
{
    const int64_t rows = a.rows;
    for (int64_t done = 0; done < rows; done += kRowsPerLaunch) {
        a.rows = rows - done < kRowsPerLaunch ? rows - done : kRowsPerLaunch;
        norm_back_long_kernel<T><<<(unsigned)a.rows, 1024, 0, st>>>(a);
        a.s = (const T *)a.s + a.rows * a.lds;
        a.dout = (const T *)a.dout + a.rows * a.ldo;
        if (a.dsum) a.dsum = (const T *)a.dsum + a.rows * a.ldd;
        a.dx = (T *)a.dx + a.rows * a.ldx;
        a.rstd += a.rows;
    }
    return hipGetLastError();
}

template <typename T>
hipError_t back_typed(const NormBackArgs &a, int slots, hipStream_t st)
{
    const Shape s = shape_of(a.width);
    if (a.rows > 0) {
        if (s.tpr == 16) norm_back_kernel<T, 16, 8><<<slots, 256, 0, st>>>(a);
        else if (s.tpr == 32) norm_back_kernel<T, 32, 8><<<slots, 256, 0, st>>>(a);
        else if (s.tpr == 64) norm_back_kernel<T, 64, 8><<<slots, 256, 0, st>>>(a);
        else if (s.tpr == 128) norm_back_kernel<T, 128, 8><<<slots, 128, 0, st>>>(a);
        else if (s.tpr == 256) norm_back_kernel<T, 256, 8><<<slots, 256, 0, st>>>(a);
        else if (s.tpr == 384) norm_back_kernel<T, 384, 8><<<slots, 384, 0, st>>>(a);
        else if (s.tpr == 512) norm_back_kernel<T, 512, 8><<<slots, 512, 0, st>>>(a);
        else if (s.tpr == 768) norm_back_kernel<T, 768, 8><<<slots, 768, 0, st>>>(a);
        else if (s.tpr == 1024 && s.fpt == 8)
            norm_back_kernel<T, 1024, 8><<<slots, 1024, 0, st>>>(a);
        else if (s.tpr == 1024) norm_back_kernel<T, 1024, 16><<<slots, 1024, 0, st>>>(a);
        else {
            // dw first: dx may take dout's place
            const dim3 grid((unsigned)((a.width + 255) / 256), slots);
            norm_back_long_weight_kernel<T><<<grid, 256, 0, st>>>(a);
            const hipError_t e = back_long_rows<T>(a, st);
            if (e != hipSuccess) return e;
        }
    }
    norm_weight_kernel<<<(a.width + 31) / 32, 1024, 0, st>>>(a.part, slots, a.width, a.dw);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(int dtype, bool held, const NormArgs &a, hipStream_t st)
{
    if (dtype == KR_F32) return held ? norm_typed<float, true>(a, st) : norm_typed<float, false>(a, st);
    if (dtype == KR_F16) return held ? norm_typed<f16, true>(a, st) : norm_typed<f16, false>(a, st);
    return held ? norm_typed<bf16, true>(a, st) : norm_typed<bf16, false>(a, st);
}

int norm_back_slots(int, int64_t rows, int width)
{
    if (rows <= 0) return 0;
    const Shape s = shape_of(width);
    const int rpb = rows_per_block(s);
    // 12 to 16 waves a CU: enough loads in flight, and the shares of dw, written once and read
    // once, stay a few per cent of the traffic
    const int most = s.tpr == 0 ? 64 : s.tpr == 128 ? 2048 : s.tpr <= 256 ? 1024 : s.tpr <= 512 ? 512 : 256;
    const int64_t blocks = (rows + rpb - 1) / rpb;
    return (int)(blocks < most ? blocks : most);
}

hipError_t launch_norm_back(int dtype, const NormBackArgs &a, hipStream_t st)
{
    const int slots = norm_back_slots(dtype, a.rows, a.width);
    if (dtype == KR_F32) return back_typed<float>(a, slots, st);
    if (dtype == KR_F16) return back_typed<f16>(a, slots, st);
    return back_typed<bf16>(a, slots, st);
}

}  // namespace kr
