// Layer norm with the residual's addition and dropout of the branch, forward and backward.
//
//   s = r + D(x),  m = mean(s),  f = 1 / sqrt(mean((s - m)^2) + eps),  n = (s - m) f w + b
//
// A row stays in the registers of the threads that share it, so that each element is read once and
// written once, and the variance is that of the differences from the mean: no sum of squares
// from which a square is taken.  Rows of more than 16,384 elements are read again from memory
// instead: three times forward, twice backward and once more for the sums over rows.
// All arithmetic is in 32 bits; stored values are rounded once.
//
// Bound by memory.  16384 x 4096 in bfloat16: forward 97 us (5.6 TB/s of its 537 MB), with dropout 103;
// backward 107 us (5.0 TB/s), with dropout, which writes a gradient more, 138 (4.9 TB/s).  What that took
// of the backward pass was registers: with 129 of them a CU held one block of 512 threads (254 us).
// Rows of whole vectors (the WHOLE forms) need no shifts, the waves' sums are joined in lanes, and
// loaded values are converted twice.  Wide rows, forward and backward, without dropout: 4096 x 16384 in
// bfloat16 107 and 136 us, in float32 196 and 245 us; 2048 x 28672 in bfloat16 145 and 194 us.  Odd rows
// start at odd places: 24000 x 2057 in float32 154 and 168 us (5.1, 4.7 TB/s), in bfloat16, whose vectors
// then straddle words, 125 and 177 us (3.2, 2.2 TB/s).
#include "kr_drop.h"
#include "kr_rows.h"

namespace kr {

namespace {

// x of the lane that is N before in its 16, in a ring.
template <int N>
__device__ inline float ring(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xF, 0xF, true));
}

// Sum over groups of 16 lanes, in every one of them; the pairs are the same seen from either, so
// that all have the same bits.
__device__ inline float sum16(float x)
{
    x += ring<8>(x);
    x += ring<4>(x);
    x += ring<2>(x);
    return x + ring<1>(x);
}

// Sums over the TPR threads that share a row, in an order of its own: 16 lanes, those of a wave, then
// the waves' by 16 lanes again (read one by one, 16 waves' pairs of sums take 32 registers at once).
// `part`: as row_sum's.
template <int TPR, int N>
__device__ inline void row_sums(float (&x)[N], float (*part)[N])
{
#pragma unroll
    for (int n = 0; n < N; ++n) {
        x[n] = sum16(x[n]);
        if (TPR > 16) x[n] += __shfl_xor(x[n], 16);
        if (TPR > 32) x[n] += __shfl_xor(x[n], 32);
    }
    if (TPR <= 64) return;
    const int lane = threadIdx.x & 63;
    if (lane == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n) part[threadIdx.x >> 6][n] = x[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = sum16(lane % 16 < TPR / 64 ? part[lane % 16][n] : 0.0f);
}

template <typename T, int TPR, int FPT, bool DROP, bool WHOLE>
__global__ __launch_bounds__(kBlock<TPR>) void layer_norm_kernel(LayerNormArgs a)
{
    constexpr int V = kVec<T>, NV = FPT / V, RPB = kBlock<TPR> / TPR;
    __shared__ float part[2][TPR > 64 ? TPR / 64 : 1][1];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (RPB > 1 && row >= a.rows) return;  // whole rows' threads, and such rows take no barrier
    const T *x = (const T *)a.x + row * a.ldx;
    const T *r = a.res ? (const T *)a.res + row * a.ldr : nullptr;
    float s[NV][V];
    Pack<T, V> xs[NV], rs[NV], ws[NV], bs[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) xs[j] = load_part<WHOLE>(x, (j * TPR + t) * V, a.width);
    if (r) {
#pragma unroll
        for (int j = 0; j < NV; ++j) rs[j] = load_part<WHOLE>(r, (j * TPR + t) * V, a.width);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) ws[j] = load_part<WHOLE>((const T *)a.w, (j * TPR + t) * V, a.width);
    if (a.b) {
#pragma unroll
        for (int j = 0; j < NV; ++j) bs[j] = load_part<WHOLE>((const T *)a.b, (j * TPR + t) * V, a.width);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) floats(xs[j], s[j]);
    if (DROP) {
        const uint64_t seed = drop_seed(a.drop);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            drop_out<V>(a.drop, seed, (j * TPR + t) * V, (uint32_t)(a.row0 + row), s[j]);
    }
    if (r) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) s[j][e] += (float)rs[j].v[e];
    }
    if (a.sum) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            store_part<WHOLE>((T *)a.sum + row * a.lds, (j * TPR + t) * V, a.width, s[j]);
    }
    float total[1] = {}, squares[1] = {};  // past the row's end there are zeros
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) total[0] += s[j][e];
    row_sums<TPR>(total, part[0]);
    const float m = total[0] / (float)a.width;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s[j][e] = (j * TPR + t) * V + (WHOLE ? 0 : e) < a.width ? s[j][e] - m : 0.0f;
            squares[0] = fmaf(s[j][e], s[j][e], squares[0]);
        }
    row_sums<TPR>(squares, part[1]);
    const float f = 1.0f / sqrtf(squares[0] / (float)a.width + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[row] = m;
        if (a.rstd) a.rstd[row] = f;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s[j][e] = s[j][e] * f * (float)ws[j].v[e];
            if (a.b) s[j][e] += (float)bs[j].v[e];
        }
        store_part<WHOLE>((T *)a.out + row * a.ldo, (j * TPR + t) * V, a.width, s[j]);
    }
}

// Rows of any length.  Each thread writes an element after its last read of it.
template <typename T, bool DROP>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(LayerNormArgs a)
{
    constexpr int V = kVec<T>, STEP = 1024 * V;
    __shared__ float part[2][16];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *x = (const T *)a.x + row * a.ldx;
    const T *r = a.res ? (const T *)a.res + row * a.ldr : nullptr;
    const uint64_t seed = DROP ? drop_seed(a.drop) : 0;
    auto load = [&](int64_t c, float *s) {
        floats(load_row(x, (int)c, a.width), s);
        if (DROP) drop_out<V>(a.drop, seed, (int)c, (uint32_t)(a.row0 + row), s);
        if (r) {
            const Pack<T, V> b = load_row(r, (int)c, a.width);
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] += (float)b.v[e];
        }
    };
    float total = 0.0f, squares = 0.0f, s[V];
    for (int64_t c = t * V; c < a.width; c += STEP) {
        load(c, s);
#pragma unroll
        for (int e = 0; e < V; ++e) total += s[e];
    }
    const float m = row_sum<1024>(total, part[0]) / (float)a.width;
    for (int64_t c = t * V; c < a.width; c += STEP) {
        load(c, s);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = c + e < a.width ? s[e] - m : 0.0f;
            squares = fmaf(d, d, squares);
        }
    }
    const float f = 1.0f / sqrtf(row_sum<1024>(squares, part[1]) / (float)a.width + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[row] = m;
        if (a.rstd) a.rstd[row] = f;
    }
    for (int64_t c = t * V; c < a.width; c += STEP) {
        load(c, s);
        float n[V], b[V];
        const Pack<T, V> w = load_row((const T *)a.w, (int)c, a.width);
        if (a.b) {
            floats(load_row((const T *)a.b, (int)c, a.width), b);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) b[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) n[e] = (s[e] - m) * f * (float)w.v[e] + b[e];
        if (a.sum) store_row((T *)a.sum + row * a.lds, (int)c, a.width, s);
        store_row((T *)a.out + row * a.ldo, (int)c, a.width, n);
    }
}

// Gradients, with h = (s - m) f, g = dn w:  ds = f (g - mean(g) - h mean(g h)) + dsum,
// dx = D(ds),  dw = sum dn h,  db = sum dn.
// A block takes rows in turn and keeps its shares of dw and db in registers; the blocks' shares
// are added by layer_norm_weight_kernel in a fixed order.
template <typename T, int TPR, int FPT, bool DROP, bool WHOLE>
__global__ __launch_bounds__(kBlock<TPR>) __attribute__((amdgpu_waves_per_eu(4))) void
layer_norm_back_kernel(LayerNormBackArgs a)
{
    constexpr int V = kVec<T>, NV = FPT / V, RPB = kBlock<TPR> / TPR;
    // the next row's loads: with 16, or with dropout between odd rows in 32 bits, there are no
    // registers left
    constexpr bool AHEAD = FPT == 8 && (WHOLE || !DROP || sizeof(T) == 2);
    __shared__ float part[2][TPR > 64 ? TPR / 64 : 1][2];
    __shared__ float share[RPB > 1 ? RPB * TPR * FPT : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const uint64_t seed = DROP ? drop_seed(a.drop) : 0;
    float dw[NV][V], db[NV][V];
    Pack<T, V> ws[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        ws[j] = load_part<WHOLE>((const T *)a.w, (j * TPR + t) * V, a.width);
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = db[j][e] = 0.0f;
    }
    Pack<T, V> hs[NV], gs[NV], ds[NV];
    float m = 0.0f, f = 0.0f;
    auto load = [&](int64_t row) {  // of the next row, while one is worked on
        m = a.mean[row];
        f = a.rstd[row];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            hs[j] = load_part<WHOLE>((const T *)a.s + row * a.lds, (j * TPR + t) * V, a.width);
            gs[j] = load_part<WHOLE>((const T *)a.dout + row * a.ldo, (j * TPR + t) * V, a.width);
            if (a.dsum)
                ds[j] = load_part<WHOLE>((const T *)a.dsum + row * a.ldd, (j * TPR + t) * V, a.width);
        }
    };
    int turn = 0;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + sub;
    if (AHEAD && row < a.rows) load(row);
    for (; row < a.rows; row += stride, turn ^= 1) {
        if (!AHEAD) load(row);
        Pack<T, V> hn[NV], gn[NV], dn[NV];
        const float m0 = m, f0 = f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            hn[j] = hs[j];
            gn[j] = gs[j];
            dn[j] = ds[j];
        }
        if (AHEAD && row + stride < a.rows) load(row + stride);
        float c[2] = {};  // past the row's end g is 0
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float h = ((float)hn[j].v[e] - m0) * f0, g = (float)gn[j].v[e];
                dw[j][e] = fmaf(g, h, dw[j][e]);
                db[j][e] += g;
                const float gw = g * (float)ws[j].v[e];
                c[0] += gw;
                c[1] = fmaf(gw, (j * TPR + t) * V + (WHOLE ? 0 : e) < a.width ? h : 0.0f, c[1]);
            }
            if (FPT == 16) __builtin_amdgcn_sched_barrier(0);  // a vector at a time: registers
        }
        // two sets of words in turn: one barrier a row keeps a set until all have read it
        row_sums<TPR>(c, part[turn]);
        c[0] /= (float)a.width;
        c[1] /= (float)a.width;
        // what was loaded is converted again: kept in 32 bits it would take twice the registers
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            anew(hn[j]);
            anew(gn[j]);
            float d[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float h = ((float)hn[j].v[e] - m0) * f0, g = (float)gn[j].v[e] * (float)ws[j].v[e];
                d[e] = (a.dsum ? (float)dn[j].v[e] : 0.0f) + (g - c[0] - h * c[1]) * f0;
            }
            store_part<WHOLE>((T *)a.dres + row * a.ldr, (j * TPR + t) * V, a.width, d);
            if (DROP) {
                drop_out<V>(a.drop, seed, (j * TPR + t) * V, (uint32_t)(a.row0 + row), d);
                store_part<WHOLE>((T *)a.dx + row * a.ldx, (j * TPR + t) * V, a.width, d);
            }
            if (FPT == 16) __builtin_amdgcn_sched_barrier(0);
        }
    }
    float *slot = a.part + (int64_t)blockIdx.x * 2 * a.width;
    if (RPB > 1) {  // the block's rows side by side: their shares in turn
#pragma unroll
        for (int what = 0; what < 2; ++what) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    share[sub * TPR * FPT + (j * TPR + t) * V + e] = what ? db[j][e] : dw[j][e];
            __syncthreads();
            for (int c = threadIdx.x; c < a.width; c += 256) {
                float x = 0.0f;
#pragma unroll
                for (int k = 0; k < RPB; ++k) x += share[k * TPR * FPT + c];
                slot[(int64_t)what * a.width + c] = x;
            }
            __syncthreads();
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; e += kVec<float>) {
                store_row(slot, (j * TPR + t) * V + e, a.width, dw[j] + e);
                store_row(slot + a.width, (j * TPR + t) * V + e, a.width, db[j] + e);
            }
        (void)share;
    }
}

// Rows of any length: one block a row, read twice.
template <typename T, bool DROP>
__global__ __launch_bounds__(1024) void layer_norm_back_long_kernel(LayerNormBackArgs a)
{
    constexpr int V = kVec<T>, STEP = 1024 * V;
    __shared__ float part[16][2];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const uint64_t seed = DROP ? drop_seed(a.drop) : 0;
    const float m = a.mean[row], f = a.rstd[row];
    const T *sr = (const T *)a.s + row * a.lds, *gr = (const T *)a.dout + row * a.ldo;
    float c[2] = {}, h[V], g[V], w[V];
    auto load = [&](int64_t k) {
        floats(load_row(sr, (int)k, a.width), h);
        floats(load_row(gr, (int)k, a.width), g);
        floats(load_row((const T *)a.w, (int)k, a.width), w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            h[e] = k + e < a.width ? (h[e] - m) * f : 0.0f;
            g[e] *= w[e];
        }
    };
    for (int64_t k = t * V; k < a.width; k += STEP) {
        load(k);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            c[0] += g[e];
            c[1] = fmaf(g[e], h[e], c[1]);
        }
    }
    row_sums<1024>(c, part);
    c[0] /= (float)a.width;
    c[1] /= (float)a.width;
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
        for (int e = 0; e < V; ++e) d[e] += (g[e] - c[0] - h[e] * c[1]) * f;
        store_row((T *)a.dres + row * a.ldr, (int)k, a.width, d);
        if (DROP) {
            drop_out<V>(a.drop, seed, (int)k, (uint32_t)(a.row0 + row), d);
            store_row((T *)a.dx + row * a.ldx, (int)k, a.width, d);
        }
    }
}

// Their dw and db: 256 columns and every gridDim.y-th row a block.
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_back_long_weight_kernel(LayerNormBackArgs a)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.width) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float g = (float)((const T *)a.dout)[row * a.ldo + c];
        dw = fmaf(g, ((float)((const T *)a.s)[row * a.lds + c] - a.mean[row]) * a.rstd[row], dw);
        db += g;
    }
    float *slot = a.part + (int64_t)blockIdx.y * 2 * a.width;
    slot[c] = dw;
    slot[a.width + c] = db;
}

// dw and db = sums of the slots: 32 columns a block, 32 half waves that take every 32nd slot.
__global__ __launch_bounds__(1024) void layer_norm_weight_kernel(const float *part, int slots,
                                                                 int64_t width, float *dw, float *db)
{
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane, both = 2 * width;
    float s = 0.0f;
    if (c < both) {
#pragma unroll 8
        for (int k = group; k < slots; k += 32) s += part[k * both + c];
    }
    sums[group][lane] = s;
    __syncthreads();
    if (group == 0 && c < both) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s += sums[k][lane];
        if (c < width) dw[c] = s;
        else if (db) db[c - width] = s;
    }
}

template <typename T, bool DROP>
hipError_t typed(LayerNormArgs a, hipStream_t st)
{
    const Shape s = shape_of(a.width);
    const int rpb = rows_per_block(s);
    const int64_t rows = a.rows;
    for (int64_t done = 0; done < rows; done += kRowsPerLaunch) {
        a.rows = rows - done < kRowsPerLaunch ? rows - done : kRowsPerLaunch;
        const unsigned grid = (unsigned)((a.rows + rpb - 1) / rpb);
        if (!with_shape(s, [&](auto tpr, auto fpt) {
                constexpr int TPR = decltype(tpr)::value, FPT = decltype(fpt)::value;
                if (a.width % kVec<T> == 0)
                    layer_norm_kernel<T, TPR, FPT, DROP, true><<<grid, kBlock<TPR>, 0, st>>>(a);
                else
                    layer_norm_kernel<T, TPR, FPT, DROP, false><<<grid, kBlock<TPR>, 0, st>>>(a);
            }))
            layer_norm_long_kernel<T, DROP><<<grid, 1024, 0, st>>>(a);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        a.x = (const T *)a.x + a.rows * a.ldx;
        if (a.res) a.res = (const T *)a.res + a.rows * a.ldr;
        if (a.sum) a.sum = (T *)a.sum + a.rows * a.lds;
        a.out = (T *)a.out + a.rows * a.ldo;
        if (a.mean) a.mean += a.rows;
        if (a.rstd) a.rstd += a.rows;
        a.row0 += a.rows;
    }
    return hipSuccess;
}

template <typename T, bool DROP>
hipError_t back_long(LayerNormBackArgs a, int slots, hipStream_t st)
{
    // dw and db first: an output may take dout's place
    const dim3 grid((unsigned)((a.width + 255) / 256), slots);
    layer_norm_back_long_weight_kernel<T><<<grid, 256, 0, st>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int64_t rows = a.rows;
    for (int64_t done = 0; done < rows; done += kRowsPerLaunch) {
        a.rows = rows - done < kRowsPerLaunch ? rows - done : kRowsPerLaunch;
        layer_norm_back_long_kernel<T, DROP><<<(unsigned)a.rows, 1024, 0, st>>>(a);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        a.s = (const T *)a.s + a.rows * a.lds;
        a.dout = (const T *)a.dout + a.rows * a.ldo;
        if (a.dsum) a.dsum = (const T *)a.dsum + a.rows * a.ldd;
        a.dres = (T *)a.dres + a.rows * a.ldr;
        if (DROP) a.dx = (T *)a.dx + a.rows * a.ldx;
        a.mean += a.rows;
        a.rstd += a.rows;
        a.row0 += a.rows;
    }
    return hipSuccess;
}

template <typename T, bool DROP>
hipError_t back_typed(const LayerNormBackArgs &a, hipStream_t st)
{
    const int slots = layer_norm_back_slots(a.rows, a.width);
    if (a.rows > 0) {
        hipError_t e = hipSuccess;
        if (!with_shape(shape_of(a.width), [&](auto tpr, auto fpt) {
                constexpr int TPR = decltype(tpr)::value, FPT = decltype(fpt)::value;
                if (a.width % kVec<T> == 0)
                    layer_norm_back_kernel<T, TPR, FPT, DROP, true><<<slots, kBlock<TPR>, 0, st>>>(a);
                else
                    layer_norm_back_kernel<T, TPR, FPT, DROP, false><<<slots, kBlock<TPR>, 0, st>>>(a);
                e = hipGetLastError();
            }))
            e = back_long<T, DROP>(a, slots, st);
        if (e != hipSuccess) return e;
    }
    const int64_t columns = a.db ? 2 * (int64_t)a.width : a.width;
    layer_norm_weight_kernel<<<(unsigned)((columns + 31) / 32), 1024, 0, st>>>(a.part, slots, a.width,
                                                                              a.dw, a.db);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_norm(int dtype, const LayerNormArgs &a, hipStream_t st)
{
    const bool drop = a.drop.cut != 0;
    if (dtype == KR_F32) return drop ? typed<float, true>(a, st) : typed<float, false>(a, st);
    if (dtype == KR_F16) return drop ? typed<f16, true>(a, st) : typed<f16, false>(a, st);
    return drop ? typed<bf16, true>(a, st) : typed<bf16, false>(a, st);
}

int layer_norm_back_slots(int64_t rows, int width)
{
    if (rows <= 0) return 0;
    const Shape s = shape_of(width);
    const int rpb = rows_per_block(s);
    const int most = s.tpr == 0 ? 64 : s.tpr == 128 ? 2048 : s.tpr <= 256 ? 1024 : s.tpr <= 512 ? 512 : 256;
    const int64_t blocks = (rows + rpb - 1) / rpb;
    return (int)(blocks < most ? blocks : most);
}

hipError_t launch_layer_norm_back(int dtype, const LayerNormBackArgs &a, hipStream_t st)
{
    const bool drop = a.dx != nullptr;
    if (dtype == KR_F32) return drop ? back_typed<float, true>(a, st) : back_typed<float, false>(a, st);
    if (dtype == KR_F16) return drop ? back_typed<f16, true>(a, st) : back_typed<f16, false>(a, st);
    return drop ? back_typed<bf16, true>(a, st) : back_typed<bf16, false>(a, st);
}

}  // namespace kr
