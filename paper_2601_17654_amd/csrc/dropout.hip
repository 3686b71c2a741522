// Dropout: out = kept x / (1 - p) (+ residual), the mask computed from counters (kr_drop.h) and stored
// nowhere; of a gradient the same call gives the gradient.  A thread takes eight neighbours, whose random
// bits come of one counter.
//
// Bound by memory: 8192 x 14336 in bfloat16 81 us (5.8 TB/s of its 470 MB), in float32 161 us (5.9 TB/s);
// with a residual 120 and 243 us (5.9, 5.8 TB/s).
#include "kr_drop.h"
#include "kr_rows.h"

namespace kr {

namespace {

template <typename T, bool RES, bool DROP>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, Dealt s)
{
    constexpr int V = kVec<T>, NV = kDropGroup / V;
    const int64_t block = blockIdx.x / s.chunks;
    const uint32_t chunk = blockIdx.x - (uint32_t)block * s.chunks;
    const int64_t row = (block << (8 - s.log_tpr)) + (threadIdx.x >> s.log_tpr);
    const uint32_t group = (chunk << s.log_tpr) + (threadIdx.x & ((1u << s.log_tpr) - 1));
    if (row >= a.rows || group >= s.groups) return;
    const int c = (int)group * kDropGroup, width = (int)a.width;
    const T *x = (const T *)a.x + row * a.ldx;
    Pack<T, V> xs[NV], rs[NV];
    float v[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) xs[j] = load_row(x, c + j * V, width);
    if (RES) {
        const T *r = (const T *)a.res + row * a.ldr;
#pragma unroll
        for (int j = 0; j < NV; ++j) rs[j] = load_row(r, c + j * V, width);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) floats(xs[j], v[j]);
    if (DROP) {
        const DropWords w =
            drop_words(a.drop, drop_seed(a.drop), group, (uint32_t)(a.row0 + row));
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e)
                v[j][e] = w.bits(j * V + e) >= a.drop.cut ? v[j][e] * a.drop.factor : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (RES) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[j][e] += (float)rs[j].v[e];
        }
        store_row((T *)a.out + row * a.ldo, c + j * V, width, v[j]);
    }
}

template <typename T>
hipError_t typed(DropoutArgs a, hipStream_t st)
{
    const Dealt s = dealt((a.width + kDropGroup - 1) / kDropGroup);
    const int64_t most = dealt_rows(s), rows = a.rows;
    for (int64_t done = 0; done < rows; done += most) {
        a.rows = std::min(most, rows - done);
        const unsigned blocks = (unsigned)dealt_blocks(s, a.rows);
        if (a.res && a.drop.cut) dropout_kernel<T, true, true><<<blocks, 256, 0, st>>>(a, s);
        else if (a.res) dropout_kernel<T, true, false><<<blocks, 256, 0, st>>>(a, s);
        else if (a.drop.cut) dropout_kernel<T, false, true><<<blocks, 256, 0, st>>>(a, s);
        else dropout_kernel<T, false, false><<<blocks, 256, 0, st>>>(a, s);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        a.x = (const T *)a.x + a.rows * a.ldx;
        if (a.res) a.res = (const T *)a.res + a.rows * a.ldr;
        a.out = (T *)a.out + a.rows * a.ldo;
        a.row0 += a.rows;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_dropout(int dtype, const DropoutArgs &a, hipStream_t st)
{
    if (dtype == KR_F32) return typed<float>(a, st);
    if (dtype == KR_F16) return typed<f16>(a, st);
    return typed<bf16>(a, st);
}

}  // namespace kr
