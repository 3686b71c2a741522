// Dropout's random numbers: counter based, so that a mask is computed again where it is needed and
// stored nowhere.
#pragma once

#include <algorithm>
#include <cmath>

#include "kr_block.h"

namespace kr {

// Value (row, c) is kept where its 16 bits, number c % 8 of the eight in the words of
// Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) at the counter
// (c / 8, row, offset) under the key `seed`, are `cut` or more; kept values are taken times `factor`.
// Sixteen bits a value: the ten rounds (20 products of 32 x 32 bits, each at a quarter of the
// rate, and 40 exclusive ors) cost eight values a lane some 480 cycles a wave: 67 million values 26 us of the
// chip's vector units, a quarter of what their memory takes in a norm.  With 32 bits a value it would be half,
// and dropout alone of a 16-bit tensor would wait for them.
struct Drop {
    uint64_t seed, offset;
    const uint64_t *seed_at;  // read when the kernel runs, in place of seed; or null
    uint32_t cut;             // 0 .. 65536;  0: nothing is dropped
    float factor;
};

constexpr int kDropGroup = 8;

// Of a valid kr_drop, or none.
inline Drop drop_of(const kr_drop *d)
{
    Drop x{0, 0, nullptr, 0, 1.0f};
    if (!d) return x;
    x.seed = d->seed;
    x.offset = d->offset;
    x.seed_at = d->seed_at;
    x.cut = (uint32_t)std::nearbyint(d->p * 65536.0);
    x.factor = x.cut < 65536 ? (float)(65536.0 / (65536.0 - x.cut)) : 0.0f;
    return x;
}

// The key, once a thread.
__device__ inline uint64_t drop_seed(const Drop &d) { return d.seed_at ? *d.seed_at : d.seed; }

struct DropWords {
    uint32_t w[4];
    // Number e of the eight.
    __device__ uint32_t bits(int e) const { return e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu; }
};

__device__ inline DropWords drop_words(const Drop &d, uint64_t seed, uint32_t group, uint32_t row)
{
    uint32_t c0 = group, c1 = row, c2 = (uint32_t)d.offset, c3 = (uint32_t)(d.offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {c0, c1, c2, c3};
}

// x[0 .. V - 1], values c .. c + V - 1 of a row (c a multiple of V, V of 4 or 8), dropped out.
template <int V>
__device__ inline void drop_out(const Drop &d, uint64_t seed, int c, uint32_t row, float *x)
{
    static_assert(kDropGroup % V == 0, "a vector lies in one group");
    const DropWords w = drop_words(d, seed, (uint32_t)c / kDropGroup, row);
    const bool upper = V < kDropGroup && c % kDropGroup;
    const uint32_t w0 = upper ? w.w[2] : w.w[0], w1 = upper ? w.w[3] : w.w[1];
    const DropWords mine{w0, w1, w.w[2], w.w[3]};
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = mine.bits(e) >= d.cut ? x[e] * d.factor : 0.0f;
}

// dropout.hip
struct DropoutArgs {
    int64_t rows;
    int64_t width;
    const void *x, *res;  // res: added to what is kept, or null
    void *out;
    int64_t ldx, ldr, ldo;
    int64_t row0;         // of the first row, in the counters
    Drop drop;
};
hipError_t launch_dropout(int dtype, const DropoutArgs &a, hipStream_t st);

// layer_norm.hip
struct LayerNormArgs {
    int64_t rows;
    int width;
    const void *x, *res, *w, *b;
    int64_t ldx, ldr;
    float eps;
    void *sum, *out;
    int64_t lds, ldo;
    float *mean, *rstd;
    int64_t row0;
    Drop drop;
};
hipError_t launch_layer_norm(int dtype, const LayerNormArgs &a, hipStream_t st);

struct LayerNormBackArgs {
    int64_t rows;
    int width;
    const void *s, *w, *dout, *dsum;
    int64_t lds, ldo, ldd;
    const float *mean, *rstd;
    void *dres, *dx;  // gradients of the residual and, dropped out, of x; dx null: the same
    int64_t ldr, ldx;
    float *dw, *db;
    float *part;  // [layer_norm_back_slots][2][width]
    int64_t row0;
    Drop drop;
};
int layer_norm_back_slots(int64_t rows, int width);
hipError_t launch_layer_norm_back(int dtype, const LayerNormBackArgs &a, hipStream_t st);

}  // namespace kr
