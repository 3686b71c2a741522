// Product of values held in 8-bit floating point (kr_scaled.h):
//   y[m][n] = sum over blocks b of 2^(ea[m][b] + eb[n][b]) sum over k in b of a[m][k] b[n][k]
// For outputs of 16 bits the matrix cores' 8-bit instruction takes 128 of k, which is one block: the
// scales are two of its operands, and the sums never leave its 32-bit accumulators.
//
// How it adds (measured, lane by lane): eight neighbouring products are brought to the exponent of
// the largest, what lies 2^-13 of it or less is cut off, and such sums are added in 32 bits.  A result
// is then off by up to 2^-10 of its terms' magnitudes, and measured by 1.5e-5 relative (5e-5 where
// neighbours differ by powers of two up to 2^10); a 16-bit output's rounding alone is up to 4.9e-4 or
// 3.9e-3.  Outputs of 32 bits take the values to bfloat16, which holds them and their scales exactly,
// and the instruction of that type, whose sums are off by 1e-7 (8192^3: 944 us, against 381).
#include <algorithm>

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

// Few rows (up to 16), out of the weights as they lie in memory: as few_kernel, 128 bytes of k of 16
// rows a wave and step.  (From 17 rows on tiles are faster: 32 x 8192 x 8192 17.8 us, 26.4 with two groups of
// 16 rows here.)
template <int NW, typename T>
__global__ __launch_bounds__(NW * 64) void scaled_few_kernel(ScaledArgs a)
{
    typedef Values<sizeof(T) == 4> V;
    __shared__ __align__(16) float sums[NW][16][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane % 16, part = lane / 16 * 32;
    // an XCD (every eighth block) takes neighbouring rows: eight groups of 16 share a line of scales
    const int id = (int)blockIdx.x, all = (int)gridDim.x, xcd = id & 7;
    const int64_t n0 = (int64_t)(xcd * (all >> 3) + min(xcd, all & 7) + (id >> 3)) * 16;
    // rows past the last take its place: their sums are not put
    const int64_t wn = n0 + r < a.n ? n0 + r : a.n - 1, xm = r < a.m ? r : a.m - 1;
    const char *w = a.b.q + wn * a.b.ld, *x = a.a.q + xm * a.a.ld;
    const uint8_t *ws = a.b.scale + scale_place(wn), *xs = a.a.scale + scale_place(xm);
    f32x4 acc{0, 0, 0, 0};
    // the steps that are whole, some at a time: all of their loads are in flight at once
    constexpr int AHEAD = 4;
    const int whole = (int)(a.k / kScaled), steps = (int)((a.k + kScaled - 1) / kScaled);
    struct Raw {
        Pack<char, 16> v[2];
    };
    int s = wave;
    for (; s + (AHEAD - 1) * NW < whole; s += AHEAD * NW) {
        Raw fw[AHEAD], fx[AHEAD];
        int sw[AHEAD], sx[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t b = s + u * NW;
            const int c = (int)b * kScaled + part;
            fw[u] = Raw{{load16(w + c), load16(w + c + 16)}};
            sw[u] = ws[b * a.b.lds];
            fx[u] = Raw{{load16(x + c), load16(x + c + 16)}};
            sx[u] = xs[b * a.a.lds];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            acc = mma_values(V(__builtin_bit_cast(i32x8, fw[u]), sw[u]),
                             V(__builtin_bit_cast(i32x8, fx[u]), sx[u]), acc);
    }
    auto load = [&](const char *row, int c) {
        return __builtin_bit_cast(i32x8, Raw{{load_row(row, c, (int)a.k), load_row(row, c + 16, (int)a.k)}});
    };
#pragma unroll 1
    for (; s < steps; s += NW) {
        const int c = s * kScaled + part;
        acc = mma_values(V(load(w, c), ws[s * a.b.lds]), V(load(x, c), xs[s * a.a.lds]), acc);
    }
    *(f32x4 *)&sums[wave][r][lane / 16 * 4] = acc;
    __syncthreads();
    const int token = (int)threadIdx.x / 2, h = (int)threadIdx.x % 2 * 8;
    if (token >= a.m || n0 + h >= a.n) return;
    float v[8] = {};
#pragma unroll 4
    for (int k = 0; k < NW; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += sums[k][token][h + e];
    store8((T *)a.out + token * a.ldo, (int)n0 + h, (int)a.n, v);
}

// ---- tiles ---------------------------------------------------------------------------------

struct E4m3 {};  // of Mma: 32-bit sums

struct TileArgs {
    MmaArgs p;
    const uint8_t *scale[2];  // of a, of b
    int64_t lds[2];           // bytes from one block's to the next
    int64_t rows[2];          // of a block that may be read
};

// One product, or two whose blocks share a launch: those from `first` on are the second's.
template <typename Out>
struct Two {
    TileArgs a[2];
    Out out[2];
    uint32_t first;
};

// A block's copies to LDS: the operands' tiles as in mma_kernel, 16 bytes a lane, and the step's scale
// bytes, 4 a lane: the first wave those of a's tile, the second of b's, each to 256 bytes of its own (the
// others copy an empty buffer, so that every wave counts the same copies).
template <int BM, int BN, int NW>
struct Copies {
    typedef TileLoader<false, BM, NW> LoadA;
    typedef TileLoader<false, BN, NW> LoadB;
    static constexpr int N = LoadA::N + LoadB::N + 1;  // of a wave and step, the scales last
    struct Lds {
        char tile[2][(BM + BN) * kStep];
        uint8_t scale[2][NW][256];
    };
    LoadA la;
    LoadB lb;
    i32x4 ra, rb, rs;
    uint64_t at;       // of the step's scales
    int64_t ld;
    int records, k_left, step, end, wave;
    uint32_t lane4;

    __device__ void init(const TileArgs &a, int64_t m0, int64_t n0, int begin, int end_, int wave_,
                         int lane)
    {
        wave = wave_;
        step = begin;
        end = end_;
        la.init(a.p.a[0], m0, wave, lane, MapSame());
        lb.init(a.p.b[0], n0, wave, lane, MapSame());
        la.aim(begin, 0);
        lb.aim(begin, 0);
        const bool odd = wave & 1;
        const int64_t first = (odd ? n0 : m0) / kScaled * kScaled, left = (odd ? a.rows[1] : a.rows[0]) - first;
        ld = odd ? a.lds[1] : a.lds[0];
        at = (uint64_t)((odd ? a.scale[1] : a.scale[0]) + begin * ld + first);
        records = wave < 2 ? (int)(left < 256 ? left : 256) : 0;
        lane4 = lane * 4;
        k_left = (int)a.p.k_bytes - begin * kStep;
        la.bound(k_left);
        lb.bound(k_left);
        ra = la.buffer(begin < end);
        rb = lb.buffer(begin < end);
        scales();
    }
    __device__ void scales()
    {
        i32x4 x{(int)at, (int)(at >> 32) & 0xFFFF, step < end ? records : 0, 0x00020000};
        here(x);
        rs = x;
    }
    // Goes one step on, in eight parts that stand between matrix instructions.
    static constexpr int PARTS = 8;
    __device__ __attribute__((always_inline)) void part(int p)
    {
        if (p == 0) {
            ++step;
            here(step);
        }
        if (p == 1) la.next_at(false, 0);
        if (p == 2) la.next_rest(false);
        if (p == 3) ra = la.buffer(step < end);
        if (p == 4) {
            lb.next_at(false, 0);
            lb.next_rest(false);
        }
        if (p == 5) rb = lb.buffer(step < end);
        if (p == 6) {
            here(k_left);
            k_left -= kStep;
            la.bound(k_left);
            lb.bound(k_left);
        }
        if (p == 7) {
            here(at);
            at += ld;
            scales();
        }
    }
    __device__ uint32_t from(int j) const
    {
        return j < LoadA::N ? la.from(j) : j < N - 1 ? lb.from(j - LoadA::N) : lane4;
    }
    __device__ const char *to(int j, Lds &lds, int buf) const
    {
        if (j == N - 1) return (const char *)lds.scale[buf][wave];
        return j < LoadA::N ? la.to(j, lds.tile[buf], wave)
                            : lb.to(j - LoadA::N, lds.tile[buf] + BM * kStep, wave);
    }
    __device__ __attribute__((always_inline)) void go(int j, uint32_t off, uint32_t m0) const
    {
        if (j == N - 1)
            asm volatile("buffer_load_dword %0, %1, 0 offen lds" ::"v"(off), "s"(rs), "{m0}"(m0) : "memory");
        else
            copy_go(off, j < LoadA::N ? ra : rb, m0);
    }
    __device__ __attribute__((always_inline)) void all(Lds &lds, int buf) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t m0 = copy_ready(from(j), to(j, lds, buf));
            asm volatile("s_nop 0");
            go(j, from(j), m0);
        }
    }
};

// Scale bytes of a wave's 128 rows (tile t of 16 at byte t) or 64 (the half of 128 that is its).
template <int ROWS>
__device__ inline i32x2 read_scales(const uint8_t *scale, int part, int lane)
{
    if (ROWS == 128) return *(const i32x2 *)(scale + part * 128 + lane % 16 * 8);
    return i32x2{*(const int *)(scale + lane % 16 * 8 + part * 4), 0};
}

// c += a b with the scales in bytes SA of sa and SB of sb, in place as mma_in_place().
template <int SA, int SB>
__device__ inline void scaled_in_place(const i32x8 &a, const i32x8 &b, f32x4 &c, int sa, int sb)
{
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]"
                 : "+a"(c)
                 : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(SA & 1), "n"(SB & 1), "n"(SA >> 1), "n"(SB >> 1));
}

// When a step's work stands among its matrix instructions: reads one tile of 16 rows (two reads of
// LDS) each `apart` of them; from `free` on every wave has its step in registers, and the copies of the
// step after next go over it, those started before instruction x being copies(x); from `next` on the next
// step's tiles have arrived.
template <int BLOCK>
struct When;
template <>
struct When<64> {
    static constexpr int apart = 2, free = 20, next = 40;
    static constexpr int copies(int x)
    {
        return x <= free ? 0 : ((x - free) * 2 + 4) / 5 < 17 ? ((x - free) * 2 + 4) / 5 : 17;
    }
};
template <>
struct When<16> {
    static constexpr int apart = 1, free = 6, next = 10;
    static constexpr int copies(int x) { return x <= free ? 0 : x - free < 9 ? x - free : 9; }
};

// Two steps' tiles are in LDS, and the registers hold one step, no more: its sums take half of them
// already.  A step's products are four quarters, halves of a's rows by halves of b's, and the order of b's
// halves turns with each step (P), so that a half is overwritten by the next step's as soon as its last
// quarter is done, and is wanted again a quarter later at the soonest:
//   P = 0: a0 b0, a0 b1, a1 b1, a1 b0     P = 1: a0 b1, a0 b0, a1 b0, a1 b1
// In a step's first quarter come the reads of its second b half and of a1, from `next` on those of the next
// step's a0 and of its first b half.
template <int BM, int BN, typename Out>
__global__ __launch_bounds__(256) void scaled_tile_kernel(Two<Out> two)
{
    const bool second = blockIdx.x >= two.first;
    const TileArgs &a = two.a[second];
    const Out &out = two.out[second];
    const int block = (int)(second ? blockIdx.x - two.first : blockIdx.x);
    constexpr int WM = 2, WN = 2, RM = BM / WM, RN = BN / WN, TM = RM / 16, TN = RN / 16;
    constexpr int BLOCK = TM * TN, QUARTER = BLOCK / 4, HM = TM / 2, HN = TN / 2;
    typedef When<BLOCK> W;
    typedef Copies<BM, BN, 4> C;
    static_assert(HM == HN && W::free >= 2 * HM * W::apart && W::next >= 2 * QUARTER &&
                      W::next + HM * W::apart >= 3 * QUARTER && W::next + 2 * HM * W::apart <= BLOCK &&
                      2 * HM * W::apart <= QUARTER * 2 && HM * W::apart <= QUARTER &&
                      W::copies(BLOCK) == C::N,
                  "the reads and copies fit the step");
    __shared__ __align__(1024) typename C::Lds lds;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn, split;
    tile_of(a.p, block, &tm, &tn, &split);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int begin = split * a.p.per_split, end = min(begin + a.p.per_split, a.p.steps);

    C c;
    c.init(a, m0, n0, begin, end, wave, lane);
    TileReader<false, BM> reader;
    reader.init(lane);
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    i32x8 fa[TM], fb[TN];
    i32x2 sa[2], sb[2];
    auto tile = [&](const char *at, int first) __attribute__((always_inline)) {
        return __builtin_shufflevector(reader.read(at, first, 0), reader.read(at, first, 1), 0, 1, 2, 3, 4,
                                       5, 6, 7);
    };
    auto read_a = [&](int buf, int i) __attribute__((always_inline)) {
        fa[i] = tile(lds.tile[buf], wm * RM + i * 16);
    };
    auto read_b = [&](int buf, int j) __attribute__((always_inline)) {
        fb[j] = tile(lds.tile[buf] + BM * kStep, wn * RN + j * 16);
    };
    auto read_s = [&](int buf, int p) __attribute__((always_inline)) {
        sa[p] = read_scales<RM>(lds.scale[buf][0], wm, lane);
        sb[p] = read_scales<RN>(lds.scale[buf][1], wn, lane);
    };

    c.all(lds, 0);
#pragma unroll
    for (int p = 0; p < C::PARTS; ++p) c.part(p);
    c.all(lds, 1);
    arrived<C::N>();
    read_s(0, 0);
#pragma unroll
    for (int i = 0; i < HM; ++i) {
        read_a(0, i);
        read_b(0, i);
    }
    sums_done(acc);
    auto body = [&](auto parity) __attribute__((always_inline)) {
        constexpr int P = decltype(parity)::value;
        uint32_t off = 0, m0 = 0;
        each(Count<BLOCK>(), [&](auto at_x) __attribute__((always_inline)) {
            constexpr int x = decltype(at_x)::value, A = W::apart;
            if (x % A == 0 && x / A < HM) read_b(P, (1 - P) * HN + x / A);
            if (x % A == 0 && x / A >= HM && x / A < 2 * HM) read_a(P, x / A);
            if (x == W::free) read_done();
            if (x == W::next) arrived<W::copies(W::next)>();
#pragma unroll
            for (int p = 0; p < C::PARTS; ++p)
                if (p * W::free / C::PARTS == x) c.part(p);
            if (W::copies(x + 1) > W::copies(x)) c.go(W::copies(x), off, m0);
            if (x + 1 < BLOCK && W::copies(x + 2) > W::copies(x + 1)) {
                off = c.from(W::copies(x + 1));
                m0 = copy_ready(off, c.to(W::copies(x + 1), lds, P));
            }
            if (x >= W::next && (x - W::next) % A == 0) {
                constexpr int r = (x - W::next) / A;
                if (r == 0) read_s(1 - P, 1 - P);
                if (r < HM) read_a(1 - P, r);
                if (r >= HM && r < 2 * HM) read_b(1 - P, (1 - P) * HN + r - HM);
            }
            constexpr int q = x / QUARTER, y = x % QUARTER, ih = q / 2;
            constexpr int jh = q == 0 || q == 3 ? P : 1 - P;
            constexpr int jj = y / HM, ii = jj % 2 ? HM - 1 - y % HM : y % HM;  // to and fro
            constexpr int i = ih * HM + ii, j = jh * HN + jj;
            scaled_in_place<j % 4, i % 4>(fb[j], fa[i], acc[i][j], sb[P][j / 4], sa[P][i / 4]);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    int s = begin;
    for (; s + 1 < end; s += 2) {
        body(std::integral_constant<int, 0>());
        body(std::integral_constant<int, 1>());
    }
    if (s < end) body(std::integral_constant<int, 0>());
    sums_done(acc);
    read_done();
    arrived<0>();  // the tiles' LDS is free, and no copy will write to it
    put_tile<BM, BN, WM, WN>(E4m3(), a.p, out, acc, lds.tile[0], m0, n0, wave, split, lane);
}

// The same for outputs of 32 bits, in tiles of 128 x BN: a step's values go to bfloat16 on their way to the
// instructions, which the compiler places.  A lane's four sums are neighbours in a row and leave as they are.
template <int BN>
__global__ __launch_bounds__(256) void scaled_wide_kernel(Two<PutAs<float>> two)
{
    const bool second = blockIdx.x >= two.first;
    const TileArgs &a = two.a[second];
    float *out = two.out[second].out;
    int64_t ldo = two.out[second].ldo;
    const int block = (int)(second ? blockIdx.x - two.first : blockIdx.x);
    constexpr int BM = 128, WN = 2, TM = 4, TN = BN / WN / 16;
    typedef Copies<BM, BN, 4> C;
    __shared__ __align__(1024) typename C::Lds lds;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn, split;
    tile_of(a.p, block, &tm, &tn, &split);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int begin = split * a.p.per_split, end = min(begin + a.p.per_split, a.p.steps);
    C c;
    c.init(a, m0, n0, begin, end, wave, lane);
    TileReader<false, BM> reader;
    reader.init(lane);
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    auto tile = [&](const char *at, int first) __attribute__((always_inline)) {
        return __builtin_shufflevector(reader.read(at, first, 0), reader.read(at, first, 1), 0, 1, 2, 3, 4,
                                       5, 6, 7);
    };
    c.all(lds, 0);
#pragma unroll
    for (int p = 0; p < C::PARTS; ++p) c.part(p);
    c.all(lds, 1);
    for (int s = begin; s < end; ++s) {
        const int buf = (s - begin) & 1;
        arrived<C::N>();
        // of 16-row tiles, side by side; a tile of 64 rows of b is half of its 128
        const uint8_t *of_a = lds.scale[buf][0] + lane % 16 * 8 + wm * TM;
        const uint8_t *of_b = lds.scale[buf][1] + lane % 16 * 8 + n0 % kScaled / 16 + wn * TN;
        const uint32_t sa = *(const uint32_t *)of_a;
        const uint32_t sb = TN == 4 ? *(const uint32_t *)of_b : *(const uint16_t *)of_b;
        i32x8 qa[TM], qb[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) qa[i] = tile(lds.tile[buf], (wm * TM + i) * 16);
#pragma unroll
        for (int j = 0; j < TN; ++j) qb[j] = tile(lds.tile[buf] + BM * kStep, (wn * TN + j) * 16);
        read_done();
#pragma unroll
        for (int p = 0; p < C::PARTS; ++p) c.part(p);
        c.all(lds, buf);
        auto byte = [](uint32_t x, int t) { return (int)(x >> (8 * t) & 255); };
        const Values<true> va[TM] = {{qa[0], byte(sa, 0)}, {qa[1], byte(sa, 1)}, {qa[2], byte(sa, 2)},
                                     {qa[3], byte(sa, 3)}};
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const Values<true> vb(qb[j], byte(sb, j));
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[i][j] = mma(bf16(), vb.v[q], va[i].v[q], acc[i][j]);
        }
    }
    if (a.p.splits > 1) {
        out = a.p.part + (int64_t)split * a.p.m * a.p.n;
        ldo = a.p.n;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t m = m0 + (wm * TM + i) * 16 + lane % 16;
            const int n = (int)n0 + (wn * TN + j) * 16 + lane / 16 * 4;
            if (m < a.p.m) store_row(out + m * ldo, n, a.p.n, (const float *)&acc[i][j]);
        }
    arrived<0>();  // no copy is under way when the block's LDS is given up
}

// How a product is cut.  16-bit outputs: as the other products, whose steps take as long.  32-bit outputs:
// tiles of 128 x 128 or 128 x 64 and up to 16 splits of the sum, by an estimate in microseconds: 1.05 and
// 0.8 a step, a tile a CU at a time (two share the time), 5 around them, 5 for a split's join and its sums
// at 4 TB/s.  Measured, 128 x 128 / 128 x 64 at the splits in brackets: 333 x 5001 x 2059 26.3 / 21.0 us (1),
// 1000 x 4096 x 4096 46.5 / 49.3 (1), 32 x 8192 x 8192 26.4 (4) / 36.0 (2), 100 x 1000 x 16000 26.3 / 22.1 (8).
struct Plan {
    MmaPlan p;
    bool narrow;  // of 32-bit outputs: tiles of 128 x 64
};
Plan plan_of(int out_type, int64_t m, int64_t n, int steps)
{
    if (out_type != KR_F32) return {mma_plan(m, n, 1, steps), false};
    Plan best{};
    double least = 0;
    for (const bool narrow : {false, true}) {
        const int64_t tm = (m + 127) / 128, tn = narrow ? (n + 63) / 64 : (n + 127) / 128;
        for (int s = 1; s <= 16 && (s == 1 || (steps + s - 1) / s >= 4); ++s) {
            const int per = (steps + s - 1) / s;
            if ((steps + per - 1) / per != s) continue;
            const int64_t part = s > 1 ? 4 * s * m * n : 0;
            const double cost = (tm * tn * s + 255) / 256 * per * (narrow ? 0.8 : 1.05) +
                                (s > 1 ? 5 + 2 * (double)part / 4e6 : 0);
            if (best.p.tiles_m && cost >= least) continue;
            least = cost;
            best = {{false, (int)tm, (int)tn, s, per, part}, narrow};
        }
    }
    return best;
}

TileArgs tile_args(const ScaledArgs &a, const MmaPlan &p)
{
    TileArgs x{};
    x.p.a[0] = Operand{a.a.q, a.a.ld, a.m, a.a.bytes};
    x.p.b[0] = Operand{a.b.q, a.b.ld, a.n, a.b.bytes};
    x.p.m = (int)a.m;
    x.p.n = (int)a.n;
    x.p.k_bytes = a.a.bytes;
    x.p.steps = (int)((a.k + kScaled - 1) / kScaled);
    x.p.pairs = 1;
    x.p.tiles_m = p.tiles_m;
    x.p.tiles_n = p.tiles_n;
    x.p.splits = p.splits;
    x.p.per_split = p.per_split;
    x.p.part = (float *)a.part;
    for (int i = 0; i < 2; ++i) {
        const HeldMatrix &h = i ? a.b : a.a;
        x.scale[i] = h.scale;
        x.lds[i] = h.lds;
        x.rows[i] = ((i ? a.n : a.m) + kScaled - 1) / kScaled * kScaled;
    }
    return x;
}

// b: null, or a second product whose plan has a's tile size.
template <typename T>
hipError_t tiles(const ScaledArgs &a, const Plan &pa, const ScaledArgs *b, const Plan *pb, hipStream_t st)
{
    typedef PutAs<T> Out;
    Two<Out> two{{tile_args(a, pa.p), {}}, {{(T *)a.out, a.ldo, (int)a.n}, {}}, 0};
    two.first = (uint32_t)(pa.p.tiles_m * pa.p.tiles_n * pa.p.splits);
    unsigned blocks = two.first;
    if (b) {
        two.a[1] = tile_args(*b, pb->p);
        two.out[1] = Out{(T *)b->out, b->ldo, (int)b->n};
        blocks += (unsigned)(pb->p.tiles_m * pb->p.tiles_n * pb->p.splits);
    }
    if constexpr (sizeof(T) == 4)
        pa.narrow ? scaled_wide_kernel<64><<<blocks, 256, 0, st>>>(two)
                  : scaled_wide_kernel<128><<<blocks, 256, 0, st>>>(two);
    else if (pa.p.large)
        scaled_tile_kernel<256, 256><<<blocks, 256, 0, st>>>(two);
    else
        scaled_tile_kernel<128, 128><<<blocks, 256, 0, st>>>(two);
    for (int i = 0; i < (b ? 2 : 1); ++i) {
        const MmaArgs &p = two.a[i].p;
        if (p.splits == 1) continue;
        const int64_t threads = (int64_t)p.m * ((p.n + 7) / 8);
        mma_join_kernel<E4m3><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(p, two.out[i]);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t one(const ScaledArgs &a, hipStream_t st)
{
    return tiles<T>(a, plan_of(a.out_type, a.m, a.n, (int)((a.k + kScaled - 1) / kScaled)), nullptr, nullptr, st);
}

// What one tile takes of the chip's 256 CUs, and by itself, in microseconds (of mma_plan and plan_of).
struct TileCost {
    double share, alone;
};
TileCost cost_of(const Plan &x, bool f32)
{
    const int per = x.p.per_split;
    if (f32) return {per * (x.narrow ? 0.8 : 1.05), per * (x.narrow ? 0.8 : 1.05) + 5};
    if (x.p.large) return {1.3 * per + 9, 1.3 * per + 9};
    return {0.47 * per + 2, 0.94 * per + 4};  // two a CU
}
int64_t blocks_of(const Plan &x) { return (int64_t)x.p.tiles_m * x.p.tiles_n * x.p.splits; }
double join_of(const Plan &x) { return x.p.splits > 1 ? 4 + 2 * (double)x.p.part_bytes / 4e6 : 0; }

// Both in one launch, whose tiles fill the chip together; alone, by rounds of 256.
double cost_together(const Plan &a, const Plan &b, bool f32)
{
    const TileCost x = cost_of(a, f32), y = cost_of(b, f32);
    const double all = (blocks_of(a) * x.share + blocks_of(b) * y.share) / 256;
    const double longest = std::max(x.alone, y.alone);
    return std::max(all + 0.5 * std::min(x.alone, y.alone), longest) + join_of(a) + join_of(b);
}
double cost_alone(const Plan &a, bool f32)
{
    return (blocks_of(a) + 255) / 256 * cost_of(a, f32).share + (f32 ? 5 : 0) + join_of(a);
}

// Tiles of one size, whole sums.
Plan plan_whole(int64_t m, int64_t n, int steps, bool f32, bool other)
{
    const int bm = !f32 && other ? 256 : 128, bn = f32 ? (other ? 64 : 128) : bm;
    return {{!f32 && other, (int)((m + bm - 1) / bm), (int)((n + bn - 1) / bn), 1, steps, 0}, f32 && other};
}

// Two products (a linear layer's gradients), whose sums differ in length: one launch where that is
// cheaper by the estimate, with their own plans or with whole sums in tiles of one size.  4917 x 5056 x 832,
// 400 large tiles of 7 steps and 273 small ones of 40: 86 us alone one after the other, 62 together.
template <typename T>
hipError_t pair(const ScaledArgs &a, const ScaledArgs &b, hipStream_t st)
{
    constexpr bool F32 = sizeof(T) == 4;
    const int sa = (int)((a.k + kScaled - 1) / kScaled), sb = (int)((b.k + kScaled - 1) / kScaled);
    const Plan pa = plan_of(a.out_type, a.m, a.n, sa), pb = plan_of(b.out_type, b.m, b.n, sb);
    Plan best[2] = {pa, pb};
    bool together = pa.p.large == pb.p.large && pa.narrow == pb.narrow;
    double least = together ? cost_together(pa, pb, F32) : cost_alone(pa, F32) + cost_alone(pb, F32) + 3;
    for (const bool other : {false, true}) {
        const Plan x = plan_whole(a.m, a.n, sa, F32, other), y = plan_whole(b.m, b.n, sb, F32, other);
        const double cost = cost_together(x, y, F32);
        if (cost >= least || blocks_of(x) + blocks_of(y) > 1 << 23) continue;
        least = cost;
        best[0] = x;
        best[1] = y;
        together = true;
    }
    if (!together || blocks_of(best[0]) + blocks_of(best[1]) > 1 << 23) {
        const hipError_t e = tiles<T>(a, best[0], nullptr, nullptr, st);
        return e == hipSuccess ? tiles<T>(b, best[1], nullptr, nullptr, st) : e;
    }
    // the longer sums first, so that the shorter ones fill the end
    return best[0].p.per_split >= best[1].p.per_split ? tiles<T>(a, best[0], &b, &best[1], st)
                                                      : tiles<T>(b, best[1], &a, &best[0], st);
}

template <typename T>
hipError_t few(const ScaledArgs &a, hipStream_t st)
{
    const unsigned blocks = (unsigned)((a.n + 15) / 16);
    // four waves a block where there are blocks for every CU twice over, else eight: one row of
    // 8192 x 8192 13.1 us (8: 13.6), 4096 x 14336 13.2 us (16: 15.1), 28672 x 4096 22.7 us (8: 26.8)
    if (blocks >= 512) scaled_few_kernel<4, T><<<blocks, 256, 0, st>>>(a);
    else scaled_few_kernel<8, T><<<blocks, 512, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t scaled_part(int out_type, int64_t m, int64_t n, int64_t k)
{
    return (size_t)plan_of(out_type, m, n, (int)((k + kScaled - 1) / kScaled)).p.part_bytes;
}

hipError_t launch_scaled(const ScaledArgs &a, hipStream_t st)
{
    if (a.out_type == KR_F32) return one<float>(a, st);
    if (a.out_type == KR_F16) return one<f16>(a, st);
    return one<bf16>(a, st);
}

hipError_t launch_scaled_pair(const ScaledArgs &a, const ScaledArgs &b, hipStream_t st)
{
    if (a.out_type == KR_F32) return pair<float>(a, b, st);
    if (a.out_type == KR_F16) return pair<f16>(a, b, st);
    return pair<bf16>(a, b, st);
}

hipError_t launch_scaled_few(const ScaledArgs &a, hipStream_t st)
{
    if (a.m > kScaledFew) return hipErrorInvalidValue;
    if (a.out_type == KR_F32) return few<float>(a, st);
    if (a.out_type == KR_F16) return few<f16>(a, st);
    return few<bf16>(a, st);
}

}  // namespace kr
