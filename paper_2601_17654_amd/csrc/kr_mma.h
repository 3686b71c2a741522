// Tiled matrix products on the matrix cores: what the projections are made of.
//
//   acc[m][n] = sum over k of A(m, k) B(n, k)
//
// An operand's rows are either contiguous in k ("plain": row m holds k = 0, 1, ...) or
// contiguous in m ("crossed": row k holds m = 0, 1, ...).  A block computes a BM x BN tile with
// one wave per (BM / WM) x (BN / WN) part, over k in steps of 128 bytes (64 16-bit values or
// 128 bytes).  Operand tiles go from memory straight to LDS, 16 bytes a lane, and from there to
// registers in the matrix instructions' layout: 16 rows x 16 bytes of k for each group of 16
// lanes.
//
// LDS layout.  A direct copy writes 64 lanes' 16 bytes side by side, so the order within a tile
// is chosen by what each lane fetches:
//  - plain: 128 bytes a row; 16-byte chunk c of row r sits at place c ^ (r / 2 % 8).  The 16
//    rows that a group of lanes reads at once then lie in 16 different 16-byte places of the
//    256 bytes that the 64 banks hold.
//  - crossed: one k a row; 32-byte block b (16 values) of row k sits at place b ^ f(k), f(k) =
//    k % 4 + 4 * (k / 8 % 4) (k / 8 % 2 where a row has 8 blocks).  The transposing read takes
//    4 rows x 32 bytes for each group of 16 lanes, the four groups 8 rows apart: 16 different
//    places (8).
// Whatever lies outside an operand is read as zero: rows past its end by the buffer's bound, k
// past the end of a plain row by an offset beyond that bound.
#pragma once

#include "kr_block.h"

namespace kr {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = 128;               // bytes of k a step
constexpr uint32_t kNowhere = 1u << 31;  // an offset past every buffer
constexpr uint32_t kBufferMost = kNowhere - 1;

// An element type's matrix instruction: 16 x 16 outputs, 64 bytes of k.  The first operand's
// rows become the registers of a lane (4 in a row), the second's the lanes.
template <typename E>
struct Mma {
    typedef f32x4 Acc;
    static constexpr int size = 2;
};
template <>
struct Mma<int8_t> {
    typedef i32x4 Acc;
    static constexpr int size = 1;
};
__device__ inline f32x4 mma(bf16, i32x4 a, i32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 mma(f16, i32x4 a, i32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ inline i32x4 mma(int8_t, i32x4 a, i32x4 b, i32x4 c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// One operand as the host describes it: `rows` rows (m, or k where crossed) of `bytes` bytes,
// `ld` bytes apart.  p and ld are multiples of 16 bytes, and so is `bytes` (crossed) or it is
// followed by zeros up to the next multiple (plain, a copy of this library's).
struct Operand {
    const char *p;
    int64_t ld;
    int64_t rows, bytes;
};

// Starts the copy of 16 bytes a lane to LDS, from byte `off` of a buffer; 64 lanes side by side.
// Written out because the compiler, where it knows of such a copy, waits for all of them before
// any read of LDS; here the waits are arrived() below.  There is no output register, and the
// copies' LDS is read only after such a wait.  The five idle states cover what the compiler
// cannot see inside: a scalar register that a vector instruction wrote, and m0.
__device__ inline void copy_to_lds(i32x4 rsrc, uint32_t off, const char *lds)
{
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)lds;
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "s_nop 4\n\t"
                 "buffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(rsrc)
                 : "memory", "m0");
}

// A tile of ROWS m (or n) x kStep bytes of k, copied by NW waves.  Copy i of the tile fills
// bytes [1024 i, 1024 i + 1024) of its LDS; wave w makes copies w * N .. w * N + N - 1.
template <bool CROSSED, int ROWS, int NW>
struct TileLoader {
    static constexpr int N = ROWS / 8 / NW;
    static constexpr int ROW_BYTES = CROSSED ? ROWS * 2 : kStep;
    static constexpr int LANES = ROW_BYTES / 16;  // lanes that a row takes
    static_assert(N * 8 * NW == ROWS && (CROSSED || N % 2 == 0), "copies do not divide");

    uint32_t off[N];
    uint32_t chunk[2];  // plain: byte of k that copies of either parity fetch
    const char *base;   // of the tile's first row (column)
    int64_t left;       // bytes of the operand from there
    int64_t step;       // bytes from one k step to the next

    // first: the tile's first m.  HALVES (plain): LDS rows are strips of 64, the first 32 of
    // one operand, the rest of another, both at 32 operand rows a strip.
    template <bool HALVES = false>
    __device__ void init(const Operand &o, int64_t first, int wave, int lane)
    {
        if (CROSSED) {
            base = o.p + first * 2;
            left = (o.rows - 1) * o.ld + o.bytes - first * 2;
            step = 64 * o.ld;
        } else {
            base = o.p + first * o.ld;
            left = (o.rows - 1 - first) * o.ld + o.bytes;
            step = kStep;
        }
        if (o.rows <= 0) left = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = wave * N + j;
            const int r = i * (64 / LANES) + lane / LANES, c = lane % LANES;
            if (CROSSED) {
                const int f = LANES == 32 ? (r & 3) | (r >> 3 & 3) << 2 : (r & 3) | (r >> 3 & 1) << 2;
                off[j] = (uint32_t)r * (uint32_t)o.ld + (uint32_t)(c ^ f << 1) * 16;
            } else {
                const int at = c ^ (r >> 1 & 7);
                const int row = HALVES ? (r / 64) * 32 + r % 32 : r;
                off[j] = (uint32_t)row * (uint32_t)o.ld + (uint32_t)at * 16;
                chunk[j & 1] = (uint32_t)at * 16;
            }
        }
    }

    // Starts the copies of step t; k_left: bytes of k from that step's start (plain).
    __device__ void load(int t, int64_t k_left, char *lds, int wave) const
    {
        const int64_t rest = left - t * step;
        const uint32_t records = rest <= 0 ? 0u : rest > kBufferMost ? kBufferMost : (uint32_t)rest;
        const uint64_t at = (uint64_t)(base + t * step);
        const i32x4 rsrc = {(int)at, (int)(at >> 32) & 0xFFFF, (int)records, 0x00020000};
#pragma unroll
        for (int j = 0; j < N; ++j) {
            uint32_t o = off[j];
            if (!CROSSED) o = (int64_t)chunk[j & 1] < k_left ? o : kNowhere;
            copy_to_lds(rsrc, o, lds + (wave * N + j) * 1024);
        }
    }
};

// Reads of a tile in LDS: rows (plain) or columns (crossed) first .. first + 15, half h of the
// step (64 bytes of k).
template <bool CROSSED, int ROWS>
struct TileReader {
    int at[2];  // plain: a lane's byte for either half
    int k0, fl;

    __device__ void init(int lane)
    {
        const int g = lane / 16, i = lane % 16;
        if (CROSSED) {
            k0 = (g * 8 + i / 4) * ROWS * 2 + (i % 4) * 8;
            fl = ROWS == 256 ? i / 4 | g << 2 : i / 4 | (g & 1) << 2;
        } else {
            at[0] = i * kStep + ((g ^ i >> 1) << 4);
            at[1] = i * kStep + (((4 + g) ^ i >> 1) << 4);
        }
    }
    __device__ i32x4 read(const char *lds, int first, int h) const
    {
        if (!CROSSED) return *(const i32x4 *)(lds + first * kStep + at[h]);
        typedef __attribute__((address_space(3))) s16x4 *Lds;
        const char *p = lds + k0 + ((first / 16 ^ fl) << 5) + h * 32 * ROWS * 2;
        struct {
            s16x4 lo, hi;
        } x;
        x.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p);
        x.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * ROWS * 2));
        return __builtin_bit_cast(i32x4, x);
    }
};

// What a product's blocks have in common.
struct MmaArgs {
    Operand a[2], b[2];  // second pair: the second half of the sum, or B's second half
    int m, n;            // outputs
    int64_t k_bytes;     // bytes of k in one pair (plain operands), rows of it where crossed
    int steps;           // k steps of one pair
    int pairs;           // 1, or 2: A0 B0 + A1 B1
    int tiles_m, tiles_n, splits, per_split;  // steps of a split
    float *part;         // splits > 1: [split][plane][m][n] (int32 for bytes)
};

// The tile of a block.  Blocks go to the 8 XCDs in turn: each XCD takes a run of consecutive
// tiles, and a run covers 8 tiles of m before it moves on in n, so that the tiles of an XCD
// share rows of both operands in its L2.
__device__ inline void tile_of(const MmaArgs &a, int *tm, int *tn, int *split)
{
    const int per = a.tiles_m * a.tiles_n, all = per * a.splits;
    const int id = (int)blockIdx.x, x = id & 7, q = all >> 3, r = all & 7;
    int t = x * q + min(x, r) + (id >> 3);
    *split = t / per;
    t -= *split * per;
    const int group = 8 * a.tiles_n, g = t / group, first = g * 8;
    const int size = min(8, a.tiles_m - first);
    t -= g * group;
    *tm = first + t % size;
    *tn = t / size;
}

template <typename T, typename S>
__device__ inline void store4(T *row, int n, int width, const S *v)
{
    struct __attribute__((packed)) Loose {
        T v[4];
    };
    if (n + 4 <= width) {
        Loose x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[e] = (T)v[e];
        *(Loose *)(row + n) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < width) row[n + e] = (T)v[e];
    }
}

// Waits for all but the last LEFT of the wave's copies to LDS, then for the block.
template <int LEFT>
__device__ inline void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Waits for the wave's reads of LDS, then for the block: what was read may be overwritten.
__device__ inline void read_done()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The block's waves meet; memory accesses are not moved across.
__device__ inline void block_barrier() { asm volatile("s_barrier" ::: "memory"); }

// A block's sums to the output, or to its split's part.
template <int BM, int BN, int WM, int WN, typename Out, typename Acc>
__device__ inline void put_tile(const MmaArgs &a, const Out &out, const Acc (&acc)[BM / WM / 16][BN / WN / 16],
                                int64_t m0, int64_t n0, int wm, int wn, int split, int lane)
{
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr bool TWO = Out::PLANES == 2;
    const int row = lane % 16, col = lane / 16 * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm * (BM / WM) + i * 16 + row;
        if (m >= a.m) continue;
#pragma unroll
        for (int j = 0; j < (TWO ? TN / 2 : TN); ++j) {
            const int64_t n = n0 + wn * (BN / WN / Out::PLANES) + j * 16 + col;
            if (n >= out.columns(a.n)) continue;
            const Acc v0 = acc[i][j], v1 = acc[i][TWO ? j + TN / 2 : j];
            if (a.splits > 1) {
                typedef decltype(v0[0] + v0[0]) S;
                S *p = (S *)a.part + ((int64_t)split * Out::PLANES * a.m + m) * a.n;
                store4(p, (int)n, a.n, (const S *)&v0);
                if (TWO) store4(p + (int64_t)a.m * a.n, (int)n, a.n, (const S *)&v1);
            } else {
                out.put(m, (int)n, v0, v1);
            }
        }
    }
}

// One product kernel.  Out says what happens to the sums:
//   PLANES         1, or 2: B's tile is half of b[0], half of b[1] (same rows), two sums
//   put(m, n, v0, v1)   four outputs from n on of row m, from the first and second plane
template <typename E, bool A_CROSSED, bool B_CROSSED, int BM, int BN, int WM, int WN, typename Out>
__global__ __launch_bounds__(WM *WN * 64) void mma_kernel(MmaArgs a, Out out)
{
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr bool TWO = Out::PLANES == 2;
    constexpr int OUT_N = TWO ? BN / 2 : BN;  // output columns of a tile
    static_assert(!TWO || BN / WN == 64, "a strip of both planes is 64 wide");
    typedef typename Mma<E>::Acc Acc;
    __shared__ __align__(1024) char lds[2][(BM + BN) * kStep];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn, split;
    tile_of(a, &tm, &tn, &split);
    const int64_t m0 = (int64_t)tm * BM;
    const int64_t n0 = (int64_t)tn * OUT_N;

    typedef TileLoader<A_CROSSED, BM, NW> LoadA;
    typedef TileLoader<B_CROSSED, BN, NW> LoadB;
    LoadA la;
    LoadB lb;
    TileReader<A_CROSSED, BM> ra;
    TileReader<B_CROSSED, BN> rb;
    ra.init(lane);
    rb.init(lane);

    Acc acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = Acc{0, 0, 0, 0};

    const int begin = split * a.per_split, end = min(begin + a.per_split, a.steps * a.pairs);
    int pair = -1;
    auto load = [&](int s, int buf) {
        const int p = s >= a.steps ? 1 : 0;
        if (p != pair) {
            pair = p;
            la.init(a.a[p], m0, wave, lane);
            // a wave copies rows of one half only: N * 8 = 32 of a strip's 64
            const int h = TWO ? (wave * LoadB::N / 4) & 1 : p;
            lb.template init<TWO>(a.b[h], n0, wave, lane);
        }
        const int t = s - p * a.steps;
        const int64_t k_left = a.k_bytes - (int64_t)t * kStep;
        la.load(t, k_left, lds[buf], wave);
        lb.load(t, k_left, lds[buf] + BM * kStep, wave);
    };

    if (begin < end) load(begin, 0);
    for (int s = begin; s < end; ++s) {
        const int buf = (s - begin) & 1;
        if (s + 1 < end) {
            load(s + 1, buf ^ 1);
            arrived<LoadA::N + LoadB::N>();  // all but the next step's
        } else {
            arrived<0>();
        }
        const char *sa = lds[buf], *sb = lds[buf] + BM * kStep;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = ra.read(sa, wm * (BM / WM) + i * 16, h);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = rb.read(sb, wn * (BN / WN) + j * 16, h);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = mma(E(), fb[j], fa[i], acc[i][j]);
        }
        read_done();
    }

    put_tile<BM, BN, WM, WN>(a, out, acc, m0, n0, wm, wn, split, lane);
}

// The same for 256 x 256 tiles, with the two waves of each SIMD taking turns: while one waits for
// its reads of LDS, the other keeps the matrix cores busy.  A step is four phases, one for each
// quarter of a wave's 128 x 64 sums (64 x 32 each, 16 matrix instructions); a phase is a memory
// part and a matrix part with a barrier after either, and waves 4 .. 7 run one barrier behind
// waves 0 .. 3.
//
//   phase   reads        sums       slots of waves 0-3 / 4-7 (a slot ends with a barrier)
//   0       A0, B0       A0 B0      8s,     8s + 1  /  8s + 1, 8s + 2
//   1       B1           A0 B1      8s + 2, 8s + 3  /  8s + 3, 8s + 4
//   2       A1           A1 B1      8s + 4, 8s + 5  /  8s + 5, 8s + 6
//   3       copies of    A1 B0      8s + 6, 8s + 7  /  8s + 7, 8s + 8
//           step s + 2
//
// The last reads of step s's buffer are phase 2's, waited for inside slots 8s + 4 and 8s + 5, so
// the copies that overwrite it from slot 8s + 6 on come after them.  A wave waits for its own
// copies of step s + 1 (a whole step old by then) in phase 3's memory part, slots 8s + 6 and
// 8s + 7; step s + 1's first reads are in slots 8s + 8 and 8s + 9.
template <typename E, bool A_CROSSED, bool B_CROSSED, typename Out>
__global__ __launch_bounds__(512) void mma_wide_kernel(MmaArgs a, Out out)
{
    constexpr int BM = 256, BN = 256, WM = 2, WN = 4, NW = 8;
    constexpr bool TWO = Out::PLANES == 2;
    typedef typename Mma<E>::Acc Acc;
    __shared__ __align__(1024) char lds[2][(BM + BN) * kStep];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn, split;
    tile_of(a, &tm, &tn, &split);
    const int64_t m0 = (int64_t)tm * BM;
    const int64_t n0 = (int64_t)tn * (TWO ? BN / 2 : BN);

    typedef TileLoader<A_CROSSED, BM, NW> LoadA;
    typedef TileLoader<B_CROSSED, BN, NW> LoadB;
    constexpr int COPIES = LoadA::N + LoadB::N;
    LoadA la;
    LoadB lb;
    TileReader<A_CROSSED, BM> ra;
    TileReader<B_CROSSED, BN> rb;
    ra.init(lane);
    rb.init(lane);

    Acc acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = Acc{0, 0, 0, 0};

    const int begin = split * a.per_split, end = min(begin + a.per_split, a.steps * a.pairs);
    int pair = -1;
    auto load = [&](int s, int buf) {
        const int p = s >= a.steps ? 1 : 0;
        if (p != pair) {
            pair = p;
            la.init(a.a[p], m0, wave, lane);
            const int h = TWO ? wave & 1 : p;  // a wave copies rows of one plane only
            lb.template init<TWO>(a.b[h], n0, wave, lane);
        }
        const int t = s - p * a.steps;
        const int64_t k_left = a.k_bytes - (int64_t)t * kStep;
        la.load(t, k_left, lds[buf], wave);
        lb.load(t, k_left, lds[buf] + BM * kStep, wave);
    };

    i32x4 fa[2][4], fb[2][2][2];  // [half of the step][16 rows]; B: [quarter] in front
    auto read_a = [&](const char *at, int q) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) fa[h][i] = ra.read(at, wm * 128 + q * 64 + i * 16, h);
    };
    auto read_b = [&](const char *at, int q) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                fb[q][h][j] = rb.read(at + BM * kStep, wn * 64 + q * 32 + j * 16, h);
    };
    auto sums = [&](int qa, int qb) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[qa * 4 + i][qb * 2 + j] =
                        mma(E(), fb[qb][h][j], fa[h][i], acc[qa * 4 + i][qb * 2 + j]);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        block_barrier();
    };

    if (begin < end) load(begin, 0);
    if (begin + 1 < end) {
        load(begin + 1, 1);
        arrived<COPIES>();
    } else {
        arrived<0>();
    }
    if (wm == 1) block_barrier();
    for (int s = begin; s < end; ++s) {
        const int buf = (s - begin) & 1;
        const char *at = lds[buf];
        read_a(at, 0);
        read_b(at, 0);
        block_barrier();
        sums(0, 0);
        read_b(at, 1);
        block_barrier();
        sums(0, 1);
        read_a(at, 1);
        read_done();
        sums(1, 1);
        if (s + 2 < end) {
            load(s + 2, buf);
            arrived<COPIES>();
        } else {
            arrived<0>();
        }
        sums(1, 0);
    }
    if (wm == 0) block_barrier();
    put_tile<BM, BN, WM, WN>(a, out, acc, m0, n0, wm, wn, split, lane);
}

// The splits' sums added in turn, then put: four outputs a thread.
template <typename E, typename Out>
__global__ __launch_bounds__(256) void mma_join_kernel(MmaArgs a, Out out)
{
    typedef typename Mma<E>::Acc Acc;
    typedef decltype(Acc{}[0] + Acc{}[0]) S;
    const int quads = (out.columns(a.n) + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)a.m * quads) return;
    const int64_t m = id / quads;
    const int n = (int)(id - m * quads) * 4;
    Acc v[2] = {Acc{0, 0, 0, 0}, Acc{0, 0, 0, 0}};
    for (int s = 0; s < a.splits; ++s)
#pragma unroll
        for (int p = 0; p < Out::PLANES; ++p) {
            const S *q = (const S *)a.part + (((int64_t)s * Out::PLANES + p) * a.m + m) * a.n;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < a.n) v[p][e] += q[n + e];
        }
    out.put(m, n, v[0], v[Out::PLANES - 1]);
}

// How a product is cut into tiles.
struct MmaPlan {
    bool large;   // 256 x 256 tiles of 8 waves, else 128 x 128 of 4
    int tiles_m, tiles_n, splits, per_split;
    int64_t part_bytes;
};
MmaPlan mma_plan(int64_t m, int64_t n, int planes, int steps);

template <typename E, bool A_CROSSED, bool B_CROSSED, typename Out>
hipError_t launch_mma(MmaArgs a, const MmaPlan &p, const Out &out, hipStream_t st)
{
    a.tiles_m = p.tiles_m;
    a.tiles_n = p.tiles_n;
    a.splits = p.splits;
    a.per_split = p.per_split;
    const unsigned blocks = (unsigned)(p.tiles_m * p.tiles_n * p.splits);
    if (p.large)
        mma_wide_kernel<E, A_CROSSED, B_CROSSED, Out><<<blocks, 512, 0, st>>>(a, out);
    else
        mma_kernel<E, A_CROSSED, B_CROSSED, 128, 128, 2, 2, Out><<<blocks, 256, 0, st>>>(a, out);
    if (p.splits > 1) {
        const int64_t quads = (int64_t)a.m * ((out.columns(a.n) + 3) / 4);
        mma_join_kernel<E, Out><<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(a, out);
    }
    return hipGetLastError();
}

}  // namespace kr
