// Tiled matrix products on the matrix cores: what the projections are made of.
//
//   acc[m][n] = sum over k of A(m, k) B(n, k)
//
// An operand's rows are either contiguous in k ("plain": row m holds k = 0, 1, ...) or
// contiguous in m ("crossed": row k holds m = 0, 1, ...).  A block computes a BM x BN tile with
// one wave per (BM / WM) x (BN / WN) part, over k in steps of 128 bytes (64 16-bit values or
// 128 bytes).  Operand tiles go from memory straight to LDS, 16 bytes a lane, and from there to
// registers in the layout of the 16 x 16 matrix instructions: 16 rows x 16 bytes of k for each
// group of 16 lanes.  (Under full load the clock is what the power leaves, and the 32 x 32 ones,
// which move twice the sums through the registers for the same products, leave less: out of
// registers alone, on random values, 1,820 against 1,960 TFLOP/s in bfloat16.)
//
// LDS layout.  A direct copy writes 64 lanes' 16 bytes side by side, so the order within a tile
// is chosen by what each lane fetches:
//  - plain: 128 bytes a row; 16-byte chunk c of row r sits at place c ^ (r / 2 % 8).  16
//    consecutive rows, read at one c, then lie in 16 different 16-byte places of the 256 bytes
//    that the 64 banks hold.
//  - crossed: one k a row; 32-byte block b (16 values) of row k sits at place b ^ f(k), f(k) =
//    k % 4 + 4 (k / 8 % 4) (k / 8 % 2 where a row has 8 blocks).  The transposing read takes 4
//    rows x 32 bytes for each group of 16 lanes, the four groups 8 rows apart: 16 different
//    places (8, twice).
// What a sum takes from outside an operand is zero: rows past its end by the buffer's bound, k
// past the end of a plain row by an offset beyond that bound.  (Columns past the end of a crossed
// row are what lies there, the gap between rows or the next one; they end in outputs that are not
// put.)
#pragma once

#include <type_traits>
#include <utility>

#include "kr_block.h"
#include "kr_plan.h"

namespace kr {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = 128;               // bytes of k a step
constexpr uint32_t kNowhere = 1u << 31;  // an offset past every buffer
constexpr uint32_t kBufferMost = kNowhere - 1;

// An element type's matrix instruction: 16 x 16 outputs, 64 bytes of k.  The second operand's
// rows become the lanes (row lane % 16), the first's the registers: register r is its row
// 4 (lane / 16) + r.
template <typename E>
struct Mma {
    typedef f32x4 Acc;
    typedef float Sum;
};
template <>
struct Mma<int8_t> {
    typedef i32x4 Acc;
    typedef int Sum;
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

// The same, c += a b, with the sums kept where they are.  (Left to itself, the compiler gives the
// result other registers than the sums had, and moves a hundred a step to make room.)  It adds no
// wait states around these; what they need is there by the order of things: the operands come from
// LDS, whose arrival the compiler waits for, not from a vector instruction just before, and an
// instruction's sums are not touched again before sums_done() but by the next on the same
// sums, 16 or more later.  tests/test_matrix_instructions.py reads both off the built library.
__device__ inline void mma_in_place(bf16, i32x4 a, i32x4 b, f32x4 &c)
{
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
__device__ inline void mma_in_place(f16, i32x4 a, i32x4 b, f32x4 &c)
{
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
__device__ inline void mma_in_place(int8_t, i32x4 a, i32x4 b, i32x4 &c)
{
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
// Between such instructions and any other use of their sums, which are tied to its middle: no write of
// them can come to stand after it, and no read before it, with 16 states on either side (11 are needed).
template <typename Acc, int TM, int TN>
__device__ __attribute__((always_inline)) inline void sums_done(Acc (&acc)[TM][TN])
{
    asm volatile("s_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) asm volatile("" : "+a"(acc[i][j]));
    asm volatile("s_nop 15" ::: "memory");
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
// copies' LDS is read only after such a wait.  The buffer's registers come from scalar arithmetic
// (a vector instruction's result would need five states).  In two parts, with a matrix
// instruction between them: a wave issues three instructions in a matrix instruction's time, and
// these are four.  m0 is handed on as a value, so that nothing else can come to stand in it.
__device__ inline uint32_t copy_ready(uint32_t off, const char *lds)
{
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)lds;
    uint32_t m0;
    asm volatile("s_mov_b32 %0, %1" : "={m0}"(m0) : "s"(to), "v"(off));
    return m0;
}
__device__ inline void copy_go(uint32_t off, const i32x4 &rsrc, uint32_t m0)
{
    asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "{m0}"(m0) : "memory");
}
// At once, with the idle state that stands between m0 and its use.
__device__ inline void copy_to_lds(const i32x4 &rsrc, uint32_t off, const char *lds)
{
    const uint32_t m0 = copy_ready(off, lds);
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "{m0}"(m0)
                 : "memory");
}

// Scalar work on x is neither moved up past this point nor down.
template <typename T>
__device__ __attribute__((always_inline)) inline void here(T &x)
{
    asm volatile("" : "+s"(x));
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
    int chunk[2];       // plain: byte of k that copies of either parity fetch
    uint32_t past[2];   //        kNowhere where that is past the end
    const char *base;   // of the tile's first row (column)
    int64_t left;       // bytes of the operand from there
    int64_t step;       // bytes from one k step to the next
    uint64_t at;        // the step it aims at, and the bytes of the operand from there
    int64_t rest;

    // first: the tile's first m; map: the m, from there, of a row of LDS (runs of 8 rows of LDS,
    // 16 where crossed, are runs of m).
    template <typename Map>
    __device__ void init(const Operand &o, int64_t first, int wave, int lane, Map map)
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
                const int f = (r & 3) | (r >> 3 & (LANES == 32 ? 3 : 1)) << 2;
                off[j] = (uint32_t)r * (uint32_t)o.ld + (uint32_t)map((c ^ f << 1) * 8) * 2;
            } else {
                const int at = c ^ (r >> 1 & 7);
                off[j] = (uint32_t)map(r) * (uint32_t)o.ld + (uint32_t)at * 16;
                chunk[j & 1] = at * 16;
            }
        }
    }

    // The operand from step t on, `by` bytes from the one that init() took (another of its shape).
    __device__ void aim(int t, int64_t by)
    {
        at = (uint64_t)(base + by + t * step);
        rest = left - t * step;
    }
    // The step after, or the first of the operand `by` bytes away.
    __device__ void next_at(bool first, int64_t by)
    {
        here(at);
        at = first ? (uint64_t)(base + by) : at + step;
        here(at);
    }
    __device__ void next_rest(bool first)
    {
        here(rest);
        rest = first ? left : rest - step;
        here(rest);
    }
    // What it aims at as a buffer; an empty one where there is no such step.
    __device__ i32x4 buffer(bool there) const
    {
        int high = (int)(rest >> 32);
        here(high);
        const uint32_t low = min((uint32_t)rest, kBufferMost);
        const uint32_t records = high == 0 ? low : high < 0 ? 0u : kBufferMost;
        i32x4 x{(int)at, (int)(at >> 32) & 0xFFFF, there ? (int)records : 0, 0x00020000};
        here(x);
        return x;
    }
    // Says how many bytes of k there are from the step's start (plain).
    __device__ void bound(int k_left)
    {
        if (!CROSSED) {
            const int most = min(k_left, kStep);
#pragma unroll
            for (int j = 0; j < 2; ++j) past[j] = chunk[j] < most ? 0 : kNowhere;
        }
    }
    // What the wave's copy j of a step fetches, and where to.
    __device__ uint32_t from(int j) const { return CROSSED ? off[j] : off[j] | past[j & 1]; }
    __device__ const char *to(int j, const char *lds, int wave) const
    {
        return lds + (wave * N + j) * 1024;
    }
};

// Maps of a tile's rows: as they are;  strips of STRIP rows, one half of either plane.
struct MapSame {
    __device__ int operator()(int r) const { return r; }
};
template <int STRIP>
struct MapPlanes {
    __device__ int operator()(int r) const { return r / STRIP * (STRIP / 2) + r % (STRIP / 2); }
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
            fl = i / 4 | (g & (ROWS == 256 ? 3 : 1)) << 2;
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) at[h] = i * kStep + (((h * 4 + g) ^ i >> 1) << 4);
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
    Operand a[2], b[2];  // second pair: the second half of the sum (of the first one's ld), or
                         // B's second plane
    int m, n;            // outputs
    int64_t k_bytes;     // bytes of k in one pair's plain operands; not used where both are crossed
    int steps;           // k steps of one pair
    int pairs;           // 1, or 2: A0 B0 + A1 B1
    int tiles_m, tiles_n, splits, per_split;  // steps of a split
    float *part;         // splits > 1: [split][plane][m][n] (int32 for bytes)
};

// The tile of a block.  Blocks go to the 8 XCDs in turn: each XCD takes a run of consecutive
// tiles, and a run covers 4 tiles of m before it moves on in n, so that the tiles of an XCD
// share rows of both operands in its L2.
__device__ inline void tile_of(const MmaArgs &a, int *tm, int *tn, int *split)
{
    const int per = a.tiles_m * a.tiles_n, all = per * a.splits;
    const int id = (int)blockIdx.x, x = id & 7, q = all >> 3, r = all & 7;
    int t = x * q + min(x, r) + (id >> 3);
    *split = t / per;
    t -= *split * per;
    const int group = 4 * a.tiles_n, g = t / group, first = g * 4;
    const int size = min(4, a.tiles_m - first);
    t -= g * group;
    *tm = first + t % size;
    *tn = t / size;
}

// Nothing that a lane needs or reads.
struct Plain {
    struct Mine {
    };
    struct Fetched {
    };
    __device__ Mine mine(int) const { return {}; }
    __device__ Fetched fetch(bool, int64_t, int) const { return {}; }
};

// Eight values to columns n .. n + 7 of a row of `width`.
template <typename T, typename S>
__device__ inline void store8(T *row, int n, int width, const S *v)
{
    struct __attribute__((packed)) Loose {
        T v[8];
    };
    if (n + 8 <= width) {
        Loose x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x.v[e] = (T)v[e];
        *(Loose *)(row + n) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (n + e < width) row[n + e] = (T)v[e];
    }
}

// Waits for all but the last LEFT of the wave's copies to LDS, then for the block: what was
// copied may be read.
template <int LEFT>
__device__ inline void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Waits for the wave's reads of LDS, then for the block: what was read may be overwritten.
__device__ inline void read_done() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Between the writes of a wave's LDS and reads of it by other lanes of the wave: the hardware keeps a
// wave's own order, this keeps the compiler's (no instruction comes of it).
__device__ inline void wave_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A block's sums to the output, or to its split's part.  Each wave takes them through its own
// share of the LDS, 64 rows at a time: out of the matrix layout into rows of 8 neighbouring
// columns a lane, so that whole lines are written, in a loop that is short in code (unrolled over
// the registers, this part was 150 KB of instructions that every block fetched anew, a quarter of
// a tile's time at 64 steps).  16-byte chunk c of row r lies at place c ^ r % 16.
template <int BM, int BN, int WM, int WN, typename E, typename Out, typename Acc>
__device__ inline void put_tile(E, const MmaArgs &a, const Out &out,
                                const Acc (&acc)[BM / WM / 16][BN / WN / 16], char *lds, int64_t m0,
                                int64_t n0, int wave, int split, int lane)
{
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16, PLANES = Out::PLANES;
    constexpr int STRIP = BN / WN, COLS = STRIP / PLANES;  // of a wave's sums, of its output
    constexpr int LANES = COLS / 8;                        // lanes a row
    // What the output reads of every row is asked for at once, ahead of all else: one wait for
    // memory a tile (four rows at a time, the gated backward's first product took 1 % longer).
    constexpr bool ASKS = !std::is_empty<typename Out::Fetched>::value;
    typedef typename Mma<E>::Sum Sum;
    static_assert(64 * STRIP * 4 * WM * WN <= 2 * (BM + BN) * kStep, "a wave's share of LDS");
    char *own = lds + wave * 64 * STRIP * 4;
    const int wm = wave / WN, wn = wave % WN;
    const int n = (int)n0 + wn * COLS + lane % LANES * 8, columns = out.columns(a.n);
    const int64_t m1 = m0 + wm * (BM / WM) + lane / LANES;
    typename Out::Fetched asked[TM / 4][LANES];
    if (ASKS) {
#pragma unroll
        for (int p = 0; p < TM / 4; ++p)
#pragma unroll
            for (int it = 0; it < LANES; ++it) {
                const int64_t m = m1 + p * 64 + it * (64 / LANES);
                asked[p][it] = out.fetch(m < a.m && n < columns, m, n);
            }
    }
    const typename Out::Mine mine = out.mine(n);
    auto put = [&](int p, int it, const typename Out::Fetched &f) __attribute__((always_inline)) {
        const int row = it * (64 / LANES) + lane / LANES;
        const int64_t m = m1 + p * 64 + it * (64 / LANES);
        Acc v[PLANES][2];
#pragma unroll
        for (int k = 0; k < PLANES; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = k * COLS / 4 + lane % LANES * 2 + h;
                v[k][h] = *(const Acc *)(own + row * STRIP * 4 + ((c ^ row % 16) << 4));
            }
        if (m >= a.m || n >= columns) return;
        const Sum *v0 = (const Sum *)v[0], *v1 = (const Sum *)v[PLANES - 1];
        if (a.splits > 1) {
            Sum *to = (Sum *)a.part + ((int64_t)split * PLANES * a.m + m) * a.n;
            store8(to, n, a.n, v0);
            if (PLANES == 2) store8(to + (int64_t)a.m * a.n, n, a.n, v1);
        } else {
            out.put(m, n, v0, v1, mine, f);
        }
    };
#pragma unroll
    for (int p = 0; p < TM / 4; ++p) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int row = i * 16 + lane % 16, c = j * 4 + lane / 16;
                *(Acc *)(own + row * STRIP * 4 + ((c ^ row % 16) << 4)) = acc[p * 4 + i][j];
            }
        wave_lds();
        if (ASKS) {
#pragma unroll
            for (int it = 0; it < LANES; ++it) put(p, it, asked[p][it]);
        } else {
#pragma unroll 4
            for (int it = 0; it < LANES; ++it) put(p, it, typename Out::Fetched());
        }
        wave_lds();
    }
}

// One product kernel.  Out says what happens to the sums:
//   PLANES         1, or 2: B's tile is half of b[0], half of b[1] (same rows), two sums
//   columns(n)     columns to put, n or more
//   Mine mine(n)   what a lane needs for its columns n .. n + 7 in every row (called by whole
//                  waves, but in the form of few rows)
//   Fetched fetch(there, m, n)   what it reads for them of row m, asked for ahead
//   put(m, n, v0, v1, mine, fetched)   eight outputs from n on of row m, from the first and second
//                                      plane
//
// f(0), f(1), ... with constants: 128 steps are more than the compiler unrolls of a loop.
template <int N>
using Count = std::make_integer_sequence<int, N>;
template <typename F, int... X>
__device__ __attribute__((always_inline)) inline void each(std::integer_sequence<int, X...>, F f)
{
    (f(std::integral_constant<int, X>()), ...);
}

// Two steps' tiles are in LDS, and a wave's registers hold one more: the matrix instructions of
// a step (two halves of TM x TN) run on what was read before them, and between them are
//   the reads of half 1, from the step's beginning;
//   from instruction T::free on, when every wave has its step in registers (a barrier): the
//     copies of the step after next, over this one's tile;
//   from T::next on, when every wave's copies of the next step have arrived (a barrier): the
//     reads of its half 0.
// The 256 x 256 form has one wave per SIMD: its 128 x 128 sums halve the reads of LDS against
// 8 waves' 128 x 64.  A CU takes 16 cycles, one matrix instruction, to address a copy, and 8 to
// read 1 KiB of LDS; its four waves start theirs at the same time, and what they wait for each
// other the matrix cores wait too.  So reads are two instructions apart there and copies five.
// 8192 x 8192 x 4096 in bfloat16: 394 us (1,394 TFLOP/s); 8-bit integers, 8192^3: 408 us (2,700
// TOP/s).  What bounds it is power: the clock falls from 2.4 to 2.0 GHz on random values (zeros
// take 335 us).
// The 128 x 128 form, for outputs that do not fill the chip with large tiles, has two blocks a CU.
// In a long sum a block's step takes 0.47 us, 1,120 cycles, whether a CU has one block or two (0.5
// with steps of 64 bytes, half a line each; the same with four steps' tiles in LDS and one block a
// CU): 512 cycles of LDS reads, 512 of what the copies bring there, 512 of the matrix cores.  In
// short sums that is the smaller part.  1111 x 1030 -> 2731, 387 tiles of 17 steps: 28 us, of which a
// CU's LDS is busy 8,300 cycles of 67,000 and the matrix cores 20 %; the rest is the first
// copies' way, the outputs, and CUs with one tile that wait for those with two.
template <int BLOCK>
struct Timing;  // apart: of reads;  copies(x): those started before instruction x
template <>
struct Timing<64> {
    static constexpr int free = 40, next = 96, apart = 2;
    static constexpr int copies(int x) { return x - free < 80 ? (x - free + 4) / 5 : 16; }
};
template <>
struct Timing<16> {
    static constexpr int free = 14, next = 24, apart = 1;
    static constexpr int copies(int x) { return x - free < 16 ? (x - free + 1) / 2 : 8; }
};

template <typename E, bool A_CROSSED, bool B_CROSSED, int BM, int BN, int WM, int WN, typename Out>
__global__ __launch_bounds__(WM *WN * 64) void mma_kernel(MmaArgs a, Out out)
{
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr bool TWO = Out::PLANES == 2;
    constexpr int STRIP = BN / WN;
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
    constexpr int COPIES = LoadA::N + LoadB::N, BLOCK = TM * TN, READS = TM + TN;
    typedef Timing<BLOCK> T;
    static_assert(T::free >= T::apart * READS && T::next >= BLOCK &&
                      T::next + T::apart * READS <= 2 * BLOCK && T::copies(T::free) == 0 &&
                      T::copies(2 * BLOCK) == COPIES,
                  "the timing fits the tile");
    static_assert(!TWO || LoadB::N * 8 == STRIP / 2, "a wave copies rows of one plane only");
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
    la.init(a.a[0], m0, wave, lane, MapSame());
    if (TWO)
        lb.init(a.b[wave & 1], n0, wave, lane, MapPlanes<STRIP>());
    else
        lb.init(a.b[0], n0, wave, lane, MapSame());
    const int64_t to_second_a = a.a[1].p - a.a[0].p, to_second_b = a.b[1].p - a.b[0].p;
    // The step that copies are of goes one on in parts, which stand between matrix instructions
    // (in one piece at a step's head its 55 scalar instructions were 8 % of the step).
    int step = begin, k_left = 0;
    i32x4 rsrc_a, rsrc_b;
    constexpr int PARTS = 8;
    auto aim = [&](int part) __attribute__((always_inline)) {
        const bool first = step == a.steps;  // of the second pair
        if (part == 0) {
            ++step;
            here(step);
        }
        if (part == 1) la.next_at(first, to_second_a);
        if (part == 2) la.next_rest(first);
        if (part == 3) rsrc_a = la.buffer(step < end);
        if (part == 4) lb.next_at(first, to_second_b);
        if (part == 5) lb.next_rest(first);
        if (part == 6) rsrc_b = lb.buffer(step < end);
        if (part == 7 && !(A_CROSSED && B_CROSSED)) {
            here(k_left);
            k_left = first ? (int)a.k_bytes : k_left - kStep;
            la.bound(k_left);
            lb.bound(k_left);
        }
    };
    auto from = [&](int j) { return j < LoadA::N ? la.from(j) : lb.from(j - LoadA::N); };
    auto to = [&](int j, const char *at) {
        return j < LoadA::N ? la.to(j, at, wave) : lb.to(j - LoadA::N, at + BM * kStep, wave);
    };

    i32x4 fa[2][TM], fb[2][TN];  // halves of a step
    auto read = [&](int j, const char *at, int h) {
        if (j < TM)
            fa[h][j] = ra.read(at, wm * (BM / WM) + j * 16, h);
        else
            fb[h][j - TM] = rb.read(at + BM * kStep, wn * STRIP + (j - TM) * 16, h);
    };

    // Past the last step the copies are of an empty buffer, zeros that nothing uses: every step
    // is the same, and the waits too.
    const bool second = begin >= a.steps;
    const int t = second ? begin - a.steps : begin;
    la.aim(t, second ? to_second_a : 0);
    lb.aim(t, second ? to_second_b : 0);
    if (!(A_CROSSED && B_CROSSED)) k_left = (int)a.k_bytes - t * kStep;
    la.bound(k_left);
    lb.bound(k_left);
    rsrc_a = la.buffer(begin < end);
    rsrc_b = lb.buffer(begin < end);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int j = 0; j < COPIES; ++j) copy_to_lds(j < LoadA::N ? rsrc_a : rsrc_b, from(j), to(j, lds[k]));
        if (k == 0) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) aim(p);
        }
    }
    arrived<COPIES>();
#pragma unroll
    for (int j = 0; j < TM + TN; ++j) read(j, lds[0], 0);
    sums_done(acc);
    for (int s = begin; s < end; ++s) {
        const int buf = (s - begin) & 1;
        const char *at = lds[buf], *next = lds[buf ^ 1];
        uint32_t off = 0, m0 = 0;
        each(Count<2 * BLOCK>(), [&](auto at_x) __attribute__((always_inline)) {
            constexpr int x = decltype(at_x)::value;
            if (x % T::apart == 0 && x / T::apart < READS) read(x / T::apart, at, 1);
            if (x == T::free) read_done();
            if (x == T::next) arrived<T::copies(T::next)>();
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
                if (p * T::free / PARTS == x) aim(p);
            if (x >= T::free && T::copies(x + 1) > T::copies(x))
                copy_go(off, T::copies(x) < LoadA::N ? rsrc_a : rsrc_b, m0);
            if (x + 1 >= T::free && T::copies(x + 2) > T::copies(x + 1)) {
                off = from(T::copies(x + 1));
                m0 = copy_ready(off, to(T::copies(x + 1), at));
            }
            if (x >= T::next && (x - T::next) % T::apart == 0 && (x - T::next) / T::apart < READS)
                read((x - T::next) / T::apart, next, 0);
            // to and fro: neighbours share an operand (0.4 % at full power)
            constexpr int h = x / BLOCK, j = x % BLOCK / TM, i = j % 2 ? TM - 1 - x % TM : x % TM;
            mma_in_place(E(), fb[h][j], fa[h][i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        });
    }
    sums_done(acc);
    read_done();
    arrived<0>();  // the tiles' LDS is free, and no copy will write to it
    put_tile<BM, BN, WM, WN>(E(), a, out, acc, lds[0], m0, n0, wave, split, lane);
}

// The splits' sums added in turn, then put: eight outputs a thread.
template <typename E, typename Out>
__global__ __launch_bounds__(256) void mma_join_kernel(MmaArgs a, Out out)
{
    typedef typename Mma<E>::Sum Sum;
    const int per = (out.columns(a.n) + 7) / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = id / per;
    const int n = (int)(id - m * per) * 8;
    const typename Out::Mine mine = out.mine(n);  // by every lane of the wave
    if (id >= (int64_t)a.m * per) return;
    Sum v[2][8] = {};
    // four splits' loads at a time
    for (int s = 0; s < a.splits; s += 4) {
        Pack<Sum, 4> q[4][Out::PLANES][2];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int p = 0; p < Out::PLANES; ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    q[u][p][h] = load_row(
                        (const Sum *)a.part +
                            (((int64_t)min(s + u, a.splits - 1) * Out::PLANES + p) * a.m + m) * a.n,
                        n + h * 4, s + u < a.splits ? a.n : 0);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int p = 0; p < Out::PLANES; ++p)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[p][e] += q[u][p][e / 4].v[e % 4];
    }
    out.put(m, n, v[0], v[Out::PLANES - 1], mine, out.fetch(true, m, n));
}

template <typename E, bool A_CROSSED, bool B_CROSSED, typename Out>
hipError_t launch_mma(MmaArgs a, const MmaPlan &p, const Out &out, hipStream_t st)
{
    a.tiles_m = p.tiles_m;
    a.tiles_n = p.tiles_n;
    a.splits = p.splits;
    a.per_split = p.per_split;
    const unsigned blocks = (unsigned)(p.tiles_m * p.tiles_n * p.splits);
    if (p.large)
        mma_kernel<E, A_CROSSED, B_CROSSED, 256, 256, 2, 2, Out><<<blocks, 256, 0, st>>>(a, out);
    else
        mma_kernel<E, A_CROSSED, B_CROSSED, 128, 128, 2, 2, Out><<<blocks, 256, 0, st>>>(a, out);
    if (p.splits > 1) {
        const int64_t threads = (int64_t)a.m * ((out.columns(a.n) + 7) / 8);
        mma_join_kernel<E, Out><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(a, out);
    }
    return hipGetLastError();
}

}  // namespace kr
