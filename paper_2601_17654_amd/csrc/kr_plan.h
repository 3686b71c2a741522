// How a tiled product is cut into tiles and splits of its sum.  Host code alone, plain C++.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace kr {

struct MmaPlan {
    bool large;   // 256 x 256 tiles, else 128 x 128
    int tiles_m, tiles_n, splits, per_split;
    int64_t part_bytes;
};

// The cheaper of the two tile sizes, and of up to 16 splits of the sum, by an estimate in
// microseconds.  256 x 256: 1.3 a step and 9 for what surrounds them, one tile a CU at a time.
// 128 x 128: 0.94 and 4, two a CU, so that half a round is one each.  A split adds its partial
// sums, written and read at 4 TB/s, and a launch.  Measured, bfloat16, two planes (large / small):
//   4096 x 4096 x 2048   118 / 135 us        4096 x 2176 x 4096   173 / 141 us
//   1024 x 14336 x 4096  185 / 213 us        2048 x 2048 x 512     21 / 14 us
//   700 x 8192 x 8192    163 / 190 us        3000 x 6000 x 1500   144 / 138 us
// All of these have 512 small tiles or more.  Of fewer, with short sums, the estimate is low: 120
// tiles of 17 steps (333 x 5001 x 2059 in 8 bits) 10 us, measured 15.5; 387 tiles of 17 steps (the
// gradient of 1111 x 1030 -> 2731) 20 us, measured 28.
inline MmaPlan mma_plan(int64_t m, int64_t n, int planes, int steps)
{
    MmaPlan best{};
    double least = 0;
    for (const bool large : {true, false}) {
        const int bm = large ? 256 : 128, bn = bm / planes;
        const int64_t tm = (m + bm - 1) / bm, tn = (n + bn - 1) / bn;
        for (int s = 1; s <= 16 && (s == 1 || (steps + s - 1) / s >= 4); ++s) {
            const int per = steps > 0 ? (steps + s - 1) / s : 1;
            const int splits = steps > 0 ? (steps + per - 1) / per : 1;
            if (splits != s) continue;
            const int64_t rounds = (tm * tn * s + 255) / 256;
            const double part = s > 1 ? 4.0 * s * planes * m * n : 0;
            const double cost = rounds * (large ? 1.3 * per + 9 : 0.47 * per + 2) +
                                (s > 1 ? 4 + 2 * part / 4e6 : 0);
            if (best.tiles_m && cost >= least) continue;
            least = cost;
            best = {large, (int)tm, (int)tn, s, per, (int64_t)part};
        }
    }
    return best;
}

}  // namespace kr
