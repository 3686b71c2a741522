// Launch arguments of the projections.
#pragma once

#include "kr_few.h"

namespace kr {

// Matrices to copy: rows of `bytes` bytes to rows of `to_ld` bytes (a multiple of 16), the rest
// of each filled with zeros.  All in one launch.
struct PadArgs {
    struct One {
        const char *from;
        int64_t from_ld, rows, bytes;
        char *to;
        int64_t to_ld;
    } m[3];
    int count;
};
hipError_t launch_pad(const PadArgs &a, hipStream_t st);

// gated.hip.  x [m][k], wg and wu [n][k] as operands that the tiles take, k_bytes of k a row.
struct GatedArgs {
    int type, act;
    int64_t m, n;             // rows, hidden
    int64_t k_bytes;
    Operand x, wg, wu;        // plain
    void *out;                // [m][n]
    int64_t ldo;
    void *part;               // gated_part bytes
};
size_t gated_part(int64_t m, int64_t n, int64_t k_bytes);
// x, wg, wu as they are: any alignment, a.x.bytes of k; no workspace.
hipError_t launch_gated_few(const GatedArgs &a, hipStream_t st);
hipError_t launch_gated(const GatedArgs &a, hipStream_t st);

struct GatedBackArgs {
    GatedArgs f;              // out, ldo unused
    int64_t width;            // k in elements
    const void *dh;
    int64_t ldh;
    char *d;                  // [m][2 n_pad]: dg, du, each padded with zeros to n_pad
    int64_t n_pad;
    char *tops;               // gated_back_tops bytes, or null where that is 0
    void *dx, *dwg, *dwu;
    int64_t lddx, lddg, lddu;
};
size_t gated_back_part(int64_t m, int64_t n, int64_t n_pad, int64_t width, int64_t k_bytes);
size_t gated_back_tops(int type);
hipError_t launch_gated_back(const GatedBackArgs &a, hipStream_t st);

// bytes.hip
struct BytesArgs {
    int out_type;
    int64_t m, n, k_bytes;
    Operand a, b;
    const float *sa, *sb;
    void *out;
    int64_t ldo;
    void *part;
};
size_t bytes_part(int64_t m, int64_t n, int64_t k_bytes);
hipError_t launch_bytes_few(const BytesArgs &a, hipStream_t st);
hipError_t launch_bytes(const BytesArgs &a, hipStream_t st);

}  // namespace kr
