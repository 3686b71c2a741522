// How rows are dealt to blocks by kernels that take them in groups of neighbours, and to launches.  Plain C++:
// the functions run on the host alone.
#pragma once

#include <stdint.h>

namespace kr {

// How a row's groups of neighbours, one a thread, are dealt to blocks of 256 threads: 2^log_tpr threads
// a row, the rows side by side, or `chunks` blocks to a row; of one to four waves those that leave the fewest
// threads without a group (258 groups: 64 threads five times, not 256 twice).
struct Dealt {
    uint32_t log_tpr, groups, chunks;
};
inline Dealt dealt(int64_t groups)
{
    uint32_t log = 0;
    while (log < 8 && ((int64_t)1 << log) < groups) ++log;
    auto chunks = [&](uint32_t l) { return (groups + (1 << l) - 1) >> l; };
    for (uint32_t l = log; l-- > 6;)
        if (chunks(l) << l < chunks(log) << log) log = l;
    return {log, (uint32_t)groups, (uint32_t)chunks(log)};
}

// Rows of one launch: a grid has fewer than 2^32 threads, and these have 2^31 at most (a row has no more
// than 2^23 blocks: 2^31 groups).
inline int64_t dealt_rows(Dealt s)
{
    const int64_t most = ((int64_t)1 << 23) / s.chunks;
    return (most > 1 ? most : 1) << (8 - s.log_tpr);
}
// Blocks of a launch of so many rows.
inline int64_t dealt_blocks(Dealt s, int64_t rows)
{
    return ((rows + (256 >> s.log_tpr) - 1) >> (8 - s.log_tpr)) * s.chunks;
}

}  // namespace kr
