// Where the kernels read a step of X that is not whole: inside the row, and every entry of it that a piece holds.
#include <stdio.h>

#include "../../paper_2108_12704_amd/csrc/hac_mx.h"

int main()
{
    using namespace hac_internal;
    unsigned long failures = 0, reads = 0;
    for (uint32_t E = 4; E <= 8; E *= 2)
        for (uint32_t n = E; n <= 1200; ++n) {
            const MxShape s = mx_shape(n, 16);
            for (uint64_t step = 0; step < s.groups * kMxGroup; ++step) {              // laid out: up to a whole group of steps
                const uint32_t first = (uint32_t)step * kMxTileRows, left = n > first ? n - first : 0;
                if (left >= kMxTileRows) continue;
                for (uint32_t k = 0; k < kMxTileRows; k += E) {
                    int32_t at;
                    if (!mx_piece_at(k, left, E, at)) { failures += left != 0; continue; }
                    ++reads;
                    const int64_t from = (int64_t)first + at;
                    const bool inside = from >= 0 && from + E <= n;
                    const bool whole = k >= left || (at <= (int32_t)k && at + (int32_t)E >= (int32_t)(k + E < left ? k + E : left));
                    if (!inside || !whole) {
                        if (++failures < 10) printf("E %u n %u step %llu piece %u: reads %lld ...\n", E, n, (unsigned long long)step, k, (long long)from);
                    }
                }
            }
        }
    printf("%lu reads, %lu failures\n", reads, failures);
    return failures != 0;
}
