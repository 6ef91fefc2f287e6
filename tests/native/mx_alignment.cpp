// Where the kernels load 16 bytes of a step of X that is not whole: word by word only from where a word begins, and otherwise the words that hold the
// entries, none of which lies wholly outside the row.  Memory is counted in entries of bfloat16 from an address that begins a word.
#include <stdio.h>

#include "../../paper_2108_12704_amd/csrc/hac_mx.h"

int main()
{
    using namespace hac_internal;
    constexpr uint32_t E = 8;
    unsigned long failures = 0, reads = 0, inside_a_word = 0;
    for (uint64_t X = 0; X < 2; ++X)                                     // X's first entry begins a word, or not
        for (uint32_t n = E; n <= 600; ++n)
            for (uint64_t ldx = n; ldx < n + 3; ++ldx)
                for (uint64_t row = 0; row < 2; ++row) {
                    const bool words = (X | ldx) % 2 == 0;               // every row begins at a word
                    const uint64_t first = X + row * ldx, end = first + n;
                    const MxShape s = mx_shape(n, 16);
                    for (uint64_t step = n / kMxTileRows; step < s.groups * kMxGroup; ++step) {
                        const uint64_t begin = step * kMxTileRows;
                        const uint32_t left = n > begin ? (uint32_t)(n - begin) : 0;
                        for (uint32_t k = 0; k < kMxTileRows; k += E) {
                            int32_t at;
                            if (!mx_piece_at(k, left, E, at)) continue;
                            ++reads;
                            const uint64_t from = (uint64_t)((int64_t)(first + begin) + at);
                            inside_a_word += words && from % 2;
                            if (mx_piece_words(at, E, words)) {
                                if (from % 2 && ++failures < 10) printf("X %llu n %u ldx %llu: 128 bits from entry %llu\n", (unsigned long long)X, n, (unsigned long long)ldx, (unsigned long long)from);
                                continue;
                            }
                            // four words and one more, from the word that holds entry `from` on: each has an entry of the row
                            const uint64_t odd = from % 2, lo = from - odd, more = lo + (odd ? 8 : 6);
                            if ((lo + 1 < first || lo + 6 >= end || more >= end) && ++failures < 10)
                                printf("X %llu n %u ldx %llu: words from entry %llu and at %llu\n", (unsigned long long)X, n, (unsigned long long)ldx, (unsigned long long)lo, (unsigned long long)more);
                        }
                    }
                }
    printf("%lu reads, %lu of them inside a word of a row that begins at one, %lu failures\n", reads, inside_a_word, failures);
    return failures != 0 || inside_a_word == 0;
}
