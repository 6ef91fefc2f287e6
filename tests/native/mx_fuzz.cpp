// Host-side robustness driver for 4-bit blobs, meant to be built with -fsanitize=address,undefined: encodes matrices of odd shapes, several to a
// blob too, checks the values against the format's definition, then damages the blobs (bit flips, header bytes and fields, truncation) and runs header
// checks, validator, statistics and decoder on them.  Whatever they answer, they must not read or write out of bounds.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "../../include/hac.h"

// the entry nearest to v among a block's, whose largest magnitude is `most`
static float nearest(float v, float most)
{
    int e = 0;
    std::frexp((double)most, &e);                                        // most = f 2^e, 0.5 <= f < 1
    const int s = most == 0.0f ? -127 : (e - 3 < -127 ? -127 : e - 3);
    const double grid[8] = { 0, 0.5, 1, 1.5, 2, 3, 4, 6 }, u = std::ldexp(std::fabs((double)v), -s);
    int best = 0;
    for (int i = 1; i < 8; ++i) {
        const double a = std::fabs(grid[i] - u), b = std::fabs(grid[best] - u);
        if (a < b || (a == b && i % 2 == 0)) best = i;
    }
    return (float)std::copysign(std::ldexp(grid[best], s), v);
}

static int exercise(const void* blob, size_t bytes, size_t entries, const std::vector<float>* expect)
{
    hac_desc_t d;
    const int described = hac_describe(blob, bytes, &d);
    const int deep = hac_validate(blob, bytes, 1), shallow = hac_validate(blob, bytes, 0);
    hac_stats_t st;
    const int counted = hac_stats(blob, bytes, &st);
    if ((described != HAC_OK && (deep == HAC_OK || shallow == HAC_OK || counted == HAC_OK)) || (shallow != HAC_OK && deep == HAC_OK)) {
        std::fprintf(stderr, "answers contradict one another: %d %d %d %d\n", described, shallow, deep, counted);
        return 1;
    }
    if (described != HAC_OK || d.format != HAC_FORMAT_MX || (uint64_t)d.k_sym * d.n * d.m > entries) return 0;     // do not size buffers from a damaged header
    std::vector<float> W((size_t)d.k_sym * d.n * d.m, -1.0f);
    std::vector<int32_t> sym(W.size());
    const int rc = hac_decode_host(blob, bytes, W.data(), sym.data(), nullptr, nullptr);
    hac_decode_host(blob, bytes, W.data(), nullptr, nullptr, nullptr);
    hac_decode_host(blob, bytes, nullptr, sym.data(), nullptr, nullptr);
    if (!expect) return 0;
    if (deep != HAC_OK || counted != HAC_OK || rc != HAC_OK || std::memcmp(W.data(), expect->data(), W.size() * 4) != 0) {
        std::fprintf(stderr, "round trip failed: %d %d %d\n", deep, counted, rc);
        return 1;
    }
    return 0;
}

int main()
{
    std::mt19937 rng(4321);
    int failures = 0;
    long cases = 0;
    const int shapes[][3] = { {1, 1, 1}, {1, 31, 3}, {1, 33, 17}, {1, 128, 16}, {1, 513, 5}, {1, 2000, 40}, {2, 1, 1}, {3, 100, 20}, {7, 129, 33}, {300, 5, 2} };
    for (const auto& sh : shapes)
        for (int kind = 0; kind < 3; ++kind)
            for (int pad = 0; pad < 2; ++pad) {
                const size_t count = sh[0], n = sh[1], m = sh[2], ldw = m + 3 * pad, stride = n * ldw + 5 * pad;
                // exactly as much memory as the matrices take, so that any read past them is caught
                const size_t room = (count - 1) * stride + (n - 1) * ldw + m;
                float* W = (float*)std::malloc(room * sizeof(float));
                std::normal_distribution<double> normal;
                for (size_t i = 0; i < room; ++i)
                    W[i] = (float)std::ldexp(normal(rng), kind == 0 ? 0 : kind == 1 ? (int)(rng() % 276) - 149 : -(int)(rng() % 2) * 140) * (rng() % 8 ? 1.0f : 0.0f);
                for (size_t i = 0; i < room; ++i) if (!std::isfinite(W[i])) W[i] = 1.0f;
                std::vector<float> expect(count * n * m);
                for (size_t e = 0; e < count; ++e)
                    for (size_t j = 0; j < m; ++j)
                        for (size_t b = 0; b < n; b += 32) {
                            const size_t end = b + 32 < n ? b + 32 : n;
                            float most = 0.0f;
                            for (size_t i = b; i < end; ++i) most = std::fmax(most, std::fabs(W[e * stride + i * ldw + j]));
                            for (size_t i = b; i < end; ++i) expect[(e * n + i) * m + j] = nearest(W[e * stride + i * ldw + j], most);
                        }
                void* blob = nullptr; size_t bytes = 0;
                const int rc = mx_encode(W, (int64_t)count, (int64_t)n, (int64_t)m, (int64_t)ldw, (int64_t)stride, &blob, &bytes);
                std::free(W);
                if (rc != HAC_OK) { std::fprintf(stderr, "encode failed: %d\n", rc); ++failures; continue; }
                failures += exercise(blob, bytes, expect.size(), &expect);
                ++cases;
                const std::vector<uint8_t> copy((const uint8_t*)blob, (const uint8_t*)blob + bytes);
                hac_free(blob);
                for (int t = 0; t < 150; ++t) {
                    std::vector<uint8_t> bad = copy;
                    const int how = (int)(rng() % 6);
                    if (how == 0) bad[rng() % bad.size()] ^= (uint8_t)(1u << (rng() % 8));
                    else if (how == 1) bad[rng() % 256] = (uint8_t)rng();                        // the header
                    else if (how == 2) { for (int q = 0; q < 8; ++q) bad[rng() % bad.size()] = (uint8_t)rng(); }
                    else if (how == 3) bad.resize(rng() % bad.size());
                    else if (how == 4) {                                                         // a header that is whole, for other sizes than the blob's
                        hac_desc_t d;
                        const int64_t k = 1 + (int64_t)(rng() % 400), r = 1 + (int64_t)(rng() % 3000), c = 1 + (int64_t)(rng() % 60);
                        if (mx_describe(k, r, c, &d) == HAC_OK) std::memcpy(bad.data(), &d, sizeof d);
                    } else {                                                                     // a field at an end of its range
                        const uint64_t ends[] = { 0, 1, 0x7fffff00ull, 0x7fffffffull, 0xffffffffull, 1ull << 32, 1ull << 40, ~0ull };
                        std::memcpy(bad.data() + 8 * (rng() % 32), &ends[rng() % 8], 8);
                    }
                    uint8_t* heap = (uint8_t*)std::malloc(bad.size() ? bad.size() : 1);
                    std::memcpy(heap, bad.data(), bad.size());
                    failures += exercise(heap, bad.size(), 1u << 22, nullptr);
                    std::free(heap);
                    ++cases;
                }
            }
    // the last sizes that a header can have, and the first that it cannot
    const int64_t ends[] = { 0, 1, 65535, 65536, 1 << 20, 0x7fffff00ll, 0x7fffff01ll, INT64_MAX, INT64_MIN, -1 };
    for (int64_t k : ends)
        for (int64_t n : ends)
            for (int64_t m : ends) {
                hac_desc_t d;
                const int rc = mx_describe(k, n, m, &d);
                if (rc == HAC_OK && hac_validate(&d, sizeof d, 1) == HAC_OK) { std::fprintf(stderr, "a header alone is no blob\n"); ++failures; }
                ++cases;
            }
    std::printf("mx fuzz: %ld cases, %d failures\n", cases, failures);
    return failures ? 1 : 0;
}
