// Layout of an MX blob (microscaled 4-bit floating point), shared by host and device code.
//
// A block is 32 consecutive rows of one column.  With a = max |w| over the block the scale is 2^s, s = floor(log2 a) - 2 (at least
// -127), kept as the byte s + 127 (255: the block holds an infinity or NaN); an entry is the code of the nearest
// of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale (codes 0 .. 7, bit 3 the sign; ties to the even code, beyond 6 to 6).
//
// A tile is 16 columns x 128 rows, 1024 bytes: 64 pieces of 16 bytes, piece 16 g + c the block of column c and rows 32 g .. 32 g + 31,
// low half of a byte first.  That is the operand of v_mfma_scale_f32_16x16x128_f8f6f4 lane by lane, so a wavefront reads a tile with
// one 128-bit load per lane and multiplies what it has read.  The tiles of 16 columns follow one another down the rows, and
// their scales lie in groups of four tiles: 64 words of four bytes, byte t of word l the scale of piece l of tile t.
#ifndef HAC_MX_H
#define HAC_MX_H

#include <stdint.h>
#include <string.h>

#include "../../include/hac.h"

#if defined(__HIP__)
#define HAC_MX_BOTH __host__ __device__
#else
#define HAC_MX_BOTH
#endif

namespace hac_internal {

constexpr uint32_t kMxBlock = 32, kMxTileCols = 16, kMxTileRows = 128, kMxTileBytes = 1024, kMxGroup = 4, kMxGroupBytes = 256;
constexpr uint32_t kMxMaxCount = 65535;

struct MxShape {
    uint64_t steps, groups, ctiles;       // tiles down the rows, scale groups of them, tiles across the columns
    uint64_t code_bytes, scale_bytes;     // of one matrix
};

HAC_MX_BOTH inline MxShape mx_shape(uint64_t n, uint64_t m)
{
    MxShape s;
    s.steps = (n + kMxTileRows - 1) / kMxTileRows;
    s.groups = (s.steps + kMxGroup - 1) / kMxGroup;
    s.ctiles = (m + kMxTileCols - 1) / kMxTileCols;
    s.code_bytes = s.ctiles * s.steps * kMxTileBytes;
    s.scale_bytes = s.ctiles * s.groups * kMxGroupBytes;
    return s;
}

// where the block of rows 32 b .. of column j lies, from the start of its matrix's codes, and its scale, from that of its scales
HAC_MX_BOTH inline uint64_t mx_code_at(const MxShape& s, uint64_t b, uint64_t j)
{
    return ((j / 16 * s.steps + b / 4) * 64 + b % 4 * 16 + j % 16) * 16;
}
HAC_MX_BOTH inline uint64_t mx_scale_at(const MxShape& s, uint64_t b, uint64_t j)
{
    return ((j / 16 * s.groups + b / 16) * 64 + b % 4 * 16 + j % 16) * 4 + b / 4 % 4;
}

// Where to read the E entries that hold piece k ... k + E - 1 of a step of a row, of which the row has `left` >= 0 entries from the step's first on
// (a row of at least E): at k, or where the row's last E begin, which may be before the step.  false: nothing is left, nothing is to be read.
HAC_MX_BOTH inline bool mx_piece_at(uint32_t k, uint32_t left, uint32_t E, int32_t& at)
{
    const int32_t last = (int32_t)left - (int32_t)E;
    at = (int32_t)k < last ? (int32_t)k : last;
    return left != 0;
}

// Whether those E entries (4: of fp32, 8: of bfloat16) begin at a word, in rows of which every one does (words: or not).  A row of bfloat16 of odd length
// may have its last E begin inside one all the same.
HAC_MX_BOTH inline bool mx_piece_words(int32_t at, uint32_t E, bool words) { return words && (E == 4 || at % 2 == 0); }

// The header of `count` matrices of n x m; false where they are too many or too large.
inline bool mx_header(int64_t count, int64_t n, int64_t m, hac_desc_t& d)
{
    if (count < 1 || count > (int64_t)kMxMaxCount || n < 1 || m < 1 || n > 0x7fffff00ll || m > 0x7fffff00ll) return false;
    const MxShape s = mx_shape((uint64_t)n, (uint64_t)m);
    if (s.ctiles * s.steps > (1ull << 40) / kMxTileBytes / (uint64_t)count) return false;      // at most 2^40 bytes of codes
    memset(&d, 0, sizeof d);
    d.magic = 0x31434148u; d.version = 2; d.format = HAC_FORMAT_MX; d.header_bytes = 256;
    d.n = (uint64_t)n; d.m = (uint64_t)m;
    d.total_bits = 4ull * (uint64_t)count * d.n * d.m;
    d.k_sym = (uint32_t)count; d.ent_bits = 4; d.chunk = kMxBlock;
    d.off_codebook = sizeof(hac_desc_t);
    d.off_stream = d.off_codebook + (uint64_t)count * s.scale_bytes;
    d.blob_bytes = d.off_stream + (uint64_t)count * s.code_bytes;
    return true;
}

// true when d is what mx_header writes for its own sizes
inline bool mx_header_ok(const hac_desc_t& d)
{
    hac_desc_t want;
    return d.format == HAC_FORMAT_MX && d.n <= 0x7fffff00ull && d.m <= 0x7fffff00ull &&
           mx_header((int64_t)d.k_sym, (int64_t)d.n, (int64_t)d.m, want) && memcmp(&d, &want, sizeof d) == 0;
}

// the byte of the scale of a block whose largest magnitude has these bits (finite)
HAC_MX_BOTH inline uint32_t mx_scale_byte(uint32_t abs_bits)
{
    const uint32_t e = abs_bits >> 23;
    return e > 2 ? e - 2 : 0u;
}

} // namespace hac_internal

#endif
