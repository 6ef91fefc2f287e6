// 4-bit microscaled layers on gfx950 (MI355X): quantisation, its inverse, the product and the product grouped by expert.
// Formulas and layout: include/hac.h (mx_encode) and hac_mx.h.
//
// Lane layouts used below.  v_mfma_scale_f32_16x16x128_f8f6f4 on 4-bit operands: lane l holds row (column) l % 16 and the 32 k
// 32 (l / 16) ..., which is a block, and one byte of a register as its scale; v_mfma_f32_16x16x32_bf16: eight k.  The order of k is free
// as long as both operands agree, so a tile of W (16 columns x 128 k) is four bf16 operands: operand j multiplies the k
// 32 (l / 16) + 8 j ... + 7.  W is the first operand: a lane's four sums are then four neighbouring columns of one row of Y.
// The conversions v_cvt_scalef32_pk_* take the scale's exponent field alone: 0 is 2^-127 there, as in a scale byte.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "hac_hostlib.h"
#include "hac_internal.h"
#include "hac_mx.h"

using namespace hac_internal;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 word4 __attribute__((aligned(4)));                   // global memory takes 128-bit loads at any word
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
#define ALWAYS_INLINE __attribute__((always_inline))

// how X enters the matrix instructions: quantised, as bf16, as three bf16 parts of an fp32
enum Mode { FP4 = 0, ONE = 1, THREE = 3 };

struct MxW {
    const uint8_t *codes, *scales;
    uint64_t code_stride, scale_stride;      // bytes from one matrix to the next
    uint32_t n, m, steps, groups, ctiles, count;
};

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ bf16x2 pair(uint32_t word) { return __builtin_bit_cast(bf16x2, word); }   // (of a copy: not of a vector's element)

// ---- 32 entries of a row of X ------------------------------------------------------------

// Exchanges lane bit 5 (4) with the choice between two registers: a keeps its lower half (even rows of 16 lanes) and gets b's as its upper half.
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0]; b = r[1];
}
__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0]; b = r[1];
}

// load_step: lane 16 g + c has row c and wants its entries 32 g ... of a step of 128.  Read that way, a load of 16 bytes a lane touches 64 lines; so
// the four lanes of a row read 64 bytes side by side and then exchange pieces.
// 16 bytes of a row from any entry on.  Loads that start at a word are as quick as aligned ones, loads that start inside a word several times
// slower; so where entries of bfloat16 may (not `words`), the words that hold them are read and shifted.  A word that holds an entry is
// readable as a whole.  (301 x 400, 64 rows: 3.5 us with every second row inside a word, 3.1 with the ends of rows alone, 302 x 400 2.8.)
template <typename T> __device__ __forceinline__ bool whole_words(const T* X, uint64_t ldx)      // every row begins at a word
{
    return sizeof(T) == 4 || ((reinterpret_cast<uintptr_t>(X) | 2 * ldx) & 3) == 0;
}
__device__ __forceinline__ u32x4 load16(const float* p, bool) { return *reinterpret_cast<const word4*>(p); }
__device__ __forceinline__ u32x4 load16(const __bf16* p, bool words)
{
    if (words) return *reinterpret_cast<const word4*>(p);
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), odd = at & 2;
    const u32x4 q = *reinterpret_cast<const word4*>(at - odd);
    const uint32_t e = *reinterpret_cast<const uint32_t*>(at - odd + (odd ? 16 : 12));
    return odd ? u32x4{q.x >> 16 | q.y << 16, q.y >> 16 | q.z << 16, q.z >> 16 | q.w << 16, q.w >> 16 | e << 16} : q;
}

// 16 bytes from entry k of a step on, of which the row has `left` entries, zeros behind: the row's last 16 bytes, moved down by the entries that
// come before k, where they end first.  One load whatever k is, so that no lane waits for another's.  (A row of less than 16 bytes: entry by entry.)
template <typename T> __device__ __forceinline__ u32x4 piece_of(const T* row, uint32_t k, uint32_t left, uint32_t n, bool words)
{
    constexpr int E = 16 / sizeof(T);
    u32x4 p = {0, 0, 0, 0};
    if (n < (uint32_t)E) {
        for (uint32_t i = 0; i < (uint32_t)E && k + i < left; ++i) {
            if constexpr (E == 4) { if (i == 0) p.x = __float_as_uint(row[k]); else if (i == 1) p.y = __float_as_uint(row[k + 1]); else p.z = __float_as_uint(row[k + 2]); }
            else {
                const uint32_t v = (uint32_t)reinterpret_cast<const uint16_t*>(row)[k + i] << (16 * (i & 1));
                if (i < 2) p.x |= v; else if (i < 4) p.y |= v; else if (i < 6) p.z |= v; else p.w |= v;
            }
        }
        return p;
    }
    int32_t at;
    if (!mx_piece_at(k, left, E, at)) return p;
    const int d = (int)k - at;
    p = load16(row + at, mx_piece_words(at, E, words));
    if constexpr (E == 8) {
        if (d & 1) p = u32x4{p.x >> 16 | p.y << 16, p.y >> 16 | p.z << 16, p.z >> 16 | p.w << 16, p.w >> 16};
    }
    const int moved = d / (E / 4);                                  // in words
    if (moved & 1) p = u32x4{p.y, p.z, p.w, 0};
    if (moved & 2) p = u32x4{p.z, p.w, 0, 0};
    if (moved >= 4) p = u32x4{0, 0, 0, 0};
    return p;
}

template <typename T> struct Block32;
template <> struct Block32<float> {
    f32x4 v[8];
    __device__ __forceinline__ void load_step(const float* row, uint32_t g, bool words)
    {
        u32x4 p[8];                                                  // piece 4 i + g of the row's 32
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = load16(row + 16 * i + 4 * g, words);
        exchange(p);
    }
    __device__ __forceinline__ void load_step(const float* row, uint32_t g, bool words, uint32_t left, uint32_t n)      // ... of which the first `left` are there
    {
        u32x4 p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = piece_of(row, 16 * i + 4 * g, left, n, words);
        exchange(p);
    }
    __device__ __forceinline__ void exchange(u32x4* p)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) { uint32_t a = p[i][e], b = p[i + 4][e]; swap32(a, b); p[i][e] = a; p[i + 4][e] = b; }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i & 2) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) { uint32_t a = p[i][e], b = p[i + 2][e]; swap16(a, b); p[i][e] = a; p[i + 2][e] = b; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(f32x4, p[(i & 2) << 1 | (i & 1) << 1 | i >> 2]);
        // (register 4 p1 + 2 p0 + p2 has piece 8 g + 4 p2 + 2 p1 + p0)
    }
    __device__ __forceinline__ uint32_t most() const                             // bits of the largest magnitude
    {
        // (as integers the largest of the positive ones, and of all: a negative one's pattern is above every positive one's)
        int32_t up = 0;
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            up = max(up, (int32_t)__float_as_uint(v[i / 4][i % 4]));
            any = max(any, __float_as_uint(v[i / 4][i % 4]));
        }
        return max((uint32_t)up, any & 0x7fffffffu);
    }
    __device__ __forceinline__ u32x4 codes(float scale) const
    {
        u32x4 c;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t r = 0;
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2 * w].x, v[2 * w].y, scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2 * w].z, v[2 * w].w, scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2 * w + 1].x, v[2 * w + 1].y, scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2 * w + 1].z, v[2 * w + 1].w, scale, 3);
            c[w] = r;
        }
        return c;
    }
    // entries 8 j ... 8 j + 7 as three bf16 parts, cut off: x = x1 + x2 + x3 exactly (8 bits each), down to 2^-133.
    // An infinity is its first part alone.
    __device__ __forceinline__ void parts(int j, u32x4* p) const
    {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint32_t w[3][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float x = v[2 * j + h / 2][2 * (h % 2) + i];
                const uint32_t x1 = __float_as_uint(x) & 0xffff0000u;
                const float r1 = fabsf(x) == __builtin_inff() ? 0.0f : x - __uint_as_float(x1);
                const uint32_t x2 = __float_as_uint(r1) & 0xffff0000u;
                w[0][i] = x1; w[1][i] = x2;
                w[2][i] = __float_as_uint(r1 - __uint_as_float(x2));
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) p[q][h] = __builtin_amdgcn_perm(w[q][1], w[q][0], 0x07060302u);
        }
    }
};
template <> struct Block32<__bf16> {
    u32x4 v[4];
    __device__ __forceinline__ void load_step(const __bf16* row, uint32_t g, bool words)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = load16(row + 32 * i + 8 * g, words);       // piece 4 i + g of 16
        exchange();
    }
    __device__ __forceinline__ void load_step(const __bf16* row, uint32_t g, bool words, uint32_t left, uint32_t n)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = piece_of(row, 32 * i + 8 * g, left, n, words);
        exchange();
    }
    __device__ __forceinline__ void exchange()
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) { uint32_t a = v[i][e], b = v[i + 2][e]; swap32(a, b); v[i][e] = a; v[i + 2][e] = b; }
#pragma unroll
        for (int i = 0; i < 4; i += 2)
#pragma unroll
            for (int e = 0; e < 4; ++e) { uint32_t a = v[i][e], b = v[i + 1][e]; swap16(a, b); v[i][e] = a; v[i + 1][e] = b; }
    }
    __device__ __forceinline__ uint32_t most() const
    {
        u16x2 a = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t w = v[i / 4][i % 4] & 0x7fff7fffu;
            a = __builtin_elementwise_max(a, __builtin_bit_cast(u16x2, w));
        }
        return (uint32_t)max(a.x, a.y) << 16;
    }
    __device__ __forceinline__ u32x4 codes(float scale) const
    {
        u32x4 c;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t r = 0;
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(v[w].x), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(v[w].y), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(v[w].z), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(v[w].w), scale, 3);
            c[w] = r;
        }
        return c;
    }
    __device__ __forceinline__ void parts(int j, u32x4* p) const { p[0] = v[j]; }
};

// A block's scale byte and codes; with a NaN or infinity in it: byte 255, codes 0.
template <typename T> __device__ __forceinline__ u32x4 quantise(const Block32<T>& x, uint32_t& byte)
{
    const uint32_t a = x.most();
    byte = mx_scale_byte(a);
    u32x4 c = x.codes(scale_of(byte));
    if (a >= 0x7f800000u) { byte = 255; c = u32x4{0, 0, 0, 0}; }
    return c;
}

// eight codes of W as bf16 (exact)
__device__ __forceinline__ bf16x8 weights(uint32_t word, float scale)
{
    const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
    const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
    const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
    const uint32_t d = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
    return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d});
}

__device__ __forceinline__ i32x8 operand(u32x4 c) { return i32x8{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}; }

template <int BYTE> __device__ __forceinline__ f32x4 multiply_fp4(u32x4 w, uint32_t ws, u32x4 x, uint32_t xs, f32x4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w), operand(x), acc, 4, 4, BYTE, (int)ws, BYTE, (int)xs);
}
__device__ __forceinline__ f32x4 multiply_bf16(bf16x8 w, u32x4 x, f32x4 acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
}

// ---- groups of rows ------------------------------------------------------------------------

// A stretch of at most R rows of one group: matrix, first row, rows (0: there is none), and the number of tiles of 16 rows in the
// groups and stretches before it.
struct Item { uint32_t expert, row0, rows, tile; };

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// Stretch `item`; all lanes of a wavefront call it with the same arguments.  Offsets are read a wavefront's width at a time, and held to
// 0 .. B, so that rows lie inside X and Y whatever they are.
__device__ __forceinline__ Item find_item(const int32_t* __restrict__ offsets, uint32_t count, uint32_t B, uint32_t R, uint32_t item)
{
    if (!offsets) {
        const uint32_t row0 = item * R;
        return Item{0u, row0, row0 < B ? min(R, B - row0) : 0u, item * (R / 16)};
    }
    const uint32_t lane = threadIdx.x & 63;
    uint32_t items = 0, tiles = 0;
    for (uint32_t base = 0; base < count; base += 64) {
        const uint32_t e = base + lane;
        int32_t a = 0, b = 0;
        if (e < count) { a = offsets[e]; b = offsets[e + 1]; }
        a = min(max(a, 0), (int32_t)B); b = min(max(b, 0), (int32_t)B);
        const uint32_t rows = b > a ? (uint32_t)(b - a) : 0u;
        const uint32_t mine = (rows + R - 1) / R, mine16 = (rows + 15) / 16;
        uint32_t upto = mine, upto16 = mine16;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t u = __shfl_up(upto, d), v = __shfl_up(upto16, d);
            if (lane >= (uint32_t)d) { upto += u; upto16 += v; }
        }
        const unsigned long long past = __ballot(items + upto > item);
        if (past) {
            const int f = __builtin_ctzll(past);
            const uint32_t within = item - (items + __shfl(upto, f) - __shfl(mine, f));
            const uint32_t r = __shfl(rows, f), row0 = (uint32_t)__shfl(a, f) + within * R;
            const uint32_t tile = tiles + __shfl(upto16, f) - __shfl(mine16, f) + within * (R / 16);
            return Item{uniform(base + (uint32_t)f), uniform(row0), uniform(min(R, r - within * R)), uniform(tile)};
        }
        items += __shfl(upto, 63); tiles += __shfl(upto16, 63);
    }
    return Item{0u, 0u, 0u, 0u};
}

// four neighbouring columns of a row of Y (col < m is the first)
template <typename T> __device__ __forceinline__ void store4(T* y, uint32_t col, uint32_t m, bool wide, f32x4 v)
{
    if (wide && col + 4 <= m) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(y + col) = v;
        else *reinterpret_cast<bf16x4*>(y + col) = bf16x4{(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < m) y[col + i] = (T)v[i];
}

// eight, of which `left` are inside the row, as bfloat16
__device__ __forceinline__ void store8(__bf16* y, uint32_t left, u32x4 v)
{
    if (left >= 8) *reinterpret_cast<u32x4*>(y) = v;
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((uint32_t)i < left) reinterpret_cast<uint16_t*>(y)[i] = (uint16_t)(v[i / 2] >> 16 * (i & 1));
}

// ---- quantisation and its inverse ------------------------------------------------------------
// A thread has a block: 32 rows of one column, so that the 64 lanes of a wavefront read 64 neighbouring columns row by row and need
// no exchange.  A block of threads covers 64 columns x 512 rows, a group of scales: their bytes meet in LDS.  Bound by memory.
// STREAM: past the last-level cache, for W larger than that.  25088 x 4096 of fp32 (411 MB) are encoded in 87 us (5.3 TB/s of a copy's 5.1) and decoded in
// 80, not streamed in 98 and 93, one after the other in 168 and 197; 16 x 1024 x 2048 of bfloat16 (67 MB) one after the other in 35 with streamed
// loads, 30 without, and whoever reads the values next finds them in the cache.  (Two columns a thread: 230 and 34.)
constexpr uint64_t kCacheBytes = 256ull << 20;
constexpr uint32_t kCodeCols = 64, kCodeRows = 512;

template <typename T, bool STREAM>
__global__ void __launch_bounds__(1024)
mx_encode_kernel(const T* __restrict__ W, uint64_t ldw, uint64_t stride, MxW w, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                 uint8_t* __restrict__ header, hac_desc_t desc)
{
    __shared__ uint8_t bytes[kCodeCols * 16];
    const uint32_t c = threadIdx.x & 63, b = threadIdx.x >> 6;               // column, block of rows
    const uint64_t e = blockIdx.z;
    const uint32_t j = blockIdx.x * kCodeCols + c, group = blockIdx.y, step = group * 4 + b / 4;
    const uint32_t k = group * kCodeRows + 32 * b;
    if (header && blockIdx.x == 0 && group == 0 && e == 0 && threadIdx.x < 64)
        reinterpret_cast<uint32_t*>(header)[threadIdx.x] = reinterpret_cast<const uint32_t*>(&desc)[threadIdx.x];
    Block32<float> x;
    const T* p = W + e * stride + (uint64_t)k * ldw + j;
    if (j < w.m && k + 32 <= w.n) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x.v[i / 4][i % 4] = (float)(STREAM ? __builtin_nontemporal_load(p + (uint64_t)i * ldw) : p[(uint64_t)i * ldw]);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) x.v[i / 4][i % 4] = j < w.m && k + i < w.n ? (float)p[(uint64_t)i * ldw] : 0.0f;
    }
    uint32_t byte;
    const u32x4 q = quantise(x, byte);
    const uint32_t ct = j / 16, lane = b % 4 * 16 + j % 16;
    if (ct < w.ctiles && step < w.steps)
        *reinterpret_cast<u32x4*>(codes + e * w.code_stride + (((uint64_t)ct * w.steps + step) * 64 + lane) * 16) = q;
    // word (tile of columns, lane) of the group, byte step
    bytes[((c / 16) * 64 + lane) * 4 + b / 4] = (uint8_t)byte;
    __syncthreads();
    if (threadIdx.x < 256) {
        const uint32_t t = threadIdx.x / 64, at = blockIdx.x * 4 + t;
        if (at < w.ctiles)
            reinterpret_cast<uint32_t*>(scales + e * w.scale_stride)[((uint64_t)at * w.groups + group) * 64 + threadIdx.x % 64] =
                reinterpret_cast<const uint32_t*>(bytes)[threadIdx.x];
    }
}

template <typename T, bool STREAM>
__global__ void __launch_bounds__(1024)
mx_decode_kernel(T* __restrict__ W, uint64_t ldw, uint64_t stride, MxW w)
{
    const uint32_t c = threadIdx.x & 63, b = threadIdx.x >> 6;
    const uint64_t e = blockIdx.z;
    const uint32_t j = blockIdx.x * kCodeCols + c, group = blockIdx.y, step = group * 4 + b / 4;
    const uint32_t k = group * kCodeRows + 32 * b;
    if (j >= w.m || k >= w.n) return;
    const uint32_t ct = j / 16, lane = b % 4 * 16 + j % 16;
    const u32x4 q = *reinterpret_cast<const u32x4*>(w.codes + e * w.code_stride + (((uint64_t)ct * w.steps + step) * 64 + lane) * 16);
    const uint32_t byte = w.scales[e * w.scale_stride + (((uint64_t)ct * w.groups + group) * 64 + lane) * 4 + b / 4];
    const float s = scale_of(byte);
    T* p = W + e * stride + (uint64_t)k * ldw + j;
    float v[32];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], s, 0);
        v[8 * i] = a.x; v[8 * i + 1] = a.y;
        a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], s, 1);
        v[8 * i + 2] = a.x; v[8 * i + 3] = a.y;
        a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], s, 2);
        v[8 * i + 4] = a.x; v[8 * i + 5] = a.y;
        a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], s, 3);
        v[8 * i + 6] = a.x; v[8 * i + 7] = a.y;
    }
    const uint32_t rows = min(32u, w.n - k);
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if ((uint32_t)i < rows) {
            const T value = (T)(byte == 255 ? __builtin_nanf("") : v[i]);
            if constexpr (STREAM) __builtin_nontemporal_store(value, p + (uint64_t)i * ldw);
            else p[(uint64_t)i * ldw] = value;
        }
}

// ---- few rows, or little work ------------------------------------------------------------------
// 16 rows of X at a time: what counts is to have everything in flight at once and to launch one kernel.  A block owns 16 rows and NC tiles of
// columns (and, with splits, a range of k), its wavefronts share the steps, each reads its tiles of W straight into operands; X comes from memory
// (from the L2 after the first block), is turned into parts or quantised by the lane that holds the block, and the wavefronts' sums are
// added in LDS in order.  A lane past the last row reads that row again: what it adds goes to sums that nobody stores.
// Bound by the launch and the first trips to memory where there is little work (4096 x 4096, one row of bfloat16: 4.8 us, the 8.9 MB of W alone
// 1.8; 64 experts of 2048 x 1408, 64 rows: 13, the W of those that have rows 8.6), by the turning of X into operands, which every block of columns
// repeats, where there is more: from some hundreds of rows on tiles are quicker, and the estimates below say which.
template <int MODE, typename T, int NC, int U>
__global__ void __launch_bounds__(512)
mx_rows_kernel(MxW w, const T* __restrict__ X, uint64_t ldx, uint32_t B, const int32_t* __restrict__ offsets,
               T* __restrict__ Y, uint64_t ldy, uint32_t each, uint32_t more, float* __restrict__ part)
{
    extern __shared__ __align__(16) f32x4 red[];                 // [wavefronts][NC][64]
    const uint32_t lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, lane16 = 16 * lane, lane4 = 4 * lane;
    const uint32_t wave = uniform(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t cb = blockIdx.x, split = blockIdx.z, splits = gridDim.z;
    const Item it = find_item(offsets, w.count, B, 16, blockIdx.y);
    if (!it.rows) return;
    // every wavefront of every split has `each` steps, the first `more` of them one more
    const uint32_t share = split * waves + wave, s0 = share * each + min(share, more), s1 = s0 + each + (share < more ? 1u : 0u);
    const uint8_t* code[NC];
    const uint8_t* scale[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
        const uint32_t ct = min(cb * NC + q, w.ctiles - 1);
        code[q] = w.codes + it.expert * w.code_stride + (uint64_t)ct * w.steps * 1024;
        scale[q] = w.scales + it.expert * w.scale_stride + (uint64_t)ct * w.groups * 256;
    }
    const T* row = X + (uint64_t)(it.row0 + min(c, it.rows - 1)) * ldx;
    const bool words = whole_words(X, ldx);
    f32x4 acc[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) acc[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto load_w = [&](uint32_t step, u32x4* codes, uint32_t* byte) ALWAYS_INLINE {
#pragma unroll
        for (int q = 0; q < NC; ++q) {
            codes[q] = *reinterpret_cast<const u32x4*>(code[q] + (uint64_t)step * 1024 + lane16);
            byte[q] = *(scale[q] + (uint64_t)(step / 4) * 256 + step % 4 + lane4);
        }
    };
    auto multiply = [&](const Block32<T>& x, const u32x4* codes, const uint32_t* byte) ALWAYS_INLINE {
        if constexpr (MODE == FP4) {
            uint32_t xs;
            const u32x4 xc = quantise(x, xs);
#pragma unroll
            for (int q = 0; q < NC; ++q) acc[q] = multiply_fp4<0>(codes[q], byte[q], xc, xs, acc[q]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4 p[MODE];
                x.parts(j, p);
#pragma unroll
                for (int q = 0; q < NC; ++q) {
                    const bf16x8 v = weights(codes[q][j], scale_of(byte[q]));
#pragma unroll
                    for (int i = MODE - 1; i >= 0; --i) acc[q] = multiply_bf16(v, p[i], acc[q]);
                }
            }
        }
    };
    // U steps at a time are requested before the first is multiplied (behind the last: that one again, not multiplied)
    const uint32_t full = min(s1, w.n / 128);
    for (uint32_t s = s0; s < full; s += U) {
        Block32<T> x[U];
        u32x4 codes[U][NC];
        uint32_t byte[U][NC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t step = min(s + u, full - 1);
            load_w(step, codes[u], byte[u]);
            x[u].load_step(row + (uint64_t)step * 128, g, words);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s + u >= full) break;
            multiply(x[u], codes[u], byte[u]);
        }
    }
    if (max(full, s0) < s1) {                                    // a last step that is not whole
        Block32<T> x;
        u32x4 codes[NC];
        uint32_t byte[NC];
        load_w(s1 - 1, codes, byte);
        x.load_step(row + (uint64_t)(s1 - 1) * 128, g, words, w.n - (s1 - 1) * 128, w.n);
        multiply(x, codes, byte);
    }
#pragma unroll
    for (int q = 0; q < NC; ++q) red[((size_t)wave * NC + q) * 64 + lane] = acc[q];
    __syncthreads();
    const bool wide = (reinterpret_cast<uintptr_t>(Y) | ldy * sizeof(T)) % (4 * sizeof(T)) == 0;
    for (uint32_t o = threadIdx.x; o < NC * 64; o += blockDim.x) {
        f32x4 v = red[o];
        for (uint32_t z = 1; z < waves; ++z) v += red[(size_t)z * NC * 64 + o];
        const uint32_t at = o & 15, col = (cb * NC + o / 64) * 16 + 4 * ((o & 63) >> 4);
        if (at >= it.rows || col >= w.m) continue;
        if (splits == 1) store4(Y + (uint64_t)(it.row0 + at) * ldy, col, w.m, wide, v);
        else store4(part + ((uint64_t)split * B + it.row0 + at) * w.m, col, w.m, w.m % 4 == 0, v);
    }
}

// ---- many rows -----------------------------------------------------------------------------------
// X in operand order, group by group, each group from a tile of 16 rows of its own on, zeros behind entry n up to a whole group of four steps: quantised codes (and
// their scales in groups of four tiles, as W's); bf16 rows as [tile][step][row][piece of 8 k], pieces in an order that differs from
// row to row (turned); the three parts of fp32 rows as [tile][step][half][part][operand][lane][16 bytes].
// (A wavefront has a tile's step, a lane a block of its row.)  Bound by memory: 4096 rows of 8192 bfloat16 to codes in 20 us, 4.1 TB/s.
__host__ __device__ constexpr uint32_t step_bytes(int mode) { return mode == FP4 ? 1024u : 4096u * mode; }
// Steps of a chunk, which is what a block stages and requests at once, and chunks of a step.  Few rows are multiplied quickly: several steps
// at once keep more of W in flight (9973 x 1511, 137 bf16 rows 24.0 -> 20.8 us), unless three parts of them leave LDS room for one block
// a CU (25088 x 4096, 32 fp32 rows 31.9 -> 34.9).
__host__ __device__ constexpr int chunk_steps(int mode, int nr) { return mode == FP4 ? 4 : mode == THREE ? 1 : nr <= 2 ? 4 : nr <= 4 ? 2 : 1; }
__host__ __device__ constexpr int chunk_halves(int mode) { return mode == THREE ? 2 : 1; }
__host__ __device__ constexpr uint32_t chunk_bytes(int mode, int nr)                 // of 16 rows
{
    return mode == FP4 ? 4096u + 256u : step_bytes(mode) * chunk_steps(mode, nr) / chunk_halves(mode);
}
// where a piece of a row lies: any 16 lanes that LDS serves at a time (0 .. 3, 12 .. 15, 20 .. 27 and so on) read from 16 different ones
__device__ __forceinline__ uint32_t turned(uint32_t row, uint32_t piece) { return piece ^ ((row & 3) | ((0u - row / 4) & 3) << 2); }
__device__ __forceinline__ uint32_t place(uint32_t row, uint32_t piece) { return row * 256 + turned(row, piece) * 16; }

template <int MODE, typename T>
__global__ void __launch_bounds__(256)
mx_lay_out_kernel(const T* __restrict__ X, uint64_t ldx, uint32_t n, uint32_t groups, uint32_t B,
                  const int32_t* __restrict__ offsets, uint32_t count, uint8_t* __restrict__ out, uint8_t* __restrict__ out_scales)
{
    __shared__ uint8_t bytes[256];
    const uint32_t lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const uint32_t wave = uniform(threadIdx.x >> 6);
    const uint32_t tile = blockIdx.x, step = blockIdx.y * 4 + wave;
    const Item it = find_item(offsets, count, B, 16, tile);
    if (!it.rows) return;
    const T* row = X + (uint64_t)(it.row0 + min(c, it.rows - 1)) * ldx;
    const bool words = whole_words(X, ldx);
    Block32<T> x;
    if (step * 128 + 128 <= n) x.load_step(row + step * 128, g, words);
    else x.load_step(row + step * 128, g, words, n > step * 128 ? n - step * 128 : 0u, n);
    if constexpr (MODE == FP4) {
        uint32_t byte;
        const u32x4 q = quantise(x, byte);
        *reinterpret_cast<u32x4*>(out + (((uint64_t)tile * groups * 4 + step) * 64 + lane) * 16) = q;
        bytes[lane * 4 + wave] = (uint8_t)byte;
        __syncthreads();
        if (threadIdx.x < 64)
            reinterpret_cast<uint32_t*>(out_scales)[((uint64_t)tile * groups + blockIdx.y) * 64 + lane] = reinterpret_cast<const uint32_t*>(bytes)[lane];
    } else {
        uint8_t* to = out + ((uint64_t)tile * groups * 4 + step) * step_bytes(MODE);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 p[MODE];
            x.parts(j, p);
            if constexpr (MODE == ONE) *reinterpret_cast<u32x4*>(to + place(c, 4 * g + j)) = p[0];
            else
#pragma unroll
                for (int i = 0; i < 3; ++i) *reinterpret_cast<u32x4*>(to + ((j / 2 * 3 + i) * 2 + j % 2) * 1024 + lane * 16) = p[i];
        }
    }
}

// The product.  A block of 4 wavefronts owns 16 NR rows x 64 NC columns, wavefront w the 16 NC columns from 16 NC w on and all rows.
// A chunk of X (a step of 128 k; half of one as three parts; four of them as codes) goes to LDS past the registers, one chunk ahead; a
// column belongs to one wavefront, so W goes from memory into its registers, ahead too, and is expanded once per block.
// The order of a chunk is spelled out in beats of NC matrix instructions: left to itself the compiler reads an operand right before its
// use and waits.  A beat's operand of X is read two beats ahead, and W's operands of the next 32 k are expanded beside this one's products.
// DIRECT: bf16 rows whose pieces of 8 k are whole and aligned need no laying out, they are staged from where they are.
// Measured: 4096 x 4096, 2048 rows of bfloat16 60 us, 1.15 PFLOP/s, 8 groups of it with 4096 rows 1.0 (a library's bfloat16 product of the first size
// 1.01, of 8192 x 8192 x 8192 1.26; the instructions alone, from registers, 1.8); 8192 x 8192, 4096 rows in codes 137 us, 4.0 PFLOP/s (7.1 from
// registers; without W's loads 24 us less, without staging 20, without either 45; 137 is the least of a trace, its median is 144, 3.8 PFLOP/s).
__device__ __constant__ __attribute__((aligned(16))) uint32_t zeros16[4] = {0, 0, 0, 0};

// 16 bytes (4) a lane from memory to lds + 16 (4) * lane, past the registers.  In assembly, so that the compiler counts its own loads only: with
// these among them it waits for everything in flight wherever it needs one load or one read of LDS.  A wait for its own loads waits for these too
// then, never the other way round: loads_done() is what says that they are.
__device__ __forceinline__ uint32_t lds_offset(const uint8_t* p) { return uniform((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p); }
__device__ __forceinline__ void to_lds(const void* from, const uint8_t* lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_offset(lds)), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void to_lds(const void* base, uint32_t offset, const uint8_t* lds)      // (base: the wavefront's)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_offset(lds)), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void word_to_lds(const void* base, uint32_t offset, const uint8_t* lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_offset(lds)), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void block_sync_lds()                                  // loads from global memory stay in flight across it
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int MODE, bool DIRECT, typename T, int NR, int NC>
__global__ void __launch_bounds__(256, 2)
mx_tile_kernel(MxW w, const uint8_t* __restrict__ xt, const uint8_t* __restrict__ xs, uint64_t ldx, uint32_t max_tiles, uint32_t B,
               const int32_t* __restrict__ offsets, T* __restrict__ Y, uint64_t ldy, uint32_t rows_each, uint32_t stretches,
               uint32_t col_blocks, uint32_t splits, uint32_t per_split, float* __restrict__ part)
{
    constexpr uint32_t CH = chunk_bytes(MODE, NR), STAGE = NR * CH;
    constexpr int CS = chunk_steps(MODE, NR), HALVES = chunk_halves(MODE);
    extern __shared__ __align__(16) uint8_t lds[];               // two stages
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    // consecutive items on one XCD; the stretches of a column block follow one another and share its part of W in that L2
    const uint32_t id = (blockIdx.x & 7u) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (id >= stretches * col_blocks * splits) return;
    const uint32_t split = id / (stretches * col_blocks), rest = id - split * stretches * col_blocks;
    const uint32_t cb = rest / stretches, stretch = rest - cb * stretches;
    const Item it = find_item(offsets, w.count, B, rows_each, stretch);
    const uint32_t tiles = (it.rows + 15) / 16;
    if (!it.rows || (!DIRECT && it.tile + tiles > max_tiles)) return;
    const uint32_t chunks = (w.steps + CS - 1) / CS;
    const uint32_t c0 = split * per_split, c1 = min(chunks, c0 + per_split);

    const uint8_t* code[NC];
    const uint8_t* scale[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
        const uint32_t ct = min((cb * 4 + wave) * NC + q, w.ctiles - 1);
        code[q] = w.codes + it.expert * w.code_stride + (uint64_t)ct * w.steps * 1024;       // (the wavefront's: lanes add 16 and 4 bytes each)
        scale[q] = w.scales + it.expert * w.scale_stride + (uint64_t)ct * w.groups * 256;
    }
    const uint32_t lane16 = 16 * lane, lane4 = 4 * lane;
    // pieces of 1024 bytes (and of 256 for the scales) are dealt to the wavefronts; rows past the last tile keep what LDS holds
    const uint32_t row4 = 4 * wave + lane / 16, piece = turned(row4, lane & 15);
    const uint8_t *first = nullptr, *end = nullptr;              // DIRECT: a lane's row of the first tile and, the last row again, of the last
    if constexpr (DIRECT) {
        first = xt + ((uint64_t)(it.row0 + min(row4, it.rows - 1)) * ldx + 8 * piece) * 2;
        end = xt + ((uint64_t)(it.row0 + min(16 * (tiles - 1) + row4, it.rows - 1)) * ldx + 8 * piece) * 2;
    }
    auto stage = [&](auto count, uint32_t ch, uint32_t half, uint8_t* to) ALWAYS_INLINE {
        constexpr uint32_t N = decltype(count)::value;
        if constexpr (DIRECT) {
#pragma unroll
            for (int c = 0; c < CS; ++c) {
                const uint32_t step = ch * CS + c;
                const bool inside = step * 128 + 8 * piece < w.n;
#pragma unroll
                for (uint32_t t = 0; t < N; ++t) {
                    const uint8_t* from = (t + 1 < tiles ? first + t * (32 * ldx) : end) + (uint64_t)step * 256;
                    to_lds(inside ? from : reinterpret_cast<const uint8_t*>(zeros16), to + t * CH + c * 4096 + wave * 1024);
                }
            }
        } else {
            constexpr uint32_t PIECES = CH / 1024;               // (the scales' 256 bytes apart)
#pragma unroll
            for (uint32_t i = 0; i < (N * PIECES + 3) / 4; ++i) {
                const uint32_t z = wave + 4 * i, t = z / PIECES, p = z - t * PIECES;
                if (N * PIECES % 4 && z >= N * PIECES) break;
                const uint64_t at = ((uint64_t)(it.tile + min(t, tiles - 1)) * w.groups * 4 + ch * CS) * step_bytes(MODE) + half * CH;
                to_lds(xt + at + p * 1024, lane16, to + t * (PIECES * 1024) + p * 1024);
            }
            if constexpr (MODE == FP4)
                for (uint32_t t = wave; t < N; t += 4)
                    word_to_lds(xs + ((uint64_t)(it.tile + min(t, tiles - 1)) * w.groups + ch) * 256, lane4, to + NR * 4096 + t * 256);
        }
    };
    f32x4 acc[NR][NC];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int q = 0; q < NC; ++q) acc[r][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t at_lane[4];                                         // of a lane's operand in LDS
#pragma unroll
    for (int j = 0; j < 4; ++j) at_lane[j] = MODE == ONE ? place(lane & 15, 4 * (lane >> 4) + j) : lane16;

    // step s of chunk ch (behind the last one: any tile, X is 0 there and W's scales too)
    auto load_codes = [&](uint32_t ch, int s, u32x4 (&to)[NC]) ALWAYS_INLINE {
        const uint32_t step = min(ch * CS + s, w.steps - 1);
#pragma unroll
        for (int q = 0; q < NC; ++q) to[q] = *reinterpret_cast<const u32x4*>(code[q] + (uint64_t)step * 1024 + lane16);
    };
    // the scales of chunk ch, its first step's in the lowest byte
    auto load_scales = [&](uint32_t ch, uint32_t* to) ALWAYS_INLINE {
#pragma unroll
        for (int q = 0; q < NC; ++q) {
            if constexpr (CS == 1) to[q] = *(scale[q] + (uint64_t)(ch / 4) * 256 + ch % 4 + lane4);
            else to[q] = *reinterpret_cast<const uint32_t*>(scale[q] + (uint64_t)(ch * CS / 4) * 256 + lane4) >> (CS == 2 ? 16 * (ch & 1) : 0);
        }
    };

    // the chunks with the first N of the NR tiles of rows
    auto walk = [&](auto count) ALWAYS_INLINE {
        constexpr int N = decltype(count)::value;
        u32x4 cur[CS][NC], next[MODE == FP4 ? 1 : CS][NC];
        uint32_t cur_s[NC], next_s[NC];
        bf16x8 v[2][NC];                                         // W's operand of these 32 k and the next
        const uint32_t last = (c1 - c0) * HALVES - 1;            // chunk u: step c0 + u / HALVES, half u % HALVES
        stage(count, c0, 0, lds);
        load_scales(c0, cur_s);
#pragma unroll
        for (int s = 0; s < CS; ++s) load_codes(c0, s, cur[s]);
        if constexpr (MODE != FP4) {
#pragma unroll
            for (int q = 0; q < NC; ++q) v[0][q] = weights(cur[0][q][0], scale_of(cur_s[q] & 255));
        }
        loads_done();
        uint32_t u = 0;
        for (uint32_t ch = c0; ch < c1; ++ch) {
            const uint32_t ahead = min(ch + 1, c1 - 1);
#pragma unroll
            for (int half = 0; half < HALVES; ++half) {
                const uint8_t* x = lds + (u & 1) * STAGE;
                block_sync_lds();                                // all have their part of this chunk, and have read the one before
                if (half == 0) {
                    load_scales(ahead, next_s);
                    if constexpr (MODE != FP4)
#pragma unroll
                        for (int s = 0; s < CS; ++s) load_codes(ahead, s, next[s]);
                }
                if (u < last) stage(count, c0 + (u + 1) / HALVES, (u + 1) % HALVES, lds + (~u & 1) * STAGE);
                ++u;
                __builtin_amdgcn_sched_barrier(0);
                // beat b multiplies one operand of X; what it is depends on b alone
                constexpr int PARTS = MODE == THREE ? 3 : 1, JS = MODE == FP4 ? 4 : 4 * CS / HALVES, PER = N * PARTS, BEATS = JS * PER;
                auto operand_at = [&](int b) ALWAYS_INLINE -> u32x4 {
                    const int j = b / PER, i = PARTS - 1 - b % PER / N, r = b % N;
                    if constexpr (MODE == FP4) return *reinterpret_cast<const u32x4*>(x + r * 4096 + j * 1024 + at_lane[0]);
                    else if constexpr (MODE == ONE) return *reinterpret_cast<const u32x4*>(x + r * CH + j / 4 * 4096 + at_lane[j % 4]);
                    else return *reinterpret_cast<const u32x4*>(x + r * CH + (j / 2 * 6 + i * 2 + j % 2) * 1024 + at_lane[0]);
                };
                u32x4 xq[3];
                uint32_t sx[N];
                xq[0] = operand_at(0);
                if (BEATS > 1) xq[1] = operand_at(1);
                if constexpr (MODE == FP4) {
#pragma unroll
                    for (int r = 0; r < N; ++r) sx[r] = *reinterpret_cast<const uint32_t*>(x + NR * 4096 + r * 256 + lane * 4);
                }
#pragma unroll
                for (int b = 0; b < BEATS; ++b) {
                    const int j = b / PER, t = b % PER, r = b % N;
                    if (b + 2 < BEATS) xq[(b + 2) % 3] = operand_at(b + 2);
                    if constexpr (MODE == FP4) {
#pragma unroll
                        for (int q = 0; q < NC; ++q) {
                            if (j == 0) acc[r][q] = multiply_fp4<0>(cur[0][q], cur_s[q], xq[b % 3], sx[r], acc[r][q]);
                            if (j == 1) acc[r][q] = multiply_fp4<1>(cur[1][q], cur_s[q], xq[b % 3], sx[r], acc[r][q]);
                            if (j == 2) acc[r][q] = multiply_fp4<2>(cur[2][q], cur_s[q], xq[b % 3], sx[r], acc[r][q]);
                            if (j == 3) acc[r][q] = multiply_fp4<3>(cur[3][q], cur_s[q], xq[b % 3], sx[r], acc[r][q]);
                        }
                    } else {
                        const int jj = half * JS + j;            // 32 k of the chunk
#pragma unroll
                        for (int q = 0; q < NC; ++q) acc[r][q] = multiply_bf16(v[jj & 1][q], xq[b % 3], acc[r][q]);
#pragma unroll
                        for (int q = t * NC / PER; q < (t + 1) * NC / PER; ++q)
                            v[(jj & 1) ^ 1][q] = jj + 1 < 4 * CS ? weights(cur[(jj + 1) / 4 % CS][q][(jj + 1) % 4], scale_of(cur_s[q] >> 8 * ((jj + 1) / 4) & 255))
                                                               : weights(next[0][q][0], scale_of(next_s[q] & 255));
                    }
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
                    for (int q = 0; q < NC; ++q) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    // what was staged at the start of the chunk has had three quarters of it to arrive
                    if (b == (BEATS * 3 + 3) / 4 - 1) loads_done();
                    if (MODE == FP4 && t == PER - 1) {
                        if (j != 1) load_codes(ahead, j, cur[j]);
                        if (j == 2) load_codes(ahead, 1, cur[1]);
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < NC; ++q) {
                cur_s[q] = next_s[q];
                if constexpr (MODE != FP4)
#pragma unroll
                    for (int s = 0; s < CS; ++s) cur[s][q] = next[s][q];
            }
        }
    };
    if (c0 < c1) {
        if (NR >= 4 && tiles <= NR / 2) walk(std::integral_constant<int, NR >= 4 ? NR / 2 : NR>{});
        else if (NR >= 4 && tiles <= NR * 3 / 4) walk(std::integral_constant<int, NR >= 4 ? NR * 3 / 4 : NR>{});
        else walk(std::integral_constant<int, NR>{});
    }
    const uint32_t l16 = lane & 15, first_col = (cb * 4 + wave) * NC * 16, col0 = first_col + 4 * (lane >> 4);
    const bool wide = (reinterpret_cast<uintptr_t>(Y) | ldy * sizeof(T)) % (4 * sizeof(T)) == 0;
    if constexpr (sizeof(T) == 2 && NC > 1) {
        // two tiles of columns at a time: the lanes of a row exchange halves and have eight neighbouring columns each, so that an instruction
        // writes 64 bytes of a row side by side, not 32 (4096 x 8192 results of k = 8192 in 4 bits 160 -> 156 us; 128 bytes: no better)
        if (splits == 1 && (reinterpret_cast<uintptr_t>(Y) | ldy * 2) % 16 == 0) {
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int q = 0; q < NC; q += 2) {
                    uint32_t h[2][2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const f32x4 v = acc[r][q + i];
                        h[i][0] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v.x, (__bf16)v.y});
                        h[i][1] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v.z, (__bf16)v.w});
                    }
                    swap16(h[0][0], h[1][0]); swap16(h[0][1], h[1][1]);
                    const uint32_t at = 16 * r + l16, col = first_col + 16 * (q + (lane >> 4 & 1)) + 8 * (lane >> 5);
                    if (at < it.rows && col < w.m) store8(Y + (uint64_t)(it.row0 + at) * ldy + col, w.m - col, u32x4{h[0][0], h[0][1], h[1][0], h[1][1]});
                }
            return;
        }
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const uint32_t at = 16 * r + l16;
        if (at >= it.rows) continue;
        const uint64_t row = it.row0 + at;
#pragma unroll
        for (int q = 0; q < NC; ++q) {
            const uint32_t col = col0 + 16 * q;
            if (col >= w.m) continue;
            if (splits == 1) store4(Y + row * ldy, col, w.m, wide, acc[r][q]);
            else store4(part + ((uint64_t)split * B + row) * w.m, col, w.m, w.m % 4 == 0, acc[r][q]);
        }
    }
}

// Y = part[0] + part[1] + ... in that order, for the rows that some group holds.  A thread has four neighbouring sums where columns come in fours
// (V = f32x4), so that all splits' are in flight.  16 splits of 32 x 4096 sums: 3.9 us, of which 2 are the launch.
template <typename T, typename V>
__global__ void __launch_bounds__(256)
mx_sum_kernel(const float* __restrict__ part, uint32_t splits, uint32_t B, uint32_t m, const int32_t* __restrict__ offsets, uint32_t count,
              T* __restrict__ Y, uint64_t ldy)
{
    constexpr uint32_t E = sizeof(V) / 4;
    uint32_t lo = 0, hi = B;
    if (offsets) {
        lo = (uint32_t)min(max(offsets[0], 0), (int32_t)B);
        hi = (uint32_t)min(max(offsets[count], 0), (int32_t)B);
    }
    const uint32_t col = (blockIdx.x * 256 + threadIdx.x) * E;
    if (col >= m) return;
    const bool wide = (reinterpret_cast<uintptr_t>(Y) | ldy * sizeof(T)) % (4 * sizeof(T)) == 0;
    const uint64_t next = (uint64_t)B * m;
    for (uint32_t row = lo + blockIdx.y; row < hi; row += gridDim.y) {
        const float* p = part + (uint64_t)row * m + col;
        V v = *reinterpret_cast<const V*>(p);
        uint32_t s = 1;
        for (; s + 3 < splits; s += 4) {
            const V a = *reinterpret_cast<const V*>(p + s * next), b = *reinterpret_cast<const V*>(p + (s + 1) * next);
            const V c = *reinterpret_cast<const V*>(p + (s + 2) * next), d = *reinterpret_cast<const V*>(p + (s + 3) * next);
            v += a; v += b; v += c; v += d;
        }
        for (; s < splits; ++s) v += *reinterpret_cast<const V*>(p + s * next);
        T* y = Y + (uint64_t)row * ldy;
        if constexpr (E == 4) store4(y, col, m, wide, v);
        else y[col] = (T)v;
    }
}

// ---- host --------------------------------------------------------------------------------------

int hip_fail(hipError_t e) { set_last_hip_error((int)e); return HAC_EHIP; }
int launched() { const hipError_t e = hipGetLastError(); return e == hipSuccess ? HAC_OK : hip_fail(e); }

const char* type_name(const float*) { return "float"; }
const char* type_name(const __bf16*) { return "__bf16"; }

MxW matrices(const hac_desc_t& d, const void* blob)
{
    const MxShape s = mx_shape(d.n, d.m);
    const uint8_t* b = static_cast<const uint8_t*>(blob);
    return MxW{ b + d.off_stream, b + d.off_codebook, s.code_bytes, s.scale_bytes, (uint32_t)d.n, (uint32_t)d.m, (uint32_t)s.steps,
                (uint32_t)s.groups, (uint32_t)s.ctiles, d.k_sym };
}

constexpr int64_t kMostRows = 1 << 27;
constexpr uint64_t kMostStretches = 65535;       // of 16 rows, in a launch of the kernel for few rows

// How a product is split.  rows: the kernel for few rows, nc tiles of columns a block of `waves` wavefronts; else tiles of 16 nr rows x 64 nc
// columns.  splits: parts that the k of a column are cut into.
struct Choice { bool rows; uint32_t nr, nc, waves, splits; };

constexpr uint32_t least_nc(int mode, uint32_t nr) { return mode == THREE || nr == 8 ? 2 : 1; }           // (one column tile was never the quickest there)
constexpr uint32_t most_nc(int mode, uint32_t nr) { return mode == ONE && nr == 8 ? 2 : 4; }       // (more sums and operands than registers)

struct Plan {
    Choice c;
    bool direct;                                 // tiles of X as it lies
    int mode;
    uint32_t rows_each, per_split;               // rows a stretch; chunks a split (tiles)
    uint64_t stretches, col_blocks, tiles;       // stretches, tiles: as many as B rows in `count` groups can fill
    size_t xt_bytes, xs_bytes, part_bytes, bytes;
};

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
uint64_t fill(uint64_t B, uint64_t count, uint64_t R) { return std::min<uint64_t>(B, (B + (R - 1) * count) / R); }

// The split with the shortest estimate of a call's time.  Its form and constants (us) were fitted to the measured times of all splits of 800 products
// drawn over n 64 .. 25088, m 10 .. 8192, 1 .. 12544 rows, 1 .. 64 groups: estimates are off by 10 to 14 % in the mean, and the splits they choose are
// 3.0 % slower in the mean than the best measured ones, at most 1.47 times, and 3.7 % over 350 products that they were not fitted to (one split per
// kernel, chosen by rows alone: 45 %).  These figures are of the time of the fit: since then results in bfloat16 leave 64 bytes of a row side by side, which
// takes 2 to 6 % off products on tiles.  The constants predict, they do not explain: on tiles quantised X is multiplied by the same loop whatever
// its type was, yet the fit put that loop's time into t_tile for fp32 and into t_chunk_mm, in part, for bfloat16.  Too low where blocks are fewer than
// CUs: 4096 x 4096, 16 quantised fp32 rows take 11.6 us in 64 blocks, estimated at 9.1; in four splits of four wavefronts they take 9.1.  Groups are taken
// to be as full as a router leaves them: one in five or so without rows (used).
//   few rows: a launch; trips to memory, two steps each, and what a trip grows by with each tile of columns; wavefronts beyond eight on a CU;
//     steps of X turned into operands and of W multiplied per SIMD, what the former cost more where X is larger than the L2s (big) or its rows of
//     bfloat16 have an odd length, and those that a SIMD has more where blocks are fewer than CUs; sums stored; the pass that adds the
//     splits and its megabytes
//   tiles: a launch; X laid out and its megabytes; chunks of a block and their matrix instructions; the blocks of a CU; a hundred steps of a
//     block times the blocks of a CU, for 2, 4, 8 tiles of rows and 1, 2, 4 of columns a wavefront (0: there is no such kernel); the pass that adds the
//     splits and its megabytes; Y's megabytes and W's
struct Costs {
    double call, trip, trip_nc, waves, steps, steps_nc, big, odd, alone, sums, split, split_mb;
    double t_call, t_lay, t_lay_mb, t_chunk, t_chunk_mm, t_cu, t_tile[9], t_split, t_split_mb, t_mb, t_w_mb;
};
const Costs kCosts[4] = {
    { 3.85, 0.456, 0.074, 0.414, 0.584, 0.081, 0.360, 0.000, 0.311, 0.435, 1.92, 4.51,                      // codes, from fp32
      0.00, 7.60, 0.199, 0.014, 0.029, 0.000, { 6.58, 10.7, 20.4, 11.4, 16.7, 28.8, 0.0, 30.5, 58.9 }, 1.77, 2.23, 0.583, 0.122 },
    { 3.64, 0.609, 0.082, 0.354, 0.203, 0.070, 0.269, 0.222, 0.219, 0.381, 2.19, 2.93,                      // codes, from bf16
      0.00, 7.13, 0.246, 0.012, 0.790, 0.000, { 5.48, 8.69, 15.4, 8.84, 11.9, 17.6, 0.0, 19.2, 29.6 }, 2.63, 1.65, 0.780, 0.082 },
    { 3.39, 0.845, 0.270, 0.793, 0.597, 0.121, 0.474, 0.000, 0.335, 0.387, 2.63, 1.73,                      // fp32
      0.00, 8.16, 0.557, 0.249, 0.329, 0.000, { 0.0, 61.6, 84.9, 0.0, 113.0, 176.0 }, 2.11, 1.60, 0.658, 0.000 },
    { 3.66, 0.493, 0.159, 0.392, 0.031, 0.087, 0.280, 0.424, 0.145, 0.285, 2.18, 2.77,                      // bf16
      3.72, 3.60, 0.648, 0.196, 0.465, 0.356, { 15.8, 21.6, 36.9, 29.4, 37.8, 55.3, 0.0, 67.0 }, 2.28, 1.87, 0.957, 0.001 },
};

Choice choose(const MxShape& s, uint64_t B, uint64_t count, uint64_t n, uint64_t m, uint32_t type, int mode, bool direct)
{
    const Costs& k = kCosts[(mode == FP4 ? 0 : 2) + (type == HAC_TYPE_BF16 ? 1 : 0)];
    const double b = (double)B, used = count > 1 ? 0.8 * (double)std::min(count, B) : 0.0, out_mb = b * (double)m / 1e6;
    // stretches of R rows that hold rows: in groups, the last of each is half full
    auto live = [&](uint64_t R) {
        const uint64_t least = ceil_div(B, R);
        return count > 1 ? std::min(b, std::max((double)least, used + b / (double)R)) : (double)least;
    };
    Choice best = { true, 1, 1, 2, 1 };
    double best_us = 1e300;
    auto consider = [&](double us, const Choice& c) { if (us < best_us) { best_us = us; best = c; } };
    const double stretches16 = live(16), x_mb = b * (double)n * (type == HAC_TYPE_F32 ? 4 : 2) / 1e6;
    const double step = k.steps + k.big * std::min(1.0, std::max(0.0, x_mb / 8 - 0.5)) + (type == HAC_TYPE_BF16 && n % 2 ? k.odd : 0.0);
    const bool rows_fit = fill(B, count, 16) <= kMostStretches;
    for (uint32_t nc = 1; rows_fit && nc <= 4; nc *= 2) {
        const double blocks = stretches16 * (double)ceil_div(s.ctiles, nc), steps = blocks * (double)s.steps / 1024;
        for (uint32_t splits = 1; splits <= 16; splits *= 2) {
            if (splits > 1 && s.steps < 8 * splits) break;
            for (uint32_t waves = 2; waves <= 8; waves *= 2) {
                const uint64_t each = ceil_div(s.steps, waves * splits);
                const double trips = (double)ceil_div(each, 2), items = blocks * splits;
                double us = k.call + trips * (k.trip + k.trip_nc * nc) + k.waves * std::max(0.0, items * waves / 2048 - 1) +
                            steps * (step + k.steps_nc * nc) + k.alone * std::max(0.0, waves * (double)each / 4 - steps) +
                            k.sums * items * nc / 1024;
                if (splits > 1) us += k.split + k.split_mb * splits * out_mb;
                consider(us, Choice{ true, 1, nc, waves, splits });
                if (waves >= s.steps) break;
            }
        }
    }
    const double laid = direct ? 0.0 : k.t_lay + k.t_lay_mb * b * (double)s.steps * 128 * (type == HAC_TYPE_F32 ? 4 : 2) / 1e6;
    const double w_mb = (count > 1 ? used : 1.0) * (double)n * (double)m / 2e6;
    const double fixed = k.t_call + laid + k.t_mb * out_mb * (type == HAC_TYPE_F32 ? 4 : 2) + k.t_w_mb * w_mb;
    if (fixed >= best_us || (rows_fit && B <= 8 * std::min(count, B))) return best;      // (up to 8 rows a group tiles were never measured to be quicker)
    const uint32_t most_nr = mode == THREE ? 4 : 8;
    for (uint32_t nr = 2; nr <= most_nr; nr *= 2) {
        if (nr > 2 && B <= 8 * nr) break;
        uint64_t rows = 16 * nr;
        if (count == 1) { const uint64_t tiles = ceil_div(B, 16); rows = 16 * ceil_div(tiles, ceil_div(tiles, nr)); }   // (dealt evenly)
        const uint64_t chunks = ceil_div(s.steps, chunk_steps(mode, nr));
        const double stretches = live(rows);
        for (uint32_t nc = least_nc(mode, nr); nc <= most_nc(mode, nr); nc *= 2) {
            const double blocks = stretches * (double)ceil_div(s.ctiles, 4 * nc);
            const double step_us = k.t_tile[(nr / 4) * 3 + nc / 2] / 100 * chunk_steps(mode, nr) * (0.2 + 0.8 * (double)rows / (16 * nr));
            const double mm = (mode == FP4 ? 1.0 : mode == THREE ? 4.0 * 3 : 4.0) * chunk_steps(mode, nr) * (double)(rows / 16) * nc / 100;
            for (uint32_t splits = 1; splits <= 16; splits *= 2) {
                if (splits > chunks) break;
                const uint64_t per = ceil_div(chunks, splits), parts = ceil_div(chunks, per);
                const double cu = std::max(1.0, blocks * (double)parts / 256);
                double us = fixed + (double)per * (k.t_chunk + k.t_chunk_mm * mm + cu * step_us) + k.t_cu * cu;
                if (parts > 1) us += k.t_split + k.t_split_mb * (double)parts * out_mb;
                consider(us, Choice{ false, nr, nc, 4, splits });
            }
        }
    }
    return best;
}

// whole: rows of X consist of whole, aligned pieces of 16 bytes.  bytes is what a call needs wherever X lies, for its size is asked without X: where
// tiles take X as it lies, xt_bytes of it stay unused.
Plan plan_mx(const hac_desc_t& d, uint32_t type, uint64_t B, uint32_t flags, bool grouped, bool whole)
{
    const MxShape s = mx_shape(d.n, d.m);
    const uint64_t count = grouped ? d.k_sym : 1;
    Plan p = {};
    p.mode = flags & HAC_MX_QUANTIZE_X ? FP4 : type == HAC_TYPE_F32 ? THREE : ONE;
    const bool pieces = p.mode == ONE && d.n % 8 == 0;
    p.c = choose(s, B, count, d.n, d.m, type, p.mode, pieces);
    auto up = [](uint64_t v) { return (size_t)((v + 255) / 256 * 256); };
    if (p.c.rows) {
        p.rows_each = 16;
        p.col_blocks = ceil_div(s.ctiles, p.c.nc);
    } else {
        p.direct = pieces && whole;
        p.rows_each = 16 * p.c.nr;
        if (!grouped) { const uint64_t tiles = ceil_div(B, 16); p.rows_each = 16 * (uint32_t)ceil_div(tiles, ceil_div(tiles, p.c.nr)); }
        p.col_blocks = ceil_div(s.ctiles, 4 * p.c.nc);
        p.tiles = fill(B, count, 16);
        const uint64_t chunks = ceil_div(s.steps, chunk_steps(p.mode, p.c.nr));
        p.per_split = (uint32_t)ceil_div(chunks, p.c.splits);
        p.c.splits = (uint32_t)ceil_div(chunks, p.per_split);
        p.xt_bytes = up(p.tiles * s.groups * 4 * step_bytes(p.mode));
        p.xs_bytes = p.mode == FP4 ? up(p.tiles * s.groups * 256) : 0;
    }
    p.stretches = fill(B, count, p.rows_each);
    p.part_bytes = p.c.splits > 1 ? up((uint64_t)p.c.splits * B * d.m * sizeof(float)) : 0;
    p.bytes = p.xt_bytes + p.xs_bytes + p.part_bytes;
    return p;
}

template <int MODE, typename T, int NC>
int launch_rows(const Plan& p, const MxW& w, const T* X, uint64_t ldx, uint32_t B, const int32_t* offsets, T* Y, uint64_t ldy, float* part,
                hipStream_t stream)
{
    constexpr int U = 2;
    hipLaunchKernelGGL((mx_rows_kernel<MODE, T, NC, U>), dim3((uint32_t)p.col_blocks, (uint32_t)p.stretches, p.c.splits), dim3(64 * p.c.waves),
                       (size_t)p.c.waves * NC * 1024, stream, w, X, ldx, B, offsets, Y, ldy, w.steps / (p.c.splits * p.c.waves),
                       w.steps % (p.c.splits * p.c.waves), part);
    note_kernel("mx_rows_kernel<%d, %s, %d, %d>", MODE, type_name(X), NC, U);
    return launched();
}

struct Operands {                                // of a product on tiles: X laid out, or X itself (ldx), and where partial sums go
    const uint8_t *xt, *xs;
    uint64_t ldx;
    float* part;
};

template <int MODE, bool DIRECT, typename T, int NR, int NC>
int launch_tile(const Plan& p, const MxW& w, const Operands& x, uint32_t B, const int32_t* offsets, T* Y, uint64_t ldy, hipStream_t stream)
{
    auto k = mx_tile_kernel<MODE, DIRECT, T, NR, NC>;
    constexpr size_t lds = 2 * NR * chunk_bytes(MODE, NR);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return hip_fail(e);
    }
    const uint64_t items = p.stretches * p.col_blocks * p.c.splits;
    hipLaunchKernelGGL(k, dim3((uint32_t)((items + 7) / 8 * 8)), dim3(256), lds, stream, w, x.xt, x.xs, x.ldx, (uint32_t)p.tiles, B, offsets, Y, ldy,
                       p.rows_each, (uint32_t)p.stretches, (uint32_t)p.col_blocks, p.c.splits, p.per_split, x.part);
    note_kernel("mx_tile_kernel<%d, %s, %s, %d, %d>", MODE, DIRECT ? "true" : "false", type_name(Y), NR, NC);
    return launched();
}

template <int MODE, bool DIRECT, typename T>
int pick_tile(const Plan& p, const MxW& w, const Operands& x, uint32_t B, const int32_t* offsets, T* Y, uint64_t ldy, hipStream_t stream)
{
    auto columns = [&](auto rows) {
        constexpr int NR = decltype(rows)::value;
        if constexpr (least_nc(MODE, NR) == 1)
            if (p.c.nc == 1) return launch_tile<MODE, DIRECT, T, NR, 1>(p, w, x, B, offsets, Y, ldy, stream);
        if constexpr (most_nc(MODE, NR) == 4)
            if (p.c.nc == 4) return launch_tile<MODE, DIRECT, T, NR, 4>(p, w, x, B, offsets, Y, ldy, stream);
        return launch_tile<MODE, DIRECT, T, NR, 2>(p, w, x, B, offsets, Y, ldy, stream);
    };
    if (p.c.nr == 2) return columns(std::integral_constant<int, 2>{});
    if (p.c.nr == 4) return columns(std::integral_constant<int, 4>{});
    return columns(std::integral_constant<int, MODE == THREE ? 4 : 8>{});
}

template <int MODE, typename T>
int run_mode(const Plan& p, const MxW& w, const T* X, uint64_t ldx, uint32_t B, const int32_t* offsets, T* Y, uint64_t ldy, uint8_t* ws,
             hipStream_t stream)
{
    const Operands x = { p.direct ? reinterpret_cast<const uint8_t*>(X) : ws, ws + p.xt_bytes, ldx,
                         reinterpret_cast<float*>(ws + p.xt_bytes + p.xs_bytes) };
    int rc = HAC_OK;
    if (p.c.rows) {
        rc = p.c.nc == 1 ? launch_rows<MODE, T, 1>(p, w, X, ldx, B, offsets, Y, ldy, x.part, stream)
           : p.c.nc == 2 ? launch_rows<MODE, T, 2>(p, w, X, ldx, B, offsets, Y, ldy, x.part, stream)
                       : launch_rows<MODE, T, 4>(p, w, X, ldx, B, offsets, Y, ldy, x.part, stream);
    } else if (p.direct) {
        if constexpr (MODE == ONE) rc = pick_tile<MODE, true, T>(p, w, x, B, offsets, Y, ldy, stream);
    } else {
        hipLaunchKernelGGL((mx_lay_out_kernel<MODE, T>), dim3((uint32_t)p.tiles, w.groups), dim3(256), 0, stream, X, ldx, w.n, w.groups, B,
                           offsets, w.count, ws, ws + p.xt_bytes);
        note_kernel("mx_lay_out_kernel<%d, %s>", MODE, type_name(X));
        rc = launched();
        if (!rc) rc = pick_tile<MODE, false, T>(p, w, x, B, offsets, Y, ldy, stream);
    }
    if (rc || p.c.splits == 1) return rc;
    const bool fours = w.m % 4 == 0;
    const dim3 grid((uint32_t)ceil_div(w.m, fours ? 1024 : 256), std::min(B, 16384u));
    if (fours) hipLaunchKernelGGL((mx_sum_kernel<T, f32x4>), grid, dim3(256), 0, stream, x.part, p.c.splits, B, w.m, offsets, w.count, Y, ldy);
    else hipLaunchKernelGGL((mx_sum_kernel<T, float>), grid, dim3(256), 0, stream, x.part, p.c.splits, B, w.m, offsets, w.count, Y, ldy);
    note_kernel("mx_sum_kernel<%s, %s>", type_name(Y), fours ? "float __vector(4)" : "float");
    return launched();
}

template <typename T>
int run_typed(const Plan& p, const MxW& w, const void* X, uint64_t ldx, uint32_t B, const int32_t* offsets, void* Y, uint64_t ldy, uint8_t* ws,
              hipStream_t stream)
{
    const T* x = static_cast<const T*>(X);
    T* y = static_cast<T*>(Y);
    if (p.mode == FP4) return run_mode<FP4, T>(p, w, x, ldx, B, offsets, y, ldy, ws, stream);
    return run_mode<sizeof(T) == 4 ? THREE : ONE, T>(p, w, x, ldx, B, offsets, y, ldy, ws, stream);
}

// a launch's grid, in threads per dimension, has 32 bits
bool grids_fit(const Plan& p, const MxShape& s, const hac_desc_t& d)
{
    if (p.c.splits > 1 && ceil_div(d.m, 256) > 0xffffffull) return false;                 // (of the pass that adds them)
    if (p.c.rows) return p.col_blocks <= 0xffffffffull / (64 * p.c.waves) && p.stretches <= kMostStretches;
    return p.tiles <= 0xffffffull && s.groups <= 65535 && p.stretches * p.col_blocks <= 0xfffff0ull / p.c.splits;
}

bool aligned(const void* p, uint32_t type) { return reinterpret_cast<uintptr_t>(p) % (type == HAC_TYPE_F32 ? 4 : 2) == 0; }

int product(const hac_desc_t* desc, const void* d_blob, uint32_t type, const void* d_X, int64_t B, int64_t ldx, const int32_t* d_offsets,
            void* d_Y, int64_t ldy, uint32_t flags, void* d_ws, size_t ws_bytes, hac_stream_t stream, bool grouped)
{
    if (!desc || !d_blob || !mx_header_ok(*desc) || reinterpret_cast<uintptr_t>(d_blob) % 256) return HAC_EINVAL;
    if (type > HAC_TYPE_BF16 || (flags & ~HAC_MX_QUANTIZE_X) || B < 0) return HAC_EINVAL;
    if (grouped ? !d_offsets || reinterpret_cast<uintptr_t>(d_offsets) % 4 : desc->k_sym != 1) return HAC_EINVAL;
    if (B == 0) return HAC_OK;
    if (!d_X || !d_Y || ldx < (int64_t)desc->n || ldy < (int64_t)desc->m || !aligned(d_X, type) || !aligned(d_Y, type)) return HAC_EINVAL;
    if (B > kMostRows) return HAC_ERANGE;
    const bool whole = desc->n % 8 == 0 && ldx % 8 == 0 && reinterpret_cast<uintptr_t>(d_X) % 16 == 0;
    const Plan p = plan_mx(*desc, type, (uint64_t)B, flags, grouped, whole);
    if (!grids_fit(p, mx_shape(desc->n, desc->m), *desc)) return HAC_ERANGE;
    if (p.bytes && (!d_ws || ws_bytes < p.bytes)) return HAC_EWORKSPACE;
    if (p.bytes && reinterpret_cast<uintptr_t>(d_ws) % 256) return HAC_EINVAL;
    set_last_hip_error(0);
    const MxW w = matrices(*desc, d_blob);
    uint8_t* ws = static_cast<uint8_t*>(d_ws);
    hipStream_t hs = static_cast<hipStream_t>(stream);
    if (type == HAC_TYPE_F32) return run_typed<float>(p, w, d_X, (uint64_t)ldx, (uint32_t)B, d_offsets, d_Y, (uint64_t)ldy, ws, hs);
    return run_typed<__bf16>(p, w, d_X, (uint64_t)ldx, (uint32_t)B, d_offsets, d_Y, (uint64_t)ldy, ws, hs);
}

// the grid of the encode and decode kernels; false where it has too many blocks
bool code_grid(const hac_desc_t& d, dim3& grid)
{
    const MxShape s = mx_shape(d.n, d.m);
    const uint64_t x = (d.m + kCodeCols - 1) / kCodeCols;
    if (x > 0x3fffffull || s.groups > 65535) return false;
    grid = dim3((uint32_t)x, (uint32_t)s.groups, d.k_sym);
    return true;
}

// calls launch(an element of W, whether W is streamed)
template <typename F> void by_size(const hac_desc_t& d, uint32_t type, F launch)
{
    const bool large = (uint64_t)d.k_sym * d.n * d.m * (type == HAC_TYPE_F32 ? 4 : 2) > kCacheBytes;
    if (type == HAC_TYPE_F32) { if (large) launch(0.0f, std::true_type{}); else launch(0.0f, std::false_type{}); }
    else { if (large) launch((__bf16)0.0f, std::true_type{}); else launch((__bf16)0.0f, std::false_type{}); }
}

bool layout_ok(const hac_desc_t& d, int64_t ldw, int64_t stride)
{
    return ldw >= (int64_t)d.m && (d.k_sym == 1 || (stride >= 0 && stride / ldw >= (int64_t)d.n));
}

} // namespace

size_t hac_internal::mx_layer_bytes(const hac_desc_t* desc, int64_t B) { return mx_workspace_bytes(desc, HAC_TYPE_F32, B, 0, 0); }

int hac_internal::mx_layer(const hac_desc_t* desc, const void* d_blob, const float* d_X, int64_t B, int64_t ldx, float* d_Y, int64_t ldy,
                           void* d_ws, size_t ws_bytes, hac_stream_t stream)
{
    return product(desc, d_blob, HAC_TYPE_F32, d_X, B, ldx, nullptr, d_Y, ldy, 0, d_ws, ws_bytes, stream, false);
}

extern "C" int mx_encode_dev(uint32_t type, const void* d_W, int64_t count, int64_t n, int64_t m, int64_t ldw, int64_t stride,
                             void* d_blob, size_t blob_capacity, hac_desc_t* desc, hac_stream_t stream)
{
    if (!desc || !d_W || type > HAC_TYPE_BF16 || !aligned(d_W, type)) return HAC_EINVAL;
    hac_desc_t d;
    const int rc = mx_describe(count, n, m, &d);
    if (rc) return rc;
    if (!layout_ok(d, ldw, stride)) return HAC_EINVAL;
    dim3 grid;
    if (!code_grid(d, grid)) return HAC_ERANGE;
    *desc = d;
    if (!d_blob || blob_capacity < d.blob_bytes) return HAC_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(d_blob) % 256) return HAC_EINVAL;
    set_last_hip_error(0);
    note_reset();
    const MxW w = matrices(d, d_blob);
    uint8_t* b = static_cast<uint8_t*>(d_blob);
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const uint64_t apart = count > 1 ? (uint64_t)stride : 0;
    auto launch = [&](auto element, auto stream_it) {
        using T = decltype(element);
        constexpr bool S = decltype(stream_it)::value;
        hipLaunchKernelGGL((mx_encode_kernel<T, S>), grid, dim3(1024), 0, hs, static_cast<const T*>(d_W), (uint64_t)ldw, apart, w, b + d.off_stream,
                           b + d.off_codebook, b, d);
        note_kernel("mx_encode_kernel<%s, %s>", type_name(static_cast<const T*>(d_W)), S ? "true" : "false");
    };
    by_size(d, type, launch);
    return launched();
}

extern "C" int mx_decode_dev(const hac_desc_t* desc, const void* d_blob, uint32_t type, void* d_W, int64_t ldw, int64_t stride,
                             hac_stream_t stream)
{
    if (!desc || !d_blob || !d_W || type > HAC_TYPE_BF16 || !aligned(d_W, type) || !mx_header_ok(*desc)) return HAC_EINVAL;
    if (reinterpret_cast<uintptr_t>(d_blob) % 256 || !layout_ok(*desc, ldw, stride)) return HAC_EINVAL;
    dim3 grid;
    if (!code_grid(*desc, grid)) return HAC_ERANGE;
    set_last_hip_error(0);
    note_reset();
    const MxW w = matrices(*desc, d_blob);
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const uint64_t apart = desc->k_sym > 1 ? (uint64_t)stride : 0;
    auto launch = [&](auto element, auto stream_it) {
        using T = decltype(element);
        constexpr bool S = decltype(stream_it)::value;
        hipLaunchKernelGGL((mx_decode_kernel<T, S>), grid, dim3(1024), 0, hs, static_cast<T*>(d_W), (uint64_t)ldw, apart, w);
        note_kernel("mx_decode_kernel<%s, %s>", type_name(static_cast<const T*>(d_W)), S ? "true" : "false");
    };
    by_size(*desc, type, launch);
    return launched();
}

extern "C" size_t mx_workspace_bytes(const hac_desc_t* desc, uint32_t type, int64_t B, uint32_t flags, int grouped)
{
    if (!desc || !mx_header_ok(*desc) || type > HAC_TYPE_BF16 || (flags & ~HAC_MX_QUANTIZE_X) || B <= 0 || B > kMostRows) return 0;
    if (!grouped && desc->k_sym != 1) return 0;
    return plan_mx(*desc, type, (uint64_t)B, flags, grouped != 0, false).bytes;
}

extern "C" int mx_dot(const hac_desc_t* desc, const void* d_blob, uint32_t type, const void* d_X, int64_t B, int64_t ldx,
                      void* d_Y, int64_t ldy, uint32_t flags, void* d_ws, size_t ws_bytes, hac_stream_t stream)
{
    note_reset();
    return product(desc, d_blob, type, d_X, B, ldx, nullptr, d_Y, ldy, flags, d_ws, ws_bytes, stream, false);
}

extern "C" int mx_grouped_dot(const hac_desc_t* desc, const void* d_blob, uint32_t type, const void* d_X, int64_t B, int64_t ldx,
                              const int32_t* d_offsets, void* d_Y, int64_t ldy, uint32_t flags,
                              void* d_ws, size_t ws_bytes, hac_stream_t stream)
{
    note_reset();
    return product(desc, d_blob, type, d_X, B, ldx, d_offsets, d_Y, ldy, flags, d_ws, ws_bytes, stream, true);
}
