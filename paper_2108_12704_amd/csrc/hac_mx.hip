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
typedef f32x4 f32x4u __attribute__((aligned(4)));                  // global memory takes 128-bit loads at any element
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4u __attribute__((aligned(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
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

template <typename T> struct Block32;
template <> struct Block32<float> {
    f32x4 v[8];
    __device__ __forceinline__ void load(const float* p)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f32x4u*>(p + 4 * i);
    }
    __device__ __forceinline__ void load_part(const float* p, int32_t left)       // the first `left` entries, zeros behind
    {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i / 4][i % 4] = i < left ? p[i] : 0.0f;
    }
    __device__ __forceinline__ uint32_t most() const                             // bits of the largest magnitude
    {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) a = max(a, __float_as_uint(v[i / 4][i % 4]) & 0x7fffffffu);
        return a;
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
    __device__ __forceinline__ void load(const __bf16* p)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const u32x4u*>(p + 8 * i);
    }
    __device__ __forceinline__ void load_part(const __bf16* p, int32_t left)
    {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t lo = 2 * i < left ? q[2 * i] : 0u, hi = 2 * i + 1 < left ? q[2 * i + 1] : 0u;
            v[i / 4][i % 4] = lo | hi << 16;
        }
    }
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t w = v[i / 4][i % 4];
            a = max(a, max(w << 16 & 0x7fff0000u, w & 0x7fff0000u));
        }
        return a;
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

// ---- quantisation and its inverse ------------------------------------------------------------
// A thread has a block: 32 rows of one column, so that the 64 lanes of a wavefront read 64 neighbouring columns row by row and need
// no exchange.  A block of threads covers 64 columns x 512 rows, a group of scales: their bytes meet in LDS.  Bound by memory.
constexpr uint32_t kCodeCols = 64, kCodeRows = 512;

template <typename T>
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
        for (int i = 0; i < 32; ++i) x.v[i / 4][i % 4] = (float)p[(uint64_t)i * ldw];
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

template <typename T>
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
        if ((uint32_t)i < rows) p[(uint64_t)i * ldw] = (T)(byte == 255 ? __builtin_nanf("") : v[i]);
}

// ---- few rows ----------------------------------------------------------------------------------
// At most 16 NR rows of X per group: what counts is to read W once and at once.  A block owns NC tiles of columns, its wavefronts share the
// steps down the rows of W, each reads its tiles straight into operands; X comes from memory (from the L2 after the first block) in
// operand order, is turned into parts or quantised by the lane that holds the block, and the wavefronts' sums are added in LDS in order.
// A lane past the last row reads that row again: what it adds goes to sums that nobody stores.
template <int MODE, typename T, int NR, int NC, int U>
__global__ void __launch_bounds__(512)
mx_rows_kernel(MxW w, const T* __restrict__ X, uint64_t ldx, uint32_t B, const int32_t* __restrict__ offsets,
               T* __restrict__ Y, uint64_t ldy, uint32_t col_blocks)
{
    extern __shared__ __align__(16) f32x4 red[];                 // [wavefronts][NR * NC][64]
    const uint32_t lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const uint32_t wave = uniform(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t stretch = blockIdx.x / col_blocks, cb = blockIdx.x - stretch * col_blocks;
    const Item it = find_item(offsets, w.count, B, 16 * NR, stretch);
    if (!it.rows) return;
    const uint32_t s0 = (uint32_t)((uint64_t)w.steps * wave / waves), s1 = (uint32_t)((uint64_t)w.steps * (wave + 1) / waves);
    const uint32_t full = min(s1, w.n / 128);
    const uint8_t* code[NC];
    const uint8_t* scale[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
        const uint32_t ct = min(cb * NC + q, w.ctiles - 1);
        code[q] = w.codes + it.expert * w.code_stride + (uint64_t)ct * w.steps * 1024 + 16 * lane;
        scale[q] = w.scales + it.expert * w.scale_stride + (uint64_t)ct * w.groups * 256 + 4 * lane;
    }
    const T* row[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) row[r] = X + (uint64_t)(it.row0 + min(16u * r + c, it.rows - 1)) * ldx + 32 * g;
    f32x4 acc[NR][NC];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int q = 0; q < NC; ++q) acc[r][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto multiply = [&](const Block32<T>* x, const u32x4* code4, const uint32_t* byte) ALWAYS_INLINE {
        if constexpr (MODE == FP4) {
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                uint32_t xs;
                const u32x4 xc = quantise(x[r], xs);
#pragma unroll
                for (int q = 0; q < NC; ++q) acc[r][q] = multiply_fp4<0>(code4[q], byte[q], xc, xs, acc[r][q]);
            }
        } else {
            constexpr int P = MODE;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4 p[NR][P];
#pragma unroll
                for (int r = 0; r < NR; ++r) x[r].parts(j, p[r]);
#pragma unroll
                for (int q = 0; q < NC; ++q) {
                    const bf16x8 v = weights(code4[q][j], scale_of(byte[q]));
#pragma unroll
                    for (int r = 0; r < NR; ++r)
#pragma unroll
                        for (int i = P - 1; i >= 0; --i) acc[r][q] = multiply_bf16(v, p[r][i], acc[r][q]);
                }
            }
        }
    };
    uint32_t s = s0;
    for (; s + U <= full; s += U) {
        Block32<T> x[U][NR];
        u32x4 code4[U][NC];
        uint32_t byte[U][NC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int q = 0; q < NC; ++q) {
                code4[u][q] = *reinterpret_cast<const u32x4*>(code[q] + (uint64_t)(s + u) * 1024);
                byte[u][q] = scale[q][(uint64_t)((s + u) / 4) * 256 + (s + u) % 4];
            }
#pragma unroll
            for (int r = 0; r < NR; ++r) x[u][r].load(row[r] + (uint64_t)(s + u) * 128);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(x[u], code4[u], byte[u]);
    }
    for (; s < s1; ++s) {
        Block32<T> x[NR];
        u32x4 code4[NC];
        uint32_t byte[NC];
#pragma unroll
        for (int q = 0; q < NC; ++q) {
            code4[q] = *reinterpret_cast<const u32x4*>(code[q] + (uint64_t)s * 1024);
            byte[q] = scale[q][(uint64_t)(s / 4) * 256 + s % 4];
        }
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            if (s < full) x[r].load(row[r] + (uint64_t)s * 128);
            else x[r].load_part(row[r] + (uint64_t)s * 128, (int32_t)w.n - (int32_t)(s * 128 + 32 * g));
        }
        multiply(x, code4, byte);
    }
    const bool wide = (reinterpret_cast<uintptr_t>(Y) | ldy * sizeof(T)) % (4 * sizeof(T)) == 0;
    auto put = [&](uint32_t r, uint32_t q, uint32_t l, f32x4 v) ALWAYS_INLINE {
        const uint32_t at = 16 * r + (l & 15), col = (cb * NC + q) * 16 + 4 * (l >> 4);
        if (at < it.rows && col < w.m) store4(Y + (uint64_t)(it.row0 + at) * ldy, col, w.m, wide, v);
    };
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int q = 0; q < NC; ++q) red[((size_t)wave * NR * NC + r * NC + q) * 64 + lane] = acc[r][q];
    __syncthreads();
    for (uint32_t o = threadIdx.x; o < NR * NC * 64; o += blockDim.x) {
        f32x4 v = red[o];
        for (uint32_t z = 1; z < waves; ++z) v += red[(size_t)z * NR * NC * 64 + o];
        put(o / 64 / NC, o / 64 % NC, o & 63, v);
    }
}

// ---- many rows -----------------------------------------------------------------------------------
// X is first written in operand order, group by group, each group from a tile of 16 rows of its own on: quantised codes (and their
// scales in groups of four tiles, as W's), or bf16 parts, [tile][step][part][operand j][lane][16 bytes]; zeros behind entry n.
// (A wavefront has a tile's step, a lane a block of its row.)
__host__ __device__ constexpr uint32_t step_bytes(int mode) { return mode == FP4 ? 1024u : 4096u * mode; }

template <int MODE, typename T>
__global__ void __launch_bounds__(256)
mx_lay_out_kernel(const T* __restrict__ X, uint64_t ldx, uint32_t n, uint32_t steps, uint32_t groups, uint32_t B,
                  const int32_t* __restrict__ offsets, uint32_t count, uint8_t* __restrict__ out, uint8_t* __restrict__ out_scales)
{
    __shared__ uint8_t bytes[256];
    const uint32_t lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const uint32_t wave = uniform(threadIdx.x >> 6);
    const uint32_t tile = blockIdx.x, step = blockIdx.y * 4 + wave;
    const Item it = find_item(offsets, count, B, 16, tile);
    if (!it.rows) return;
    const T* row = X + (uint64_t)(it.row0 + min(c, it.rows - 1)) * ldx;
    const uint32_t k = step * 128 + 32 * g;
    Block32<T> x;
    if (k + 32 <= n) x.load(row + k);
    else x.load_part(row + k, k < n ? (int32_t)(n - k) : 0);
    if constexpr (MODE == FP4) {                             // steps: 4 * groups
        uint32_t byte;
        const u32x4 q = quantise(x, byte);
        *reinterpret_cast<u32x4*>(out + (((uint64_t)tile * groups * 4 + step) * 64 + lane) * 16) = q;
        bytes[lane * 4 + wave] = (uint8_t)byte;
        __syncthreads();
        if (threadIdx.x < 64)
            reinterpret_cast<uint32_t*>(out_scales)[((uint64_t)tile * groups + blockIdx.y) * 64 + lane] = reinterpret_cast<const uint32_t*>(bytes)[lane];
    } else {
        if (step >= steps) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 p[MODE];
            x.parts(j, p);
#pragma unroll
            for (int i = 0; i < MODE; ++i)
                *reinterpret_cast<u32x4*>(out + (((((uint64_t)tile * steps + step) * MODE + i) * 4 + j) * 64 + lane) * 16) = p[i];
        }
    }
}

// The product.  A block of 4 wavefronts owns 16 NR rows x 64 NC columns, wavefront w the 16 NC columns from 16 NC w on and all rows.
// A chunk (a step of 128 k; four of them for codes) of X goes to LDS as it lies in memory, one chunk ahead, past the registers; a column
// belongs to one wavefront, so W goes from memory into its registers, a chunk ahead too, and is expanded once per block.
template <int MODE> __host__ __device__ constexpr uint32_t chunk_bytes() { return MODE == FP4 ? 4096u + 256u : step_bytes(MODE); }

__device__ __forceinline__ void to_lds(const uint8_t* from, uint8_t* lds, bool word)
{
    if (word) __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)lds, 4, 0, 0);
    else __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

template <int MODE, typename T, int NR, int NC>
__global__ void __launch_bounds__(256, 2)
mx_tile_kernel(MxW w, const uint8_t* __restrict__ xt, const uint8_t* __restrict__ xs, uint32_t max_tiles, uint32_t B,
               const int32_t* __restrict__ offsets, T* __restrict__ Y, uint64_t ldy, uint32_t stretches, uint32_t col_blocks,
               uint32_t splits, uint32_t per_split, float* __restrict__ part)
{
    constexpr uint32_t CH = chunk_bytes<MODE>(), STAGE = NR * CH;
    extern __shared__ __align__(16) uint8_t lds[];               // two stages
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    // consecutive items on one XCD; the stretches of a column block follow one another and share its part of W in that L2
    const uint32_t id = (blockIdx.x & 7u) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (id >= stretches * col_blocks * splits) return;
    const uint32_t split = id / (stretches * col_blocks), rest = id - split * stretches * col_blocks;
    const uint32_t cb = rest / stretches, stretch = rest - cb * stretches;
    const Item it = find_item(offsets, w.count, B, 16 * NR, stretch);
    const uint32_t tiles = (it.rows + 15) / 16;
    if (!it.rows || it.tile + tiles > max_tiles) return;
    const uint32_t chunks = MODE == FP4 ? w.groups : w.steps;
    const uint32_t c0 = split * per_split, c1 = min(chunks, c0 + per_split);

    const uint8_t* code[NC];
    const uint8_t* scale[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
        const uint32_t ct = min((cb * 4 + wave) * NC + q, w.ctiles - 1);
        code[q] = w.codes + it.expert * w.code_stride + (uint64_t)ct * w.steps * 1024 + 16 * lane;
        scale[q] = w.scales + it.expert * w.scale_stride + (uint64_t)ct * w.groups * 256 + 4 * lane;
    }
    // pieces of 1024 bytes (and of 256 for the scales) are dealt to the wavefronts; rows past the last tile keep what LDS holds
    auto stage = [&](uint32_t ch, uint32_t buf) ALWAYS_INLINE {
        uint8_t* to = lds + buf * STAGE;
        constexpr uint32_t PIECES = (MODE == FP4 ? 4096u : CH) / 1024;
        for (uint32_t z = wave; z < NR * PIECES; z += 4) {
            const uint32_t t = z / PIECES, p = z - t * PIECES;
            if (t >= tiles) break;
            const uint64_t at = MODE == FP4 ? ((uint64_t)(it.tile + t) * w.groups + ch) * 4096 : ((uint64_t)(it.tile + t) * w.steps + ch) * CH;
            to_lds(xt + at + p * 1024 + lane * 16, to + t * (PIECES * 1024) + p * 1024, false);
        }
        if constexpr (MODE == FP4)
            for (uint32_t t = wave; t < tiles; t += 4)
                to_lds(xs + ((uint64_t)(it.tile + t) * w.groups + ch) * 256 + lane * 4, to + NR * 4096 + t * 256, true);
    };
    f32x4 acc[NR][NC];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int q = 0; q < NC; ++q) acc[r][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    constexpr int WS = MODE == FP4 ? 4 : 1;                      // steps of a chunk
    u32x4 cur[WS][NC];
    uint32_t cur_s[NC];
    auto load_w = [&](uint32_t ch, u32x4 (&to)[WS][NC], uint32_t* to_s) ALWAYS_INLINE {
#pragma unroll
        for (int q = 0; q < NC; ++q) {
            if constexpr (MODE == FP4) {
                to_s[q] = *reinterpret_cast<const uint32_t*>(scale[q] + (uint64_t)ch * 256);
#pragma unroll
                for (int s = 0; s < WS; ++s)                     // (behind the last step: any tile, X's codes are 0 there and W's scales too)
                    to[s][q] = *reinterpret_cast<const u32x4*>(code[q] + (uint64_t)min(ch * 4 + s, w.steps - 1) * 1024);
            } else {
                to_s[q] = scale[q][(uint64_t)(ch / 4) * 256 + ch % 4];
                to[0][q] = *reinterpret_cast<const u32x4*>(code[q] + (uint64_t)ch * 1024);
            }
        }
    };
    if (c0 < c1) {
        stage(c0, 0);
        load_w(c0, cur, cur_s);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    for (uint32_t ch = c0; ch < c1; ++ch) {
        const uint8_t* x = lds + ((ch - c0) & 1) * STAGE;
        u32x4 next[WS][NC];
        uint32_t next_s[NC];
        const uint32_t ahead = min(ch + 1, c1 - 1);
        load_w(ahead, next, next_s);
        if (ch + 1 < c1) stage(ch + 1, (ch - c0 + 1) & 1);
        if constexpr (MODE == FP4) {
            uint32_t sx[NR];
#pragma unroll
            for (int r = 0; r < NR; ++r) sx[r] = *reinterpret_cast<const uint32_t*>(x + NR * 4096 + r * 256 + lane * 4);
            auto step = [&](auto which) ALWAYS_INLINE {
                constexpr int S = decltype(which)::value;
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    const u32x4 xc = *reinterpret_cast<const u32x4*>(x + r * 4096 + S * 1024 + lane * 16);
#pragma unroll
                    for (int q = 0; q < NC; ++q) acc[r][q] = multiply_fp4<S>(cur[S][q], cur_s[q], xc, sx[r], acc[r][q]);
                }
            };
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            step(std::integral_constant<int, 2>{});
            step(std::integral_constant<int, 3>{});
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 v[NC];
#pragma unroll
                for (int q = 0; q < NC; ++q) v[q] = weights(cur[0][q][j], scale_of(cur_s[q]));
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int i = MODE - 1; i >= 0; --i) {
                        const u32x4 p = *reinterpret_cast<const u32x4*>(x + r * CH + (i * 4 + j) * 1024 + lane * 16);
#pragma unroll
                        for (int q = 0; q < NC; ++q) acc[r][q] = multiply_bf16(v[q], p, acc[r][q]);
                    }
            }
        }
#pragma unroll
        for (int q = 0; q < NC; ++q) {
            cur_s[q] = next_s[q];
#pragma unroll
            for (int s = 0; s < WS; ++s) cur[s][q] = next[s][q];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    const uint32_t l16 = lane & 15, col0 = (cb * 4 + wave) * NC * 16 + 4 * (lane >> 4);
    const bool wide = (reinterpret_cast<uintptr_t>(Y) | ldy * sizeof(T)) % (4 * sizeof(T)) == 0;
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

// Y = part[0] + part[1] + ... in that order, for the rows that some group holds.
template <typename T>
__global__ void __launch_bounds__(256)
mx_sum_kernel(const float* __restrict__ part, uint32_t splits, uint32_t B, uint32_t m, const int32_t* __restrict__ offsets, uint32_t count,
              T* __restrict__ Y, uint64_t ldy)
{
    uint64_t lo = 0, hi = B;
    if (offsets) {
        lo = (uint64_t)min(max(offsets[0], 0), (int32_t)B);
        hi = (uint64_t)min(max(offsets[count], 0), (int32_t)B);
    }
    const uint64_t total = (uint64_t)B * m, stride = (uint64_t)gridDim.x * blockDim.x;
    for (uint64_t i = lo * m + (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < hi * m; i += stride) {
        float v = part[i];
        uint32_t s = 1;
        for (; s + 3 < splits; s += 4) {
            const float a = part[s * total + i], b = part[(s + 1) * total + i], c = part[(s + 2) * total + i], d = part[(s + 3) * total + i];
            v += a; v += b; v += c; v += d;
        }
        for (; s < splits; ++s) v += part[s * total + i];
        const uint64_t row = i / m;
        Y[row * ldy + (i - row * m)] = (T)v;
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

// What a product launches.  rows: the kernel for few rows, 16 * nr rows a stretch and nc tiles of columns a block of `waves` wavefronts; else X is
// laid out and tiles of 16 nr rows x 64 nc columns are multiplied, the chunks of a column cut into `splits`.
struct Plan {
    bool rows;
    int mode, nr, nc;
    uint32_t waves, splits, per_split;
    uint64_t stretches, col_blocks, tiles;       // stretches, tiles: as many as B rows in `count` groups can fill
    size_t xt_bytes, xs_bytes, part_bytes, bytes;
};

uint64_t fill(uint64_t B, uint64_t count, uint64_t R) { return std::min<uint64_t>(B, (B + (R - 1) * count) / R); }

Plan plan_mx(const hac_desc_t& d, uint32_t type, uint64_t B, uint32_t flags, bool grouped)
{
    const MxShape s = mx_shape(d.n, d.m);
    const uint64_t count = grouped ? d.k_sym : 1;
    Plan p = {};
    p.mode = flags & HAC_MX_QUANTIZE_X ? FP4 : type == HAC_TYPE_F32 ? THREE : ONE;
    const uint64_t used = std::min(count, B), per = (B + used - 1) / used;           // rows a group has on average
    p.rows = per <= 32;
    if (p.rows) {
        p.nr = per <= 16 ? 1 : 2;
        p.stretches = fill(B, count, 16 * p.nr);
        p.nc = 1;
        p.col_blocks = s.ctiles;
        p.waves = (uint32_t)std::min<uint64_t>(8, s.steps);
        return p;
    }
    p.nr = p.mode == THREE ? 4 : per <= 64 ? 4 : 8;
    p.nc = s.ctiles <= 4 ? 1 : s.ctiles <= 8 ? 2 : 4;
    p.stretches = fill(B, count, 16 * p.nr);
    p.col_blocks = (s.ctiles + 4 * p.nc - 1) / (4 * p.nc);
    p.tiles = fill(B, count, 16);
    const uint64_t chunks = p.mode == FP4 ? s.groups : s.steps;
    const uint64_t blocks = (B + 16 * p.nr - 1) / (16 * p.nr) * p.col_blocks;
    uint64_t splits = std::max<uint64_t>(1, std::min<uint64_t>(std::min<uint64_t>(512 / std::max<uint64_t>(blocks, 1), chunks / 2), 16));
    p.per_split = (uint32_t)((chunks + splits - 1) / splits);
    p.splits = (uint32_t)((chunks + p.per_split - 1) / p.per_split);
    auto up = [](uint64_t v) { return (size_t)((v + 255) / 256 * 256); };
    p.xt_bytes = up(p.mode == FP4 ? p.tiles * s.groups * 4096 : p.tiles * s.steps * step_bytes(p.mode));
    p.xs_bytes = p.mode == FP4 ? up(p.tiles * s.groups * 256) : 0;
    p.part_bytes = p.splits > 1 ? up((uint64_t)p.splits * B * d.m * sizeof(float)) : 0;
    p.bytes = p.xt_bytes + p.xs_bytes + p.part_bytes;
    return p;
}

template <int MODE, typename T, int NR, int NC>
int launch_rows(const Plan& p, const MxW& w, const T* X, uint64_t ldx, uint32_t B, const int32_t* offsets, T* Y, uint64_t ldy, hipStream_t stream)
{
    constexpr int U = MODE == THREE ? 2 : 4;
    hipLaunchKernelGGL((mx_rows_kernel<MODE, T, NR, NC, U>), dim3((uint32_t)(p.stretches * p.col_blocks)), dim3(64 * p.waves),
                       (size_t)p.waves * NR * NC * 1024, stream, w, X, ldx, B, offsets, Y, ldy, (uint32_t)p.col_blocks);
    note_kernel("mx_rows_kernel<%d, %s, %d, %d, %d>", MODE, type_name(X), NR, NC, U);
    return launched();
}

template <int MODE, typename T, int NR, int NC>
int launch_tile(const Plan& p, const MxW& w, const uint8_t* xt, const uint8_t* xs, uint32_t B, const int32_t* offsets, T* Y, uint64_t ldy,
                float* part, hipStream_t stream)
{
    auto k = mx_tile_kernel<MODE, T, NR, NC>;
    constexpr size_t lds = 2 * NR * chunk_bytes<MODE>();
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return hip_fail(e);
    }
    const uint64_t items = p.stretches * p.col_blocks * p.splits;
    hipLaunchKernelGGL(k, dim3((uint32_t)((items + 7) / 8 * 8)), dim3(256), lds, stream, w, xt, xs, (uint32_t)p.tiles, B, offsets, Y, ldy,
                       (uint32_t)p.stretches, (uint32_t)p.col_blocks, p.splits, p.per_split, part);
    note_kernel("mx_tile_kernel<%d, %s, %d, %d>", MODE, type_name(Y), NR, NC);
    return launched();
}

template <int MODE, typename T>
int run_mode(const Plan& p, const MxW& w, const T* X, uint64_t ldx, uint32_t B, const int32_t* offsets, T* Y, uint64_t ldy, uint8_t* ws,
             hipStream_t stream)
{
    if (p.rows) {
        if (p.nr == 1) return launch_rows<MODE, T, 1, 1>(p, w, X, ldx, B, offsets, Y, ldy, stream);
        return launch_rows<MODE, T, 2, 1>(p, w, X, ldx, B, offsets, Y, ldy, stream);
    }
    uint8_t* xt = ws;
    uint8_t* xs = ws + p.xt_bytes;
    float* part = reinterpret_cast<float*>(ws + p.xt_bytes + p.xs_bytes);
    hipLaunchKernelGGL((mx_lay_out_kernel<MODE, T>), dim3((uint32_t)p.tiles, w.groups), dim3(256), 0, stream, X, ldx, w.n, w.steps, w.groups, B,
                       offsets, w.count, xt, xs);
    note_kernel("mx_lay_out_kernel<%d, %s>", MODE, type_name(X));
    int rc = launched();
    if (rc) return rc;
    constexpr int MOST = MODE == THREE ? 4 : 8;
    if (p.nr == MOST) {
        rc = p.nc == 1 ? launch_tile<MODE, T, MOST, 1>(p, w, xt, xs, B, offsets, Y, ldy, part, stream)
           : p.nc == 2 ? launch_tile<MODE, T, MOST, 2>(p, w, xt, xs, B, offsets, Y, ldy, part, stream)
                       : launch_tile<MODE, T, MOST, 4>(p, w, xt, xs, B, offsets, Y, ldy, part, stream);
    } else {
        rc = p.nc == 1 ? launch_tile<MODE, T, 4, 1>(p, w, xt, xs, B, offsets, Y, ldy, part, stream)
           : p.nc == 2 ? launch_tile<MODE, T, 4, 2>(p, w, xt, xs, B, offsets, Y, ldy, part, stream)
                       : launch_tile<MODE, T, 4, 4>(p, w, xt, xs, B, offsets, Y, ldy, part, stream);
    }
    if (rc || p.splits == 1) return rc;
    const uint64_t total = (uint64_t)B * w.m;
    hipLaunchKernelGGL(mx_sum_kernel<T>, dim3((uint32_t)std::min<uint64_t>((total + 255) / 256, 4096)), dim3(256), 0, stream, part, p.splits, B,
                       w.m, offsets, w.count, Y, ldy);
    note_kernel("mx_sum_kernel<%s>", type_name(Y));
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
bool grids_fit(const Plan& p, const MxShape& s)
{
    if (p.rows) return p.stretches * p.col_blocks <= 0xffffffffull / (64 * p.waves);
    return p.tiles <= 0xffffffull && s.groups <= 65535 && p.stretches <= 0xffffffull && p.stretches * p.col_blocks * p.splits <= 0xfffff0ull;
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
    const Plan p = plan_mx(*desc, type, (uint64_t)B, flags, grouped);
    if (!grids_fit(p, mx_shape(desc->n, desc->m))) return HAC_ERANGE;
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
    if (type == HAC_TYPE_F32)
        hipLaunchKernelGGL(mx_encode_kernel<float>, grid, dim3(1024), 0, hs, static_cast<const float*>(d_W), (uint64_t)ldw, apart, w,
                           b + d.off_stream, b + d.off_codebook, b, d);
    else
        hipLaunchKernelGGL(mx_encode_kernel<__bf16>, grid, dim3(1024), 0, hs, static_cast<const __bf16*>(d_W), (uint64_t)ldw, apart, w,
                           b + d.off_stream, b + d.off_codebook, b, d);
    note_kernel("mx_encode_kernel<%s>", type == HAC_TYPE_F32 ? "float" : "__bf16");
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
    if (type == HAC_TYPE_F32) hipLaunchKernelGGL(mx_decode_kernel<float>, grid, dim3(1024), 0, hs, static_cast<float*>(d_W), (uint64_t)ldw, apart, w);
    else hipLaunchKernelGGL(mx_decode_kernel<__bf16>, grid, dim3(1024), 0, hs, static_cast<__bf16*>(d_W), (uint64_t)ldw, apart, w);
    note_kernel("mx_decode_kernel<%s>", type == HAC_TYPE_F32 ? "float" : "__bf16");
    return launched();
}

extern "C" size_t mx_workspace_bytes(const hac_desc_t* desc, uint32_t type, int64_t B, uint32_t flags, int grouped)
{
    if (!desc || !mx_header_ok(*desc) || type > HAC_TYPE_BF16 || (flags & ~HAC_MX_QUANTIZE_X) || B <= 0 || B > kMostRows) return 0;
    if (!grouped && desc->k_sym != 1) return 0;
    return plan_mx(*desc, type, (uint64_t)B, flags, grouped != 0).bytes;
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
