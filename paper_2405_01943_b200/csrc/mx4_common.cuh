// Microscaled 4-bit values (e2m1 codes in blocks of 32 along k that share a power-of-two scale): the layout of codes and
// scales, and their decoding.  Internal header; include/dass.h states the format.
#pragma once

#include "dass_device.cuh"

namespace dass {

constexpr int MX4_BLOCK = 32;          // values of a scale
constexpr int MX4_TILE_ROWS = 128;     // a scale tile: 128 rows x 4 blocks, 512 bytes
constexpr int MX4_TILE_K = 128;
constexpr int MX4_TILE_BYTES = 512;

// Bytes of a row of codes, and scale tiles along k and along the rows.
__host__ __device__ __forceinline__ int64_t mx4_pitch(int64_t K) { return (K + MX4_BLOCK - 1) / MX4_BLOCK * (MX4_BLOCK / 2); }
__host__ __device__ __forceinline__ int64_t mx4_k_tiles(int64_t K) { return (K + MX4_TILE_K - 1) / MX4_TILE_K; }
__host__ __device__ __forceinline__ int64_t mx4_row_tiles(int64_t rows) { return (rows + MX4_TILE_ROWS - 1) / MX4_TILE_ROWS; }
inline int64_t mx4_codes_bytes(int64_t rows, int64_t K) { return rows * mx4_pitch(K); }
inline int64_t mx4_scales_bytes(int64_t rows, int64_t K) { return mx4_row_tiles(rows) * mx4_k_tiles(K) * MX4_TILE_BYTES; }

// Where the four scales of a row's k tile stand (one 32-bit word; block b of the tile is byte b).
__host__ __device__ __forceinline__ int64_t mx4_scale_word(int64_t row, int64_t k_tile, int64_t k_tiles)
{
    return ((row >> 7) * k_tiles + k_tile) * MX4_TILE_BYTES + (row & 31) * 16 + ((row >> 5) & 3) * 4;
}

// 2^(s - 127), NaN for s = 255; s = 0 is the subnormal 2^-127.
__device__ __forceinline__ float mx4_scale(uint32_t s)
{
    return __uint_as_float(s == 255u ? 0x7fffffffu : s == 0u ? 0x00400000u : s << 23);
}

// Decoding to bf16.  The 3 bits below the sign of a code, put where bf16 has the last two bits of its exponent and the
// first of its mantissa, are the code's value times 2^-126 (a subnormal where the code is one): one exact product with
// 2^(s - 1) gives the value.  For s up to 128 that factor is a bf16 itself; scales above 2, which blocks have whose largest
// value is 16 or more, take two products (1 x 4096 x 4096 with all of its scales above 2: 7.0 us instead of 6.7).
struct Mx4Factor { uint32_t first, second; };              // bf16 pairs; second is used where `two`
__device__ __forceinline__ bool mx4_two(uint32_t s) { return s > 128u && s < 255u; }
__device__ __forceinline__ Mx4Factor mx4_factor(uint32_t s)
{
    const uint32_t a = s == 255u ? 0x7fffu : s > 128u ? 0x7f00u : (s + 126u) << 7;     // 2^(s - 1), at most 2^127
    const uint32_t b = mx4_two(s) ? (s - 1u) << 7 : 0x3f80u;                           // 2^(s - 128), or 1
    return {a * 0x10001u, b * 0x10001u};
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// 8 codes (the first in the lowest bits) as bf16 pairs: w[p] holds codes p (low half) and p + 4 (high half).  A nibble's two
// copies, for the sign and for the value, are made by one product.
__device__ __forceinline__ void mx4_decode8(uint32_t x, const Mx4Factor &f, bool two, uint32_t (&w)[4])
{
    const uint32_t y = x >> 8;
    w[0] = ((x & 0x000f000fu) * 0x1040u) & 0x81c081c0u;
    w[1] = ((x & 0x00f000f0u) * 0x0104u) & 0x81c081c0u;
    w[2] = ((y & 0x000f000fu) * 0x1040u) & 0x81c081c0u;
    w[3] = ((y & 0x00f000f0u) * 0x0104u) & 0x81c081c0u;
#pragma unroll
    for (int p = 0; p < 4; ++p) w[p] = mul_bf16x2(w[p], f.first);
    if (two) {
#pragma unroll
        for (int p = 0; p < 4; ++p) w[p] = mul_bf16x2(w[p], f.second);
    }
}

// Two floats to two codes each, four pairs: v[0] in the lowest bits.
__device__ __forceinline__ uint32_t mx4_encode8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// 8 codes as floats times `scale`, in order.
__device__ __forceinline__ void mx4_decode8_f32(uint32_t x, float scale, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = x >> (4 * i);
        // the code's 3 lower bits at the end of f32's exponent field: its value times 2^-126
        const float t = __uint_as_float(((c & 8u) << 28) | ((c & 7u) << 22)) * 8.507059173023462e37f;      // 2^126
        v[i] = t * scale;
    }
}

}  // namespace dass
