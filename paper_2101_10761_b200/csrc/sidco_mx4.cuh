// Microscaled 4-bit numbers (blocks of 32 E2M1 codes with one E8M0 scale) on sm_100a: the conversions and the layout
// that the quantiser, the reader, the dense compressor and the product share.
//
// A block's scale is 2^e, e = floor(log2 max|x|) - 2 held to [-127, 125], stored as the byte e + 127; its codes are
// x 2^-e rounded to {0, .5, 1, 1.5, 2, 3, 4, 6} (ties to the even code, larger magnitudes to 6), the sign kept.  In
// terms of the bits of max|x|: the byte is the biased exponent minus two, at least 0.  A block that holds a NaN or an
// infinity gets the byte 255 (NaN) and zero codes.  Every scaling is by a power of two, so that the only rounding is
// the one to the grid, and results do not depend on how the work is split.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace sidco_mx4 {

constexpr int kBlock = 32;            // elements per scale
constexpr int kTileRows = 128;        // a tile of scales is 128 rows x 4 blocks = 512 bytes
constexpr int kTileBlocks = 4;
constexpr int kTileBytes = kTileRows * kTileBlocks;

__host__ __device__ constexpr int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

// Byte of (row, block) inside its 512-byte tile: the order in which the tensor cores' scale memory takes it (32 lanes
// of 16 bytes; a lane's four words are the rows 32 apart, a word's bytes are four neighbouring blocks).
__host__ __device__ constexpr int scale_in_tile(int row, int block) {
    return (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// From the first scale of a row to that of its eight neighbours `oct`: 64 bits, a row may have 2^31 columns.
__host__ __device__ constexpr int64_t scale_of_oct(int64_t oct) {
    return (oct >> 4) * kTileBytes + ((oct >> 2) & (kTileBlocks - 1));
}

// Scale byte from the bits of the largest magnitude of a block.
__device__ __forceinline__ uint32_t scale_byte(uint32_t max_bits) {
    const uint32_t ex = max_bits >> 23;
    return ex == 255u ? 255u : (ex > 2u ? ex - 2u : 0u);
}

// 2^(byte - 127); a NaN for 255.
__device__ __forceinline__ float scale_of(uint32_t byte) {
    return __uint_as_float(byte == 0u ? 0x00400000u : (byte == 255u ? 0x7fffffffu : byte << 23));
}

// 2^(127 - byte); 0 for 255, so that finite values of a block marked NaN become zero codes.
__device__ __forceinline__ float inverse_scale_of(uint32_t byte) {
    return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23);
}

// Eight codes, element 0 in the lowest four bits.
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], float inv) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(x[0] * inv), "f"(x[1] * inv), "f"(x[2] * inv), "f"(x[3] * inv), "f"(x[4] * inv), "f"(x[5] * inv),
          "f"(x[6] * inv), "f"(x[7] * inv));
    return r;
}

// The grid values of eight codes (without the scale).
__device__ __forceinline__ void decode8(uint32_t codes, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

}  // namespace sidco_mx4
