// Microscaled 4-bit floats (MXFP4): the element grid, the packed expert blob
// and the device conversions.
//
// A block is 32 consecutive columns of a row.  Its scale is a power of two
// 2^(s - 127) held as the byte s (255: the block is NaN), its elements are
// E2M1 codes: bit 3 the sign, bits 0..2 the magnitude 0, 0.5, 1, 1.5, 2, 3, 4, 6.
// Every value has at most two significant bits, so it is exact in bf16 and
// fp32 (below the smallest normal number as a subnormal one).
//
// Packed expert: the codes of W_gate [I][H], W_up [I][H], W_down [H][I], then
// their scales.  A matrix [R][C] is cut into tiles of 16 rows x 128 columns,
// row block by row block; a tile's 1024 code bytes lie as the 16-byte pieces
// of the lanes of a wave: lane l has row l % 16 and the block of 32 columns
// l / 16, which is the row operand of four 16x16x32 matrix instructions, so a
// wave reads one contiguous KiB per tile.  Scales lie in groups of four tiles: lane l's four
// bytes at 4 l of 256.  Rows and columns beyond the matrix hold zero codes.
#pragma once

#include "common.h"

namespace stmoe {
namespace mx {

constexpr int kBlock = 32;          // columns per scale
constexpr int kTileRows = 16;
constexpr int kTileCols = 128;
constexpr int kTileBytes = kTileRows * kTileCols / 2;
constexpr int kGroupTiles = 4;      // tiles whose scales lie together
constexpr int kGroupBytes = 256;
constexpr int kMaxI = 65536;

inline __host__ __device__ int row_blocks(int rows) { return (rows + kTileRows - 1) / kTileRows; }
inline __host__ __device__ int col_tiles(int cols) { return (cols + kTileCols - 1) / kTileCols; }
inline __host__ __device__ int col_groups(int cols) { return (col_tiles(cols) + kGroupTiles - 1) / kGroupTiles; }
inline __host__ __device__ size_t code_bytes(int rows, int cols) {
    return size_t(row_blocks(rows)) * col_tiles(cols) * kTileBytes;
}
inline __host__ __device__ size_t scale_bytes(int rows, int cols) {
    return size_t(row_blocks(rows)) * col_groups(cols) * kGroupBytes;
}

// Byte offsets inside a packed expert.
struct Blob {
    size_t gate, up, down, gate_s, up_s, down_s, total;
};
inline __host__ __device__ Blob blob(int H, int I) {
    Blob b;
    b.gate = 0;
    b.up = code_bytes(I, H);
    b.down = 2 * b.up;
    b.gate_s = b.down + code_bytes(H, I);
    b.up_s = b.gate_s + scale_bytes(I, H);
    b.down_s = b.up_s + scale_bytes(I, H);
    b.total = b.down_s + scale_bytes(H, I);
    return b;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The conversions take the scale as a float and use its exponent field alone:
// byte s sits there as s << 23 (0 is 2^-127, 255 NaN).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes (a word, lowest nibble first) -> eight bf16 values, exact.
__device__ __forceinline__ bf16x8 decode8(uint32_t codes, float scale) {
    union {
        bf16x2 p[4];
        bf16x8 v;
    } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return u.v;
}

// Eight values / scale -> codes, round to nearest (ties to the even code),
// saturating at 6.
__device__ __forceinline__ uint32_t encode8(const float (&v)[8], float scale) {
    uint32_t c = 0u;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return c;
}

// Scale byte of a block whose largest magnitude has the bits `top` (sign
// cleared): its exponent less 2, the exponent of the grid's 4..6, so that the
// largest element lands in [4, 8); at least 0; 255 for infinities and NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}

}  // namespace mx
}  // namespace stmoe
