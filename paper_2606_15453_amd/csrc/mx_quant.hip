// Matrices to and from microscaled 4-bit floats (mx_format.h), and the packed
// expert blob.
//
// Quantising is one pass: a lane takes eight columns (16 bytes of bf16), the
// four lanes of a block share the largest magnitude by two lane exchanges, and
// the hardware conversion divides by the scale and rounds.  The bound is the
// bytes: esz in and 17/32 out per element.
#include "mx_format.h"

namespace stmoe {
namespace {

using namespace mx;

constexpr int kThreads = 256;
constexpr int kUnit = 8;                        // columns per lane
constexpr int kUnitsPerBlock = kBlock / kUnit;  // lanes per block

template <bool BF>
__device__ __forceinline__ void load_unit(const void* x, int64_t at, int n, bool vec, float (&v)[kUnit]) {
    if (BF) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(x) + at;
        if (vec && n == kUnit) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
            v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) v[i] = i < n ? __uint_as_float(uint32_t(p[i]) << 16) : 0.f;
        }
    } else {
        const float* p = reinterpret_cast<const float*>(x) + at;
        if (vec && n == kUnit) {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) v[i] = i < n ? p[i] : 0.f;
        }
    }
}

// `vec`: x and its row stride are 16-byte aligned.  `vec_out`: so are the rows
// of codes to 4 bytes.
template <bool BF>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const void* x, int64_t rows, int cols, int64_t ld,
                                                              uint8_t* codes, uint8_t* scales, int vec, int vec_out) {
    const int nb = (cols + kBlock - 1) / kBlock, upr = nb * kUnitsPerBlock, cb = (cols + 1) / 2;
    const int64_t total = rows * upr, step = int64_t(gridDim.x) * kThreads;
    // the four lanes of a block run the same rounds: total and kThreads are multiples of four
    for (int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x; u < total; u += step) {
        const int64_t row = u / upr;
        const int c = int(u - row * upr), col = c * kUnit;
        const int n = cols - col < 0 ? 0 : cols - col < kUnit ? cols - col : kUnit;
        float v[kUnit];
        load_unit<BF>(x, row * ld + col, n, vec != 0, v);
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < kUnit; ++i) {
            const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
            top = a > top ? a : top;
        }
#pragma unroll
        for (int m = 1; m < kUnitsPerBlock; m <<= 1) {
            const uint32_t o = uint32_t(__shfl_xor(int(top), m, 64));
            top = o > top ? o : top;
        }
        const uint32_t s = scale_byte(top);
        const uint32_t q = s == 255u ? 0u : encode8(v, scale_of(s));
        uint8_t* o = codes + row * cb + col / 2;
        if (vec_out && n == kUnit) {
            *reinterpret_cast<uint32_t*>(o) = q;
        } else {
            for (int i = 0; 2 * i < n; ++i) o[i] = uint8_t(q >> (8 * i));
        }
        if (c % kUnitsPerBlock == 0) scales[row * nb + c / kUnitsPerBlock] = uint8_t(s);
    }
}

template <bool BF>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const uint8_t* codes, const uint8_t* scales,
                                                                int64_t rows, int cols, void* y, int64_t ld,
                                                                int vec_in, int vec) {
    const int nb = (cols + kBlock - 1) / kBlock, upr = (cols + kUnit - 1) / kUnit, cb = (cols + 1) / 2;
    const int64_t total = rows * upr, step = int64_t(gridDim.x) * kThreads;
    for (int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x; u < total; u += step) {
        const int64_t row = u / upr;
        const int c = int(u - row * upr), col = c * kUnit;
        const int n = cols - col < kUnit ? cols - col : kUnit;
        const uint8_t* p = codes + row * cb + col / 2;
        uint32_t q = 0u;
        if (vec_in && n == kUnit) {
            q = *reinterpret_cast<const uint32_t*>(p);
        } else {
            for (int i = 0; 2 * i < n; ++i) q |= uint32_t(p[i]) << (8 * i);
        }
        const float s = scale_of(scales[row * nb + c / kUnitsPerBlock]);
        union {
            bf16x8 v;
            uint4 q;
            uint16_t h[8];
        } d;
        d.v = decode8(q, s);
        if (BF) {
            uint16_t* o = reinterpret_cast<uint16_t*>(y) + row * ld + col;
            if (vec && n == kUnit) {
                *reinterpret_cast<uint4*>(o) = d.q;
            } else {
                for (int i = 0; i < n; ++i) o[i] = d.h[i];
            }
        } else {
            float* o = reinterpret_cast<float*>(y) + row * ld + col;
            if (vec && n == kUnit) {
                *reinterpret_cast<float4*>(o) = make_float4(bf16_lo(d.q.x), bf16_hi(d.q.x), bf16_lo(d.q.y), bf16_hi(d.q.y));
                *reinterpret_cast<float4*>(o + 4) =
                    make_float4(bf16_lo(d.q.z), bf16_hi(d.q.z), bf16_lo(d.q.w), bf16_hi(d.q.w));
            } else {
                for (int i = 0; i < n; ++i) o[i] = __uint_as_float(uint32_t(d.h[i]) << 16);
            }
        }
    }
}

// One lane piece (16 code bytes and a scale byte) per thread; not a hot path:
// an expert is packed once.
__global__ __launch_bounds__(kThreads) void mx_pack_kernel(const uint8_t* codes, const uint8_t* scales, int rows,
                                                          int cols, uint8_t* out, uint8_t* out_s) {
    const int KT = col_tiles(cols), KG = col_groups(cols), nb = (cols + kBlock - 1) / kBlock, cb = cols / 2;
    const int64_t total = int64_t(row_blocks(rows)) * KG * kGroupTiles * 64;
    const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= total) return;
    const int lane = int(i % 64), kt = int(i / 64 % (KG * kGroupTiles));
    const int rb = int(i / 64 / (KG * kGroupTiles));
    const int row = rb * kTileRows + lane % 16, blk = kt * 4 + lane / 16;
    const bool in = row < rows && blk < nb;
    if (kt < KT) {
        uint8_t* o = out + (size_t(rb) * KT + kt) * kTileBytes + lane * 16;
        for (int b = 0; b < 16; ++b) {
            const int at = blk * 16 + b;
            o[b] = in && at < cb ? codes[size_t(row) * cb + at] : 0;
        }
    }
    out_s[(size_t(rb) * KG + kt / kGroupTiles) * kGroupBytes + lane * 4 + kt % kGroupTiles] =
        in ? scales[size_t(row) * nb + blk] : 0;
}

int grid_of(int64_t units) {
    const int64_t wg = (units + kThreads - 1) / kThreads;
    return int(wg < 1 ? 1 : wg < 65536 ? wg : 65536);
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

int check_matrix(const char* fn, int64_t rows, int cols, int64_t ld, int dtype) {
    const char* bad = nullptr;
    if (rows < 0 || rows > (int64_t(1) << 31)) bad = "rows must be in [0, 2^31]";
    else if (cols < 1 || cols > (1 << 30)) bad = "cols must be in [1, 2^30]";
    else if (ld < cols || ld > (int64_t(1) << 31)) bad = "the row stride must be in [cols, 2^31]";
    else if (dtype != STMOE_BF16 && dtype != STMOE_F32) bad = "dtype must be STMOE_BF16 or STMOE_F32";
    if (!bad) return STMOE_OK;
    set_error(std::string(fn) + ": " + bad);
    return STMOE_EINVAL;
}

}  // namespace
}  // namespace stmoe

using namespace stmoe;

extern "C" int moe_mx_quantize(const void* x, int64_t rows, int cols, int64_t ld, int dtype, uint8_t* codes,
                               uint8_t* scales, void* stream) {
    clear_error();
    if (int rc = check_matrix(__func__, rows, cols, ld, dtype)) return rc;
    if (rows == 0) return STMOE_OK;
    STMOE_CHECK(x && codes && scales, "null pointer");
    const size_t esz = dtype == STMOE_BF16 ? 2 : 4;
    STMOE_CHECK(aligned(x, esz), "x must be aligned to its elements");
    const int vec = aligned(x, 16) && ld * esz % 16 == 0, vec_out = aligned(codes, 4) && (cols + 1) / 2 % 4 == 0;
    const int nb = (cols + mx::kBlock - 1) / mx::kBlock;
    const dim3 grid(unsigned(grid_of(rows * nb * kUnitsPerBlock)));
    if (dtype == STMOE_BF16)
        hipLaunchKernelGGL((mx_quantize_kernel<true>), grid, dim3(kThreads), 0, as_stream(stream), x, rows, cols, ld,
                           codes, scales, vec, vec_out);
    else
        hipLaunchKernelGGL((mx_quantize_kernel<false>), grid, dim3(kThreads), 0, as_stream(stream), x, rows, cols, ld,
                           codes, scales, vec, vec_out);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

extern "C" int moe_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, void* y,
                                 int64_t ld, int dtype, void* stream) {
    clear_error();
    if (int rc = check_matrix(__func__, rows, cols, ld, dtype)) return rc;
    if (rows == 0) return STMOE_OK;
    STMOE_CHECK(y && codes && scales, "null pointer");
    const size_t esz = dtype == STMOE_BF16 ? 2 : 4;
    STMOE_CHECK(aligned(y, esz), "y must be aligned to its elements");
    const int vec = aligned(y, 16) && ld * esz % 16 == 0, vec_in = aligned(codes, 4) && (cols + 1) / 2 % 4 == 0;
    const dim3 grid(unsigned(grid_of(rows * ((cols + kUnit - 1) / kUnit))));
    if (dtype == STMOE_BF16)
        hipLaunchKernelGGL((mx_dequantize_kernel<true>), grid, dim3(kThreads), 0, as_stream(stream), codes, scales,
                           rows, cols, y, ld, vec_in, vec);
    else
        hipLaunchKernelGGL((mx_dequantize_kernel<false>), grid, dim3(kThreads), 0, as_stream(stream), codes, scales,
                           rows, cols, y, ld, vec_in, vec);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

extern "C" int moe_mx_pack_expert(const uint8_t* gate_codes, const uint8_t* gate_scales, const uint8_t* up_codes,
                                  const uint8_t* up_scales, const uint8_t* down_codes, const uint8_t* down_scales,
                                  int H, int I, void* blob_out, void* stream) {
    clear_error();
    STMOE_CHECK(gate_codes && gate_scales && up_codes && up_scales && down_codes && down_scales && blob_out,
                "null pointer");
    STMOE_CHECK(H >= 8 && H % 8 == 0 && H <= kMaxH, "H must be a multiple of 8 in [8, 16384]");
    STMOE_CHECK(I >= 8 && I % 8 == 0 && I <= mx::kMaxI, "I must be a multiple of 8 in [8, 65536]");
    STMOE_CHECK(aligned(blob_out, 16), "the blob must be 16-byte aligned");
    const mx::Blob b = mx::blob(H, I);
    uint8_t* o = reinterpret_cast<uint8_t*>(blob_out);
    const struct {
        const uint8_t *c, *s;
        int rows, cols;
        size_t at, at_s;
    } m[3] = {{gate_codes, gate_scales, I, H, b.gate, b.gate_s},
              {up_codes, up_scales, I, H, b.up, b.up_s},
              {down_codes, down_scales, H, I, b.down, b.down_s}};
    for (const auto& k : m) {
        const int64_t total = int64_t(mx::row_blocks(k.rows)) * mx::col_groups(k.cols) * mx::kGroupTiles * 64;
        hipLaunchKernelGGL(mx_pack_kernel, dim3(unsigned((total + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                           as_stream(stream), k.c, k.s, k.rows, k.cols, o + k.at, o + k.at_s);
        STMOE_LAUNCHED();
    }
    return STMOE_OK;
}
