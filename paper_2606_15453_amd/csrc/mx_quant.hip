// Matrices to and from microscaled 4-bit floats (mx_format.h), and the packed
// expert blob.
//
// Quantising is one pass: a lane takes eight columns (16 bytes of bf16), the
// four lanes of a block share the largest magnitude by two lane exchanges, and
// the hardware conversion divides by the scale and rounds.  The bound is the
// bytes, esz and 17/32 per element: 14336 x 4096 bf16 takes 26.7 us one way (5.6
// TB/s) and 22.6 back (6.6), medians of a trace.
#include "mx_format.h"

namespace stmoe {
namespace {

using namespace mx;

constexpr int kThreads = 256;
constexpr int kUnit = 8;                        // columns per lane
constexpr int kUnitsPerBlock = kBlock / kUnit;  // lanes per block

// Rows start at any element: the loads and stores below are whole vectors of
// their type's own alignment, which the memory pipeline takes at any address.
// x is read once, past the caches (14336 x 4096 bf16: 29.9 us through them, 26.7
// past them).
template <class V, class E>
__device__ __forceinline__ V load_once(const E* p) {
    typedef V Any __attribute__((aligned(alignof(E))));
    return __builtin_nontemporal_load(reinterpret_cast<const Any*>(p));
}
template <class V, class E>
__device__ __forceinline__ V load_vec(const E* p) {
    V v;
    __builtin_memcpy(&v, __builtin_assume_aligned(p, alignof(E)), sizeof(V));
    return v;
}
template <class V, class E>
__device__ __forceinline__ void store_vec(E* p, V v) {
    __builtin_memcpy(__builtin_assume_aligned(p, alignof(E)), &v, sizeof(V));
}

template <bool BF>
__device__ __forceinline__ void load_unit(const void* x, int64_t at, int n, float (&v)[kUnit]) {
    if (BF) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(x) + at;
        if (n == kUnit) {
            const u32x4 q = load_once<u32x4>(p);
#pragma unroll
            for (int i = 0; i < kUnit; ++i) v[i] = i % 2 ? bf16_hi(q[i / 2]) : bf16_lo(q[i / 2]);
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) v[i] = i < n ? __uint_as_float(uint32_t(p[i]) << 16) : 0.f;
        }
    } else {
        const float* p = reinterpret_cast<const float*>(x) + at;
        if (n == kUnit) {
            const f32x4 a = load_once<f32x4>(p), b = load_once<f32x4>(p + 4);
#pragma unroll
            for (int i = 0; i < kUnit; ++i) v[i] = i < 4 ? a[i & 3] : b[i & 3];
        } else {
#pragma unroll
            for (int i = 0; i < kUnit; ++i) v[i] = i < n ? p[i] : 0.f;
        }
    }
}

// A unit's row and column.  FLAT: whole blocks in contiguous rows, where the
// matrix is one long row (14336 x 4096 bf16: 26.7 us, 30.2 without; reading back
// 22.6 and 24.0); else a division, of 32 bits where the units allow it.
template <bool FLAT, int W>
__device__ __forceinline__ void place(int64_t u, int upr, int64_t& row, int& col) {
    if (FLAT) return;
    if (u >> 32 == 0) {
        row = int64_t(uint32_t(u) / uint32_t(upr));
    } else {
        row = u / upr;
    }
    col = int(u - row * upr) * W;
}

template <bool BF, bool FLAT>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const void* x, int64_t rows, int cols, int64_t ld,
                                                              uint8_t* codes, uint8_t* scales) {
    const int nb = (cols + kBlock - 1) / kBlock, upr = nb * kUnitsPerBlock, cb = (cols + 1) / 2;
    const int64_t total = rows * upr, step = int64_t(gridDim.x) * kThreads;
    // the four lanes of a block go together: total and kThreads are multiples of four
    for (int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x; u < total; u += step) {
        float v[kUnit];
        int64_t row = 0;
        int col = 0;
        place<FLAT, kUnit>(u, upr, row, col);
        const int n = FLAT ? kUnit : max(0, min(kUnit, cols - col));
        load_unit<BF>(x, FLAT ? u * kUnit : row * ld + col, n, v);
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < kUnit; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
        // the block's four lanes: their neighbour, then the other pair
        top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0xB1, 0xf, 0xf, false)));
        top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0x4E, 0xf, 0xf, false)));
        const uint32_t s = scale_byte(top);
        const uint32_t q = s == 255u ? 0u : encode8(v, scale_of(s));
        if (FLAT) {
            reinterpret_cast<uint32_t*>(codes)[u] = q;
            if (u % kUnitsPerBlock == 0) scales[u / kUnitsPerBlock] = uint8_t(s);
            continue;
        }
        uint8_t* o = codes + row * cb + col / 2;
        if (n == kUnit) {
            store_vec(o, q);
        } else {
#pragma unroll
            for (int i = 0; i < kUnit / 2; ++i)
                if (2 * i < n) o[i] = uint8_t(q >> (8 * i));
        }
        if (col % kBlock == 0) scales[row * nb + col / kBlock] = uint8_t(s);
    }
}

// Reading back, a lane takes the columns of one 16-byte store, so that a wave's
// stores are contiguous (1000 x 2061 fp32: 17 us with eight columns a lane, 5
// with four).
template <bool BF>
constexpr int kOut = BF ? 8 : 4;

template <bool BF>
__device__ __forceinline__ void store_unit(void* y, int64_t at, int n, uint32_t codes, float scale) {
    const bf16x8 d = decode8(codes, scale);
    if (BF) {
        __bf16* o = reinterpret_cast<__bf16*>(y) + at;
        if (n == 8) {
            store_vec(o, d);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) o[i] = d[i];
        }
    } else {
        float* o = reinterpret_cast<float*>(y) + at;
        if (n == 4) {
            store_vec(o, f32x4{float(d[0]), float(d[1]), float(d[2]), float(d[3])});
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) o[i] = float(d[i]);
        }
    }
}

template <bool BF, bool FLAT>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const uint8_t* codes, const uint8_t* scales,
                                                                int64_t rows, int cols, void* y, int64_t ld) {
    constexpr int W = kOut<BF>, PB = kBlock / W;            // columns per lane, lanes per block
    const int nb = (cols + kBlock - 1) / kBlock, upr = (cols + W - 1) / W, cb = (cols + 1) / 2;
    const int64_t total = rows * upr, step = int64_t(gridDim.x) * kThreads;
    for (int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x; u < total; u += step) {
        int64_t row = 0;
        int col = 0;
        place<FLAT, W>(u, upr, row, col);
        const int n = FLAT ? W : min(W, cols - col);
        const uint8_t* p = codes + (FLAT ? u * (W / 2) : row * cb + col / 2);
        uint32_t q = 0u;
        if (n == W) {
            q = W == 8 ? load_vec<uint32_t>(p) : load_vec<uint16_t>(p);
        } else {
#pragma unroll
            for (int i = 0; i < W / 2; ++i)
                if (2 * i < n) q |= uint32_t(p[i]) << (8 * i);
        }
        const uint32_t s = scales[FLAT ? u / PB : row * nb + col / kBlock];
        store_unit<BF>(y, FLAT ? u * W : row * ld + col, n, q, scale_of(s));
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

// A unit per lane, in at most 16384 workgroups (with 4096 or 65536 up to 5% more at
// some sizes).
int grid_of(int64_t units) {
    const int64_t wg = (units + kThreads - 1) / kThreads;
    return int(wg < 1 ? 1 : wg < 16384 ? wg : 16384);
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
    const int nb = (cols + mx::kBlock - 1) / mx::kBlock;
    const dim3 grid(unsigned(grid_of(rows * nb * kUnitsPerBlock))), block(kThreads);
    const bool flat = ld == cols && cols % mx::kBlock == 0 && aligned(codes, 4);
    hipStream_t s = as_stream(stream);
    if (dtype == STMOE_BF16) {
        if (flat) hipLaunchKernelGGL((mx_quantize_kernel<true, true>), grid, block, 0, s, x, rows, cols, ld, codes, scales);
        else hipLaunchKernelGGL((mx_quantize_kernel<true, false>), grid, block, 0, s, x, rows, cols, ld, codes, scales);
    } else {
        if (flat) hipLaunchKernelGGL((mx_quantize_kernel<false, true>), grid, block, 0, s, x, rows, cols, ld, codes, scales);
        else hipLaunchKernelGGL((mx_quantize_kernel<false, false>), grid, block, 0, s, x, rows, cols, ld, codes, scales);
    }
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
    const int w = dtype == STMOE_BF16 ? kOut<true> : kOut<false>;
    const dim3 grid(unsigned(grid_of(rows * ((cols + w - 1) / w)))), block(kThreads);
    const bool flat = ld == cols && cols % mx::kBlock == 0 && aligned(codes, 4);
    hipStream_t s = as_stream(stream);
    if (dtype == STMOE_BF16) {
        if (flat) hipLaunchKernelGGL((mx_dequantize_kernel<true, true>), grid, block, 0, s, codes, scales, rows, cols, y, ld);
        else hipLaunchKernelGGL((mx_dequantize_kernel<true, false>), grid, block, 0, s, codes, scales, rows, cols, y, ld);
    } else {
        if (flat) hipLaunchKernelGGL((mx_dequantize_kernel<false, true>), grid, block, 0, s, codes, scales, rows, cols, y, ld);
        else hipLaunchKernelGGL((mx_dequantize_kernel<false, false>), grid, block, 0, s, codes, scales, rows, cols, y, ld);
    }
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
