// Low-rank adapters of many requests beside a shared projection, and their gradient.
//
// For token t with adapter a (rank r, A [r][Hin], B [r][Hout], scale s):
//   v = x A^T     y = base + s v B                                (forward)
//   u = s dy B^T  dx = base + u A    dA = u^T x    dB = s v^T dy   (gradient)
// Three products: over the columns of a token (shrink: v, u), over the rank (expand:
// y, dx), and over the tokens of an adapter (outer: dA, dB).  A and B are both held
// by ranks, [r][columns], so each product serves both.  v and u are fp32 throughout.
//
// The plan's tiles hold tokens of one adapter.  These kernels run on the fp32 matrix
// instruction (16 x 16 x 4): bf16 values are exact in it, and a lane takes one value
// of each operand at a time, so any layout of rows and columns does.
#include <type_traits>

#include "lora.h"

namespace stmoe {
namespace lora {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTile = 16;
constexpr int kMaxRankTiles = kMaxRank / 16;

__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <bool BF>
__device__ __forceinline__ float at(const void* p, int64_t i) {
    return BF ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(p)[i]) << 16)
              : reinterpret_cast<const float*>(p)[i];
}
template <bool BF>
__device__ __forceinline__ void put(void* p, int64_t i, float v) {
    if (BF) reinterpret_cast<__bf16*>(p)[i] = __bf16(v);
    else reinterpret_cast<float*>(p)[i] = v;
}

// One tile of 16 tokens a workgroup, its waves a part of the columns each.
template <bool BF, int RT>
__global__ __launch_bounds__(kThreads) void lora_shrink_kernel(ShrinkArgs a) {
    __shared__ float part[kWaves][RT * 16][17];
    Tile tile;
    if (!tile_of(a.g, blockIdx.x, tile)) return;
    if (tile.adapter < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int rank = rank_of(a.g, tile.adapter);
    const void* m = a.m[tile.adapter];
    const bool in = c < tile.count;
    const int t = a.g.plan.order[tile.first + (in ? c : 0)];
    f32x4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int h0 = 16 * wave; h0 < a.C; h0 += 16 * kWaves) {
        float xv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int h = h0 + 4 * q + j;
            xv[j] = in && h < a.C ? at<BF>(a.x, t * a.ld + h) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = 16 * i + c;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int h = h0 + 4 * q + j;
                acc[i] = mfma(r < rank && h < a.C ? at<BF>(m, int64_t(r) * a.C + h) : 0.f, xv[j], acc[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[wave][16 * i + 4 * q + j][c] = acc[i][j];
    __syncthreads();
    const float s = a.scaled && a.g.scales ? a.g.scales[tile.adapter] : 1.f;
    for (int i = threadIdx.x; i < tile.count * a.g.R; i += kThreads) {
        const int k = i / a.g.R, r = i - k * a.g.R;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += part[w][r][k];
        a.v[int64_t(a.g.plan.order[tile.first + k]) * a.g.R + r] = r < rank ? s * sum : 0.f;
    }
}

// One tile of 16 tokens and 256 columns a workgroup, 64 columns a wave: the lane
// (c, q) feeds columns 4 c + j of row 4 q + i and gets columns 16 q .. + 15 of token c.
template <bool BF, bool YBF>
__global__ __launch_bounds__(kThreads) void lora_expand_kernel(ExpandArgs a) {
    Tile tile;
    if (!tile_of(a.g, blockIdx.x, tile)) return;
    if (a.v_out && a.parts > 1 && blockIdx.y == 0 && tile.adapter >= 0)
        for (int i = threadIdx.x; i < tile.count * a.g.R; i += kThreads) {
            const int64_t at = int64_t(a.g.plan.order[tile.first + i / a.g.R]) * a.g.R + i % a.g.R;
            float sum = 0.f;
            for (int p = 0; p < a.parts; ++p) sum += a.v[int64_t(p) * a.g.T * a.g.R + at];
            a.v_out[at] = sum;
        }
    if (tile.adapter < 0 && a.base == a.y) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int o0 = (blockIdx.y * kWaves + wave) * 64;
    const bool in = c < tile.count;
    const int t = a.g.plan.order[tile.first + (in ? c : 0)];
    f32x4 acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float s = 1.f;
    if (tile.adapter >= 0) {
        const int rank = rank_of(a.g, tile.adapter);
        const void* m = a.m[tile.adapter];
        if (a.scaled && a.g.scales) s = a.g.scales[tile.adapter];
        for (int r0 = 0; r0 < rank; r0 += 4) {
            const int r = r0 + q;
            float vv = 0.f;
            if (in && r < rank)
                for (int p = 0; p < a.parts; ++p) vv += a.v[(int64_t(p) * a.g.T + t) * a.g.R + r];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int o = o0 + 4 * c + j;
                acc[j] = mfma(r < rank && o < a.C ? at<BF>(m, int64_t(r) * a.C + o) : 0.f, vv, acc[j]);
            }
        }
    }
    if (!in) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int o = o0 + 16 * q + 4 * i + j;
            if (o < a.C) {
                const float b = a.base ? at<YBF>(a.base, t * a.ld_base + o) : 0.f;
                put<YBF>(a.y, t * a.ld + o, tile.adapter >= 0 ? b + s * acc[j][i] : b);
            }
        }
}

// One adapter and 64 columns a workgroup, its waves a part of the tokens each.
template <bool BF, int RT>
__global__ __launch_bounds__(kThreads) void lora_outer_kernel(OuterArgs a) {
    __shared__ float part[kWaves][16][65];
    if (!planned(a.g)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int ad = blockIdx.x, h0 = blockIdx.y * 64;
    const int rank = rank_of(a.g, ad), t0 = a.g.plan.seg[ad], t1 = a.g.plan.seg[ad + 1];
    f32x4 acc[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int p0 = t0 + 4 * wave; p0 < t1; p0 += 4 * kWaves) {
        const bool in = p0 + q < t1;
        const int64_t t = a.g.plan.order[in ? p0 + q : t0];
        float xv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int h = h0 + 4 * c + j;
            xv[j] = in && h < a.C ? at<BF>(a.x, t * a.ld + h) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = 16 * i + c;
            const float uv = in && r < rank ? a.u[t * a.g.R + r] : 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma(xv[j], uv, acc[i][j]);
        }
    }
    const float s = a.scaled && a.g.scales ? a.g.scales[ad] : 1.f;
    float* d = a.d[ad];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) part[wave][c][16 * q + 4 * k + j] = acc[i][j][k];
        __syncthreads();
        for (int k = threadIdx.x; k < 16 * 64; k += kThreads) {
            const int r = 16 * i + k / 64, h = h0 + k % 64;
            if (r >= rank || h >= a.C) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum += part[w][k / 64][k % 64];
            d[int64_t(r) * a.C + h] = s * sum;
        }
    }
}

// Tiles of 64 tokens where adapters have that many on average.
bool large_tiles(int T, int n) { return T >= 64 * n && T > 64; }

// Rows of all parts of T tokens at most; never falls as T grows.
int part_rows(int T) { return T < 4096 ? 8 * T : T < 32768 ? 32768 : T; }

// Parts of a token's columns, a workgroup each, where there are few of them.  The launch
// over the rank adds them up, which costs it more with every part.  us of the two
// launches with 1, 2, 4 and 8 parts (4096 columns each way): 64 tokens of 32 adapters,
// rank 64: 22.6, 17.0, 14.5, 15.1; 4096 tokens, rank 16: 35.6, 32.6, 35.5; 8192 tokens,
// rank 64: 65.3, 70.8, 81.3.
int column_parts(int T, int n, int C) {
    const int groups = large_tiles(T, n) ? 2 * (T / 64 + n) : T / 16 + (T < n ? T : n);
    int p = 1;
    while (p < 8 && groups * p < 144 && C / (2 * p) >= 512 && 2 * p * T <= part_rows(T)) p *= 2;
    return p;
}

// Tokens per tile of the sums over tokens: 256, and 1024 for ranks above 16, whose sums
// (R x C fp32 a tile) would be as many bytes as the rows.
int outer_table(int, int, int R) { return R <= 16 ? 2 : 3; }
size_t outer_bytes(int T, int Hin, int Hout, int R) {
    return outer_slots(T, tile_tokens(outer_table(T, 1, R))) * R * (size_t(Hin) + Hout) * sizeof(float);
}

// Calls f(16-row tiles of the rank).
template <class F>
void with_rank(int R, F f) {
    if (R <= 16) f(std::integral_constant<int, 1>());
    else if (R <= 32) f(std::integral_constant<int, 2>());
    else if (R <= 64) f(std::integral_constant<int, 4>());
    else f(std::integral_constant<int, 8>());
}

int shrink(const ShrinkArgs& a, int tiles, bool bf, hipStream_t s) {
    with_rank(a.g.R, [&](auto rt) {
        if (bf) hipLaunchKernelGGL((lora_shrink_kernel<true, rt()>), dim3(unsigned(tiles)), dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL((lora_shrink_kernel<false, rt()>), dim3(unsigned(tiles)), dim3(kThreads), 0, s, a);
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int expand(const ExpandArgs& a, int tiles, bool bf, bool ybf, hipStream_t s) {
    const dim3 grid(unsigned(tiles), unsigned((a.C + 64 * kWaves - 1) / (64 * kWaves)));
    if (bf && ybf) hipLaunchKernelGGL((lora_expand_kernel<true, true>), grid, dim3(kThreads), 0, s, a);
    else if (bf) hipLaunchKernelGGL((lora_expand_kernel<true, false>), grid, dim3(kThreads), 0, s, a);
    else if (ybf) hipLaunchKernelGGL((lora_expand_kernel<false, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((lora_expand_kernel<false, false>), grid, dim3(kThreads), 0, s, a);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int outer(const OuterArgs& a, bool bf, hipStream_t s) {
    const dim3 grid(unsigned(a.g.n), unsigned((a.C + 63) / 64));
    with_rank(a.g.R, [&](auto rt) {
        if (bf) hipLaunchKernelGGL((lora_outer_kernel<true, rt()>), grid, dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL((lora_outer_kernel<false, rt()>), grid, dim3(kThreads), 0, s, a);
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

// The two products over a token's columns and over the rank, one after the other,
// by the kernels that their rows allow.
int shrink_expand(ShrinkArgs sh, ExpandArgs ex, int dtype, int ydtype, hipStream_t s) {
    const PlanLayout y = plan_layout(sh.g.T, sh.g.n);
    const bool bf = dtype == STMOE_BF16, ybf = ydtype == STMOE_BF16;
    const int esz = bf ? 2 : 4, ysz = ybf ? 2 : 4;
    const bool fast_shrink = bf && chunks16(sh.x, sh.ld, sh.C, esz);
    const bool fast_expand = bf && ex.C % 8 == 0 && chunks16(ex.y, ex.ld, ex.C, ysz) &&
                             (!ex.base || chunks16(ex.base, ex.ld_base, ex.C, ysz));
    const int table = large_tiles(sh.g.T, sh.g.n) ? 1 : 0;
    if (!fast_shrink || sh.parts == 1) {
        // one part: where the caller wants it
        sh.parts = ex.parts = 1;
        if (ex.v_out) sh.v = ex.v_out;
        ex.v = sh.v;
    }
    if (int rc = fast_shrink ? shrink_bf16(sh, table, s) : shrink(sh, y.max_tiles[0], bf, s)) return rc;
    if (!ex.y) return STMOE_OK;
    return fast_expand ? expand_bf16(ex, table, ybf, s) : expand(ex, y.max_tiles[0], bf, ybf, s);
}

size_t rows_bytes(int T, int R) { return (size_t(T) * R * sizeof(float) + 255) / 256 * 256; }

bool bad_shape(int T, int Hin, int Hout, int n, int R, int dtype) {
    return T < 0 || T > kMaxTokens || Hin < 1 || Hin > kMaxCols || Hout < 1 || Hout > kMaxCols || n < 1 ||
           n > kMaxAdapters || R < 1 || R > kMaxRank || (dtype != STMOE_BF16 && dtype != STMOE_F32);
}

const char* bad_call(int T, int Hin, int Hout, int n, int R, int dtype, int ydtype) {
    if (T < 0 || T > kMaxTokens) return "T must be in [0, 65536]";
    if (Hin < 1 || Hin > kMaxCols || Hout < 1 || Hout > kMaxCols) return "Hin and Hout must be in [1, 65536]";
    if (n < 1 || n > kMaxAdapters) return "n_adapters must be in [1, 4096]";
    if (R < 1 || R > kMaxRank) return "R must be in [1, 128]";
    if (dtype != STMOE_BF16 && dtype != STMOE_F32) return "dtype must be STMOE_BF16 or STMOE_F32";
    if (ydtype != STMOE_BF16 && ydtype != STMOE_F32) return "ydtype must be STMOE_BF16 or STMOE_F32";
    return nullptr;
}

const char* bad_rows(const void* p, int64_t ld, int cols, int dtype) {
    if (ld < cols || ld > (int64_t(1) << 31)) return "a row stride must be in [columns, 2^31]";
    if (reinterpret_cast<uintptr_t>(p) % (dtype == STMOE_BF16 ? 2 : 4)) return "rows must be aligned to their elements";
    return nullptr;
}

}  // namespace
}  // namespace lora
}  // namespace stmoe

using namespace stmoe;
using namespace stmoe::lora;

extern "C" size_t moe_lora_workspace_bytes(int T, int Hin, int Hout, int n_adapters, int R, int dtype) {
    return bad_shape(T, Hin, Hout, n_adapters, R, dtype) ? 0 : rows_bytes(part_rows(T), R) + 256;
}

extern "C" int moe_lora(const void* x, int64_t ldx, int T, int Hin, int Hout, int n_adapters, int R, int dtype, int ydtype,
                        const void* plan, const void* const* a_ptrs, const void* const* b_ptrs, const int32_t* ranks,
                        const float* scales, const void* base, int64_t ld_base, void* y, int64_t ldy, float* v, void* ws,
                        size_t ws_bytes, void* stream) {
    clear_error();
    if (const char* bad = bad_call(T, Hin, Hout, n_adapters, R, dtype, ydtype)) STMOE_CHECK(false, bad);
    if (T == 0) return STMOE_OK;
    STMOE_CHECK(x && plan && a_ptrs && b_ptrs && y && ws, "null pointer");
    if (const char* bad = bad_rows(x, ldx, Hin, dtype)) STMOE_CHECK(false, bad);
    if (const char* bad = bad_rows(y, ldy, Hout, ydtype)) STMOE_CHECK(false, bad);
    if (base)
        if (const char* bad = bad_rows(base, ld_base, Hout, ydtype)) STMOE_CHECK(false, bad);
    STMOE_CHECK(base != y || ld_base == ldy, "base in the place of y must have its row stride");
    STMOE_CHECK(ws_bytes >= moe_lora_workspace_bytes(T, Hin, Hout, n_adapters, R, dtype), "workspace too small");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(ws) % 256 == 0 && reinterpret_cast<uintptr_t>(plan) % 256 == 0,
                "ws and plan must be 256-byte aligned");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(v) % 16 == 0, "v must be 16-byte aligned");
    const Args g{plan_of(plan, T, n_adapters, 0), plan, T, n_adapters, R, ranks, scales};
    const int parts = column_parts(T, n_adapters, Hin);
    float* mine = reinterpret_cast<float*>(ws);
    return shrink_expand(ShrinkArgs{g, x, ldx, Hin, a_ptrs, 0, mine, parts},
                         ExpandArgs{g, mine, parts, v, b_ptrs, Hout, 1, base, ld_base, y, ldy}, dtype, ydtype,
                         as_stream(stream));
}

extern "C" size_t moe_lora_backward_workspace_bytes(int T, int Hin, int Hout, int n_adapters, int R, int dtype) {
    return bad_shape(T, Hin, Hout, n_adapters, R, dtype) ? 0
               : rows_bytes(T, R) + rows_bytes(part_rows(T), R) + outer_bytes(T, Hin, Hout, R) + 256;
}

extern "C" int moe_lora_backward(const void* x, int64_t ldx, const void* dy, int64_t ld_dy, const float* v, int T, int Hin,
                                 int Hout, int n_adapters, int R, int dtype, const void* plan, const void* const* a_ptrs,
                                 const void* const* b_ptrs, const int32_t* ranks, const float* scales, float* const* da_ptrs,
                                 float* const* db_ptrs, const void* base, int64_t ld_base, void* dx, int64_t ld_dx, void* ws,
                                 size_t ws_bytes, void* stream) {
    clear_error();
    if (const char* bad = bad_call(T, Hin, Hout, n_adapters, R, dtype, dtype)) STMOE_CHECK(false, bad);
    STMOE_CHECK(T >= 1, "T must be in [1, 65536]");
    STMOE_CHECK(x && dy && v && plan && a_ptrs && b_ptrs && da_ptrs && db_ptrs && ws, "null pointer");
    if (const char* bad = bad_rows(x, ldx, Hin, dtype)) STMOE_CHECK(false, bad);
    if (const char* bad = bad_rows(dy, ld_dy, Hout, dtype)) STMOE_CHECK(false, bad);
    if (dx)
        if (const char* bad = bad_rows(dx, ld_dx, Hin, dtype)) STMOE_CHECK(false, bad);
    if (dx && base)
        if (const char* bad = bad_rows(base, ld_base, Hin, dtype)) STMOE_CHECK(false, bad);
    STMOE_CHECK(!dx || base != dx || ld_base == ld_dx, "base in the place of dx must have its row stride");
    STMOE_CHECK(ws_bytes >= moe_lora_backward_workspace_bytes(T, Hin, Hout, n_adapters, R, dtype), "workspace too small");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(ws) % 256 == 0 && reinterpret_cast<uintptr_t>(plan) % 256 == 0,
                "ws and plan must be 256-byte aligned");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(v) % 16 == 0, "v must be 16-byte aligned");
    const Args g{plan_of(plan, T, n_adapters, 0), plan, T, n_adapters, R, ranks, scales};
    float* u = reinterpret_cast<float*>(ws);
    hipStream_t s = as_stream(stream);
    const bool bf = dtype == STMOE_BF16;
    // where dx is wanted, its launch adds the parts of u up
    const int parts = dx ? column_parts(T, n_adapters, Hout) : 1;
    float* mine = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + rows_bytes(T, R));
    if (int rc = shrink_expand(ShrinkArgs{g, dy, ld_dy, Hout, b_ptrs, 1, mine, parts},
                               ExpandArgs{g, mine, parts, u, a_ptrs, Hin, 0, base, ld_base, dx, ld_dx}, dtype, dtype, s))
        return rc;
    const int table = outer_table(T, n_adapters, R);
    float* sums = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + rows_bytes(T, R) + rows_bytes(part_rows(T), R));
    const OuterArgs o[2] = {{g, x, ldx, Hin, u, 0, da_ptrs, sums},
                            {g, dy, ld_dy, Hout, v, 1, db_ptrs, sums + outer_slots(T, tile_tokens(table)) * R * Hin}};
    if (bf && chunks16(x, ldx, Hin, 2) && chunks16(dy, ld_dy, Hout, 2)) return outer_bf16(o, table, s);
    if (int rc = outer(o[1], bf, s)) return rc;
    return outer(o[0], bf, s);
}
