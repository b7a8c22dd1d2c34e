// Low-rank adapters of many requests beside a shared projection, and their gradient.
//
// For token t with adapter a (rank r, A [r][Hin], B [r][Hout], scale s):
//   v = x A^T     y = base + s v B                                (forward)
//   u = s dy B^T  dx = base + u A    dA = u^T x    dB = s v^T dy   (gradient)
// Three products: over the columns of a token (shrink: v, u), over the rank (expand:
// y, dx), and over the tokens of an adapter (outer: dA, dB).  A and B are both held
// by ranks, [r][columns], so each product serves both.  v and u are fp32 throughout.
//
// The plan's tiles hold tokens of one adapter.  These kernels take fp32 rows and bf16
// ones of any length, stride and alignment (lora_bf16.hip takes bf16 ones in whole 16-byte
// chunks).  They run on the fp32 matrix instruction (16 x 16 x 4): bf16 values are exact
// in it, and a lane takes one value of each operand at a time, so any layout of rows and
// columns does.  Rows that allow it are loaded four values at once (VEC).  Small calls
// are bound by the latency of tile, order and rows, one load after the other (37 x 1000 x
// 61 fp32: 6.6 and 5.3 us); large ones by loads of a row a lane and of the adapter again
// for every 16 tokens: 4096 x 2048 x 2048 fp32, rank 64, 27 and 48 us for 100 MB.
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
// Values i to i + 3 of a row of C; 0 beyond it and where `in` is false.  VEC: C and i are
// multiples of 4, the row is aligned to four values.
template <bool BF, bool VEC>
__device__ __forceinline__ void at4(const void* p, int64_t row, int i, int C, bool in, float (&v)[4]) {
    if constexpr (VEC) {
        in = in && i < C;
        const int64_t k = in ? row + i : 0;        // row 0 of the matrix is there for all
        if constexpr (BF) {
            const uint2 q = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(p) + k);
            v[0] = in ? bf16_lo(q.x) : 0.f;
            v[1] = in ? bf16_hi(q.x) : 0.f;
            v[2] = in ? bf16_lo(q.y) : 0.f;
            v[3] = in ? bf16_hi(q.y) : 0.f;
        } else {
            const f32x4 q = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(p) + k);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = in ? q[j] : 0.f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = in && i + j < C ? at<BF>(p, row + i + j) : 0.f;
    }
}
template <bool BF>
__device__ __forceinline__ void put(void* p, int64_t i, float v) {
    if (BF) reinterpret_cast<__bf16*>(p)[i] = __bf16(v);
    else reinterpret_cast<float*>(p)[i] = v;
}

// One tile of 16 tokens a workgroup and, with several parts, some of the columns; its
// waves every fourth 16 of them.
template <bool BF, int RT, bool VEC>
__global__ __launch_bounds__(kThreads) void lora_shrink_kernel(ShrinkArgs a) {
    __shared__ float part[kWaves][RT * 16][17];
    Tile tile;
    if (!tile_of(a.g, blockIdx.x, tile)) return;
    if (tile.adapter < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int rank = rank_of(a.g, tile.adapter);
    const void* m = a.m[tile.adapter];
    // tokens beyond the last one: the first, whose sums are not stored again
    const int64_t t = a.g.plan.order[tile.first + (c < tile.count ? c : 0)];
    f32x4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (rank > 0)
#pragma unroll(RT <= 2 ? 4 : 1)
        for (int h0 = 16 * (wave + kWaves * int(blockIdx.y)); h0 < a.C; h0 += 16 * kWaves * int(gridDim.y)) {
            float xv[4], mv[RT][4];
            at4<BF, VEC>(a.x, t * a.ld, h0 + 4 * q, a.C, true, xv);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int r = 16 * i + c;          // ranks beyond the last one: the first's, not stored
                at4<BF, VEC>(m, int64_t(r < rank ? r : 0) * a.C, h0 + 4 * q, a.C, true, mv[i]);
            }
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i] = mfma(mv[i][j], xv[j], acc[i]);
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
        a.v[(int64_t(blockIdx.y) * a.g.T + a.g.plan.order[tile.first + k]) * a.g.R + r] = r < rank ? s * sum : 0.f;
    }
}

// One tile of 16 tokens and 256 columns a workgroup, 64 columns a wave: the lane (c, q)
// feeds columns 4 c .. + 3 of rank q (of every four) as the column operands and gets them
// of tokens 4 q .. + 3.  VEC: of the adapter's rows and of base and y.
template <bool BF, bool YBF, bool VEC>
__global__ __launch_bounds__(kThreads) void lora_expand_kernel(ExpandArgs a) {
    Tile tile;
    if (!tile_of(a.g, blockIdx.x, tile)) return;
    if (a.v_out && a.parts > 1 && tile.adapter >= 0)
        sum_parts(a, a.g.plan.order + tile.first, tile.count, blockIdx.y, gridDim.y);
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
#pragma unroll 4
        for (int r0 = 0; r0 < rank; r0 += 4) {
            const int r = r0 + q;
            float vv = 0.f, mv[4];
            if (in && r < rank)
                for (int p = 0; p < a.parts; ++p) vv += a.v[(int64_t(p) * a.g.T + t) * a.g.R + r];
            at4<BF, VEC>(m, int64_t(r) * a.C, o0 + 4 * c, a.C, r < rank, mv);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = mfma(vv, mv[j], acc[j]);
        }
    }
    const int o = o0 + 4 * c;
    if (o >= a.C) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (4 * q + i >= tile.count) continue;
        const int64_t t = a.g.plan.order[tile.first + 4 * q + i];
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.base) at4<YBF, VEC>(a.base, t * a.ld_base, o, a.C, true, y);
        if (tile.adapter >= 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] += s * acc[j][i];
        if constexpr (VEC) {
            if constexpr (YBF) {
                union {
                    __bf16 h[4];
                    uint2 q;
                } u;
#pragma unroll
                for (int j = 0; j < 4; ++j) u.h[j] = __bf16(y[j]);
                *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.y) + t * a.ld + o) = u.q;
            } else {
                *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.y) + t * a.ld + o) = f32x4{y[0], y[1], y[2], y[3]};
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (o + j < a.C) put<YBF>(a.y, t * a.ld + o + j, y[j]);
        }
    }
}

// A tile of tokens and 64 columns a workgroup, its waves every fourth four of the tokens.
template <bool BF, int RT, bool VEC>
__global__ __launch_bounds__(kThreads) void lora_outer_kernel(OuterArgs ox, OuterArgs oy) {
    __shared__ float part[kWaves][16][65];
    const OuterArgs a = one_of(blockIdx.z, ox, oy);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int h0 = blockIdx.x * 64;
    Tile tile;
    if (!tile_of(a.g, blockIdx.y, tile) || tile.adapter < 0 || h0 >= a.C) return;
    const int rank = rank_of(a.g, tile.adapter), tiles = a.g.plan.base[tile.adapter + 1] - a.g.plan.base[tile.adapter];
    f32x4 acc[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll(RT <= 2 ? 4 : 1)
    for (int p0 = 4 * wave; p0 < tile.count; p0 += 4 * kWaves) {
        const bool in = p0 + q < tile.count;
        const int64_t t = a.g.plan.order[tile.first + (in ? p0 + q : 0)];
        float xv[4], uv[RT];
        at4<BF, VEC>(a.x, t * a.ld, h0 + 4 * c, a.C, in, xv);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = 16 * i + c;
            uv[i] = in && r < rank ? a.u[t * a.g.R + r] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma(xv[j], uv[i], acc[i][j]);
    }
    const float s = a.scaled && a.g.scales ? a.g.scales[tile.adapter] : 1.f;
    float* d = tiles == 1 ? a.d[tile.adapter]
                          : a.part + int64_t(outer_slot(tile.first, a.g.plan.size, tile.piece == tiles - 1)) * a.g.R * a.C;
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

// The gradients of adapters with several tiles, their sums in order, and of those
// without a token: zeros.  W values at once: C is a multiple of W.
template <int W>
__global__ __launch_bounds__(kThreads) void lora_join_kernel(OuterArgs ox, OuterArgs oy) {
    typedef float vec __attribute__((ext_vector_type(W)));
    const OuterArgs a = one_of(blockIdx.z, ox, oy);
    const int ad = blockIdx.x, size = a.g.plan.size;
    // side by side
    const int tiles = a.g.plan.base[ad + 1] - a.g.plan.base[ad], first = a.g.plan.seg[ad];
    const int64_t all = int64_t(rank_of(a.g, ad)) * a.C, part = int64_t(a.g.R) * a.C;
    float* d = a.d[ad];
    if (!planned(a.g) || tiles == 1) return;
    for (int64_t i = W * (int64_t(blockIdx.y) * kThreads + threadIdx.x); i < all; i += W * int64_t(gridDim.y) * kThreads) {
        vec sum = 0.f;
        for (int k0 = 0; k0 < tiles; k0 += 8) {    // eight loads at once
            vec v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = k0 + j;
                v[j] = 0.f;
                if (k < tiles)
                    v[j] = *reinterpret_cast<const vec*>(a.part + outer_slot(first + k * size, size, k == tiles - 1) * part + i);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[j];
        }
        *reinterpret_cast<vec*>(d + i) = sum;
    }
}

// Tokens per tile of the sums over tokens: 256, and for ranks above 16, whose sums (R x C
// fp32 a tile) would be as many bytes as the rows, 1024 from as many tokens on as give
// the CUs a workgroup each (4096 x 4096 each way, one adapter of rank 64: the gradient 88
// us with 256, 108 with 1024).
int outer_limit(int Hin, int Hout) { return 131072 / (((Hin > Hout ? Hin : Hout) + 511) / 512); }
int outer_table(int T, int Hin, int Hout, int R) { return R <= 16 || T < outer_limit(Hin, Hout) ? 2 : 3; }
// Never falls as T grows.
size_t outer_bytes(int T, int Hin, int Hout, int R) {
    const int most = outer_limit(Hin, Hout);
    size_t slots = outer_slots(R <= 16 || T < most ? T : most, tile_tokens(2));
    if (outer_table(T, Hin, Hout, R) == 3 && outer_slots(T, tile_tokens(3)) > slots) slots = outer_slots(T, tile_tokens(3));
    return slots * R * (size_t(Hin) + Hout) * sizeof(float);
}

// Calls f(16-row tiles of the rank).
template <class F>
void with_rank(int R, F f) {
    if (R <= 16) f(std::integral_constant<int, 1>());
    else if (R <= 32) f(std::integral_constant<int, 2>());
    else if (R <= 64) f(std::integral_constant<int, 4>());
    else f(std::integral_constant<int, 8>());
}

// Rows of C values that are loaded four at once.
bool fours(const void* p, int64_t ld, int C, int esz) {
    return C % 4 == 0 && ld % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (4 * esz) == 0;
}

// Calls f(bf16, VEC).
template <class F>
void with_rows(bool bf, bool vec, F f) {
    if (bf && vec) f(std::true_type(), std::true_type());
    else if (bf) f(std::true_type(), std::false_type());
    else if (vec) f(std::false_type(), std::true_type());
    else f(std::false_type(), std::false_type());
}

int shrink(const ShrinkArgs& a, int tiles, bool bf, hipStream_t s) {
    const dim3 grid(unsigned(tiles), unsigned(a.parts));
    with_rows(bf, fours(a.x, a.ld, a.C, bf ? 2 : 4), [&](auto b, auto vec) {
        with_rank(a.g.R, [&](auto rt) {
            hipLaunchKernelGGL((lora_shrink_kernel<b(), rt(), vec()>), grid, dim3(kThreads), 0, s, a);
        });
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int expand(const ExpandArgs& a, int tiles, bool bf, bool ybf, hipStream_t s) {
    const dim3 grid(unsigned(tiles), unsigned((a.C + 64 * kWaves - 1) / (64 * kWaves)));
    const int ysz = ybf ? 2 : 4;
    const bool vec4 = fours(a.y, a.ld, a.C, ysz) && (!a.base || fours(a.base, a.ld_base, a.C, ysz));
    with_rows(bf, vec4, [&](auto b, auto vec) {
        if (ybf) hipLaunchKernelGGL((lora_expand_kernel<b(), true, vec()>), grid, dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL((lora_expand_kernel<b(), false, vec()>), grid, dim3(kThreads), 0, s, a);
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int outer(const OuterArgs (&a)[2], int table, bool bf, hipStream_t s) {
    const int C = a[0].C > a[1].C ? a[0].C : a[1].C;
    const dim3 grid(unsigned((C + 63) / 64), unsigned(plan_layout(a[0].g.T, a[0].g.n).max_tiles[table]), 2);
    const int esz = bf ? 2 : 4;
    with_rows(bf, fours(a[0].x, a[0].ld, a[0].C, esz) && fours(a[1].x, a[1].ld, a[1].C, esz), [&](auto b, auto vec) {
        with_rank(a[0].g.R, [&](auto rt) {
            hipLaunchKernelGGL((lora_outer_kernel<b(), rt(), vec()>), grid, dim3(kThreads), 0, s, a[0], a[1]);
        });
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int join(const OuterArgs (&a)[2], hipStream_t s) {
    const int C = a[0].C > a[1].C ? a[0].C : a[1].C, n = a[0].g.n;
    const bool vec = a[0].C % 4 == 0 && a[1].C % 4 == 0;
    const int64_t chunks = (int64_t(a[0].g.R) * C / (vec ? 4 : 1) + kThreads - 1) / kThreads, most = n < 64 ? 512 / n : 8;
    const dim3 grid(unsigned(n), unsigned(chunks < most ? chunks : most), 2);
    if (vec) hipLaunchKernelGGL(lora_join_kernel<4>, grid, dim3(kThreads), 0, s, a[0], a[1]);
    else hipLaunchKernelGGL(lora_join_kernel<1>, grid, dim3(kThreads), 0, s, a[0], a[1]);
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
    if (sh.parts == 1) {
        // one part: where the caller wants it
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
                        const void* plan, size_t plan_bytes, const void* const* a_ptrs, const void* const* b_ptrs,
                        const int32_t* ranks, const float* scales, const void* base, int64_t ld_base, void* y,
                        int64_t ldy, float* v, void* ws, size_t ws_bytes, void* stream) {
    clear_error();
    if (const char* bad = bad_call(T, Hin, Hout, n_adapters, R, dtype, ydtype)) STMOE_CHECK(false, bad);
    if (T == 0) return STMOE_OK;
    STMOE_CHECK(x && plan && a_ptrs && b_ptrs && y && ws, "null pointer");
    if (const char* bad = bad_rows(x, ldx, Hin, dtype)) STMOE_CHECK(false, bad);
    if (const char* bad = bad_rows(y, ldy, Hout, ydtype)) STMOE_CHECK(false, bad);
    if (base)
        if (const char* bad = bad_rows(base, ld_base, Hout, ydtype)) STMOE_CHECK(false, bad);
    STMOE_CHECK(base != y || ld_base == ldy, "base in the place of y must have its row stride");
    STMOE_CHECK(plan_bytes >= moe_lora_plan_bytes(T, n_adapters), "plan too small");
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
                                 int Hout, int n_adapters, int R, int dtype, const void* plan, size_t plan_bytes,
                                 const void* const* a_ptrs, const void* const* b_ptrs, const int32_t* ranks,
                                 const float* scales, float* const* da_ptrs, float* const* db_ptrs,
                                 const void* base, int64_t ld_base, void* dx, int64_t ld_dx, void* ws, size_t ws_bytes,
                                 void* stream) {
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
    STMOE_CHECK(!dx || (dx != x && dx != dy), "dx must not be x or dy");
    STMOE_CHECK(!dx || base != dx || ld_base == ld_dx, "base in the place of dx must have its row stride");
    STMOE_CHECK(plan_bytes >= moe_lora_plan_bytes(T, n_adapters), "plan too small");
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
    const int table = outer_table(T, Hin, Hout, R);
    float* sums = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + rows_bytes(T, R) + rows_bytes(part_rows(T), R));
    const Args gt = with_table(g, table);
    const OuterArgs o[2] = {{gt, x, ldx, Hin, u, 0, da_ptrs, sums},
                            {gt, dy, ld_dy, Hout, v, 1, db_ptrs, sums + outer_slots(T, tile_tokens(table)) * R * Hin}};
    const bool fast = bf && chunks16(x, ldx, Hin, 2) && chunks16(dy, ld_dy, Hout, 2);
    if (int rc = fast ? outer_bf16(o, table, s) : outer(o, table, bf, s)) return rc;
    return join(o, s);
}
