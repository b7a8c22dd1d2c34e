// Low-rank adapters over bf16 rows in whole 16-byte chunks: the products of lora.hip on
// the bf16 matrix instruction (16 x 16 x 32).
//
// One operand of every product is bf16 and exact; the fp32 one (v, u) is split into
// bf16 pieces, the value's rounding and the roundings of what is left: two hold 16 bits
// of it (2^-17 of itself off at most, where a bf16 result is rounded by 2^-9), three its
// 24.
#include <type_traits>

#include "lora.h"

namespace stmoe {
namespace lora {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ bf16x8 operand(u32x4 q) {
    union {
        u32x4 q;
        bf16x8 v;
    } u;
    u.q = q;
    return u.v;
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// N pieces of eight values.  What is left of a value that rounds to an infinity is
// nothing, not NaN.
template <int N>
__device__ __forceinline__ void split(const float (&x)[8], bf16x8 (&p)[N]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float left = x[i];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const __bf16 b = __bf16(left);
            p[k][i] = b;
            const float f = float(b);
            left = fabsf(f) < INFINITY ? left - f : 0.f;
        }
    }
}

// Columns of eight rows as operands: fragment j has column j of rows 0 to 7.
__device__ __forceinline__ bf16x8 column(const u32x4 (&rows)[8], int j) {
    u32x4 q;
#pragma unroll
    for (int d = 0; d < 4; ++d)
        q[d] = __builtin_amdgcn_perm(rows[2 * d + 1][j / 2], rows[2 * d][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return operand(q);
}

// Eight values of a row of R from r on, 0 beyond it; the sum of its parts.
__device__ __forceinline__ void load8(const float* row, int64_t part, int parts, int r, int R, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    for (int p = 0; p < parts; ++p, row += part) {
        if (R % 8 == 0) {
            if (r < R) {
                const f32x4 lo = *reinterpret_cast<const f32x4*>(row + r), hi = *reinterpret_cast<const f32x4*>(row + r + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] += lo[i];
                    v[4 + i] += hi[i];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r + i < R) v[i] += row[r + i];
        }
    }
}

// v = x A^T.  16 NT tokens a workgroup (a tile, or a part of one) and, with several
// parts, some of the columns; a wave takes every fourth 64 columns.  The lane (c, q)
// feeds columns 16 q .. + 15 of token c and of rank c: 32 bytes of a row, 128 a quarter
// wave.
template <int RT, int NT>
__global__ __launch_bounds__(kThreads) void lora_shrink_bf16_kernel(ShrinkArgs a, int table) {
    constexpr int TOK = 16 * NT, LD = 16 * RT + 4;
    __shared__ __attribute__((aligned(16))) float red[2][TOK][LD];
    if (!planned(a.g)) return;
    const int sub = tile_tokens(table) / TOK, ti = blockIdx.x / sub, k0 = (blockIdx.x % sub) * TOK;
    if (ti >= a.g.plan.head->tiles[table]) return;
    const Tile tile = a.g.plan.tiles[table][ti];
    if (tile.adapter < 0 || k0 >= tile.count) return;
    const int count = tile.count - k0 < TOK ? tile.count - k0 : TOK, first = tile.first + k0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int rank = rank_of(a.g, tile.adapter);
    const char* m = reinterpret_cast<const char*>(a.m[tile.adapter]);
    // tokens and ranks beyond the last ones take another's values: their sums are their own
    const char* xr[NT];
    const char* mr[RT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int k = 16 * i + c;
        xr[i] = reinterpret_cast<const char*>(a.x) + 2 * (a.g.plan.order[first + (k < count ? k : 0)] * a.ld);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = 16 * i + c;
        mr[i] = m + 2 * (int64_t(r < rank ? r : 0) * a.C);
    }
    f32x4 acc[NT][RT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const u32x4 zero = {0u, 0u, 0u, 0u};
    const int step = 64 * kWaves * int(gridDim.y);
    if (rank > 0)
#pragma unroll 2
        for (int h0 = 64 * (blockIdx.y * kWaves + wave); h0 < a.C; h0 += step) {
            u32x4 xv[NT][2], mv[RT][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int h = h0 + 16 * q + 8 * u;
                const bool in = h < a.C;       // C is a multiple of 8
#pragma unroll
                for (int i = 0; i < NT; ++i) xv[i][u] = in ? *reinterpret_cast<const u32x4*>(xr[i] + 2 * h) : zero;
#pragma unroll
                for (int i = 0; i < RT; ++i) mv[i][u] = in ? *reinterpret_cast<const u32x4*>(mr[i] + 2 * h) : zero;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < RT; ++j)
#pragma unroll
                    for (int i = 0; i < NT; ++i) acc[i][j] = mfma(operand(mv[j][u]), operand(xv[i][u]), acc[i][j]);
        }
    // the waves' sums, two and two
    auto at = [&](int b, int i, int j) { return reinterpret_cast<f32x4*>(&red[b][16 * i + c][16 * j + 4 * q]); };
    if (wave >= 2)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < RT; ++j) *at(wave - 2, i, j) = acc[i][j];
    __syncthreads();
    if (wave < 2)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < RT; ++j) *at(wave, i, j) += acc[i][j];
    __syncthreads();
    const float s = a.scaled && a.g.scales ? a.g.scales[tile.adapter] : 1.f;
    const int R = a.g.R;
    float* out = a.v + int64_t(blockIdx.y) * a.g.T * R;
    for (int i = threadIdx.x; i < count * R; i += kThreads) {
        const int k = i / R, r = i - k * R;
        out[int64_t(a.g.plan.order[first + k]) * R + r] = r < rank ? s * (red[0][k][r] + red[1][k][r]) : 0.f;
    }
}

// y = base + s v B.  A tile of tokens and 512 columns a workgroup, 128 a wave, whose
// lane (c, q) holds columns 8 c .. + 7 of ranks 8 q .. + 7 (of every 32) as the row
// operand, rows (columns of B) being 8 c + j for instruction j: it gets columns
// 32 q .. + 31 of token c.  With a rank of 16 at most the lanes q = 2, 3 hold the same
// ranks as q = 0, 1, against the second piece of v.
template <int KS, bool PACK, bool YBF>
__global__ __launch_bounds__(kThreads) void lora_expand_bf16_kernel(ExpandArgs a, int table) {
    constexpr int P = YBF ? 2 : 3, NM = PACK ? (P + 1) / 2 : KS * P;
    if (!planned(a.g) || int(blockIdx.x) >= a.g.plan.head->tiles[table]) return;
    const Tile tile = a.g.plan.tiles[table][blockIdx.x];
    const int R = a.g.R, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int64_t part = int64_t(a.g.T) * R;
    if (a.v_out && a.parts > 1 && blockIdx.y == 0 && tile.adapter >= 0)
        for (int i = threadIdx.x; i < tile.count * R; i += kThreads) {
            const int64_t at = int64_t(a.g.plan.order[tile.first + i / R]) * R + i % R;
            float sum = 0.f;
            for (int p = 0; p < a.parts; ++p) sum += a.v[p * part + at];
            a.v_out[at] = sum;
        }
    if (tile.adapter < 0 && a.base == a.y) return;
    const int o0 = (blockIdx.y * kWaves + wave) * 128;
    if (o0 >= a.C) return;
    const u32x4 zero = {0u, 0u, 0u, 0u};
    bf16x8 mf[KS][8];
    float s = 0.f;
    if (tile.adapter >= 0) {
        const int rank = rank_of(a.g, tile.adapter);
        const char* m = reinterpret_cast<const char*>(a.m[tile.adapter]);
        s = a.scaled && a.g.scales ? a.g.scales[tile.adapter] : 1.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            u32x4 rows[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 32 * k + 8 * (PACK ? q & 1 : q) + i, o = o0 + 8 * c;
                rows[i] = r < rank && o < a.C ? *reinterpret_cast<const u32x4*>(m + 2 * (int64_t(r) * a.C + o)) : zero;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) mf[k][j] = column(rows, j);
        }
    }
    for (int k0 = 0; k0 < tile.count; k0 += 16) {
        const bool in = k0 + c < tile.count;
        const int64_t t = a.g.plan.order[tile.first + (in ? k0 + c : 0)];
        // base: four chunks of eight columns
        constexpr int W = YBF ? 1 : 2;
        u32x4 b[4][W];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const int o = o0 + 32 * q + 8 * i;
                b[i][w] = a.base && in && o < a.C
                              ? reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.base) +
                                                               (YBF ? 2 : 4) * (t * a.ld_base + o))[w]
                              : zero;
            }
        f32x4 acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (tile.adapter >= 0) {
            bf16x8 vf[NM];
            float v[8];
            if constexpr (PACK) {
                load8(a.v + t * R, part, a.parts, 8 * (q & 1), R, v);
                bf16x8 p[P];
                split(v, p);
                vf[0] = q < 2 ? p[0] : p[1];
                if constexpr (P == 3) vf[1] = q < 2 ? p[2] : operand(zero);
            } else {
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    load8(a.v + t * R, part, a.parts, 32 * k + 8 * q, R, v);
                    bf16x8 p[P];
                    split(v, p);
#pragma unroll
                    for (int i = 0; i < P; ++i) vf[P * k + i] = p[i];
                }
            }
#pragma unroll
            for (int i = NM - 1; i >= 0; --i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = mfma(mf[PACK ? 0 : i / P][j], vf[i], acc[j]);
        }
        if (!in) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int o = o0 + 32 * q + 8 * i;
            if (o >= a.C) continue;
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = YBF ? (j % 2 ? bf16_hi(b[i][0][j / 2]) : bf16_lo(b[i][0][j / 2]))
                                    : __uint_as_float(b[i][W - 1 ? j / 4 : 0][j % 4]);
                y[j] = tile.adapter >= 0 ? f + s * acc[j][i] : f;
            }
            char* out = reinterpret_cast<char*>(a.y) + (YBF ? 2 : 4) * (t * a.ld + o);
            if constexpr (YBF) {
                union {
                    __bf16 h[8];
                    u32x4 q;
                } u;
#pragma unroll
                for (int j = 0; j < 8; ++j) u.h[j] = __bf16(y[j]);
                *reinterpret_cast<u32x4*>(out) = u.q;
            } else {
                reinterpret_cast<f32x4*>(out)[0] = f32x4{y[0], y[1], y[2], y[3]};
                reinterpret_cast<f32x4*>(out)[1] = f32x4{y[4], y[5], y[6], y[7]};
            }
        }
    }
}

// d = u^T x of a tile of tokens (a gradient, or its sum of an adapter with several
// tiles).  512 columns and up to 64 ranks a workgroup, 128 columns a wave, 32 tokens at
// a time: the lane (c, q) loads columns 8 c .. + 7 of tokens 8 q .. + 7, the row operand
// of instruction j being columns 8 c + j; u's three pieces are made once for the
// workgroup, in LDS.
template <int RT>
__global__ __launch_bounds__(kThreads) void lora_outer_bf16_kernel(OuterArgs ox, OuterArgs oy, int table) {
    constexpr int P = 3;
    __shared__ u32x4 uf[2][RT][P][64];
    const OuterArgs& a = blockIdx.z & 1 ? oy : ox;
    const int rt0 = (blockIdx.z >> 1) * 64;
    if (!planned(a.g) || int(blockIdx.x) >= a.g.plan.head->tiles[table]) return;
    const Tile tile = a.g.plan.tiles[table][blockIdx.x];
    if (tile.adapter < 0 || int(blockIdx.y) * 128 * kWaves >= a.C) return;
    const int R = a.g.R, rank = rank_of(a.g, tile.adapter);
    if (rt0 >= rank) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int h0 = (blockIdx.y * kWaves + wave) * 128, h = h0 + 8 * c;
    const bool cols = h < a.C;
    const char* x = reinterpret_cast<const char*>(a.x) + 2 * h;
    const int32_t* order = a.g.plan.order + tile.first;
    const u32x4 zero = {0u, 0u, 0u, 0u};
    f32x4 acc[RT][8];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // thread: rank ur, tokens 8 uq .. + 7 of u
    auto load_u = [&](int k0, float (&u)[8], int i) {
        const int at = threadIdx.x + i * kThreads, ur = rt0 + (at / 64) * 16 + (at & 15), uq = (at >> 4) & 3;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int p = k0 + 8 * uq + k;
            u[k] = p < tile.count && ur < rank && at < 64 * RT ? a.u[int64_t(order[p]) * R + ur] : 0.f;
        }
    };
    auto load_x = [&](int k0, u32x4 (&rows)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int p = k0 + 8 * q + k;
            rows[k] = cols && p < tile.count ? *reinterpret_cast<const u32x4*>(x + 2 * (int64_t(order[p]) * a.ld)) : zero;
        }
    };
    constexpr int UN = (64 * RT + kThreads - 1) / kThreads;
    float u[UN][8];
    u32x4 rows[8];
#pragma unroll
    for (int i = 0; i < UN; ++i) load_u(0, u[i], i);
    load_x(0, rows);
    int buf = 0;
    for (int k0 = 0; k0 < tile.count; k0 += 32, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at >= 64 * RT) continue;
            bf16x8 p[P];
            split(u[i], p);
#pragma unroll
            for (int j = 0; j < P; ++j) *reinterpret_cast<bf16x8*>(&uf[buf][at / 64][j][at & 63]) = p[j];
        }
        bf16x8 xf[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) xf[j] = column(rows, j);
        // the next tokens are on their way while these are used
        if (k0 + 32 < tile.count) {
#pragma unroll
            for (int i = 0; i < UN; ++i) load_u(k0 + 32, u[i], i);
            load_x(k0 + 32, rows);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int p = P - 1; p >= 0; --p) {
                const bf16x8 b = operand(uf[buf][i][p][lane]);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] = mfma(xf[j], b, acc[i][j]);
            }
    }
    const int tiles = a.g.plan.base[table][tile.adapter + 1] - a.g.plan.base[table][tile.adapter];
    const float s = a.scaled && a.g.scales ? a.g.scales[tile.adapter] : 1.f;
    float* d = tiles == 1 ? a.d[tile.adapter]
                          : a.part + int64_t(outer_slot(tile.first, tile_tokens(table), tile.piece == tiles - 1)) * R * a.C;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = rt0 + 16 * i + c;
        if (r >= rank) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int o = h0 + 32 * q + 8 * k;
            if (o >= a.C) continue;
            f32x4* out = reinterpret_cast<f32x4*>(d + int64_t(r) * a.C + o);
            out[0] = f32x4{s * acc[i][0][k], s * acc[i][1][k], s * acc[i][2][k], s * acc[i][3][k]};
            out[1] = f32x4{s * acc[i][4][k], s * acc[i][5][k], s * acc[i][6][k], s * acc[i][7][k]};
        }
    }
}

// The gradients of adapters with several tiles, their sums in order, and of those
// without a token: zeros.
__global__ __launch_bounds__(kThreads) void lora_join_kernel(OuterArgs ox, OuterArgs oy, int table) {
    const OuterArgs& a = blockIdx.z ? oy : ox;
    if (!planned(a.g)) return;
    const int ad = blockIdx.x, size = tile_tokens(table);
    const int tiles = a.g.plan.base[table][ad + 1] - a.g.plan.base[table][ad];
    if (tiles == 1) return;
    const int first = a.g.plan.seg[ad];
    const int64_t all = int64_t(rank_of(a.g, ad)) * a.C, part = int64_t(a.g.R) * a.C;
    float* d = a.d[ad];
    for (int64_t i = 4 * (int64_t(blockIdx.y) * kThreads + threadIdx.x); i < all; i += 4 * int64_t(gridDim.y) * kThreads) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int k = 0; k < tiles; ++k)
            sum += *reinterpret_cast<const f32x4*>(a.part + outer_slot(first + k * size, size, k == tiles - 1) * part + i);
        *reinterpret_cast<f32x4*>(d + i) = sum;
    }
}

}  // namespace

int outer_bf16(const OuterArgs (&a)[2], int table, hipStream_t s) {
    const int R = a[0].g.R, C = a[0].C > a[1].C ? a[0].C : a[1].C, n = a[0].g.n;
    const dim3 grid(unsigned(plan_layout(a[0].g.T, n).max_tiles[table]), unsigned((C + 128 * kWaves - 1) / (128 * kWaves)),
                    R > 64 ? 4 : 2);
    const auto go = [&](auto rt) {
        hipLaunchKernelGGL((lora_outer_bf16_kernel<rt()>), grid, dim3(kThreads), 0, s, a[0], a[1], table);
    };
    if (R <= 16) go(std::integral_constant<int, 1>());
    else if (R <= 32) go(std::integral_constant<int, 2>());
    else go(std::integral_constant<int, 4>());
    STMOE_LAUNCHED();
    const int64_t chunks = (int64_t(R) * C / 4 + kThreads - 1) / kThreads, most = n < 64 ? 512 / n : 8;
    hipLaunchKernelGGL(lora_join_kernel, dim3(unsigned(n), unsigned(chunks < most ? chunks : most), 2), dim3(kThreads), 0, s,
                       a[0], a[1], table);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int shrink_bf16(const ShrinkArgs& a, int table, hipStream_t s) {
    const int tiles = plan_layout(a.g.T, a.g.n).max_tiles[table];
    const auto go = [&](auto rt, auto nt) {
        const dim3 grid(unsigned(tiles * (tile_tokens(table) / (16 * nt()))), unsigned(a.parts));
        hipLaunchKernelGGL((lora_shrink_bf16_kernel<rt(), nt()>), grid, dim3(kThreads), 0, s, a, table);
    };
    const auto with = [&](auto rt) {
        if (table == 0) go(rt, std::integral_constant<int, 1>());
        else go(rt, std::integral_constant<int, rt() == 8 ? 2 : 4>());
    };
    const int R = a.g.R;
    if (R <= 16) with(std::integral_constant<int, 1>());
    else if (R <= 32) with(std::integral_constant<int, 2>());
    else if (R <= 64) with(std::integral_constant<int, 4>());
    else with(std::integral_constant<int, 8>());
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int expand_bf16(const ExpandArgs& a, int table, bool ybf, hipStream_t s) {
    const dim3 grid(unsigned(plan_layout(a.g.T, a.g.n).max_tiles[table]), unsigned((a.C + 128 * kWaves - 1) / (128 * kWaves)));
    const auto go = [&](auto ks, auto pack) {
        if (ybf) hipLaunchKernelGGL((lora_expand_bf16_kernel<ks(), pack(), true>), grid, dim3(kThreads), 0, s, a, table);
        else hipLaunchKernelGGL((lora_expand_bf16_kernel<ks(), pack(), false>), grid, dim3(kThreads), 0, s, a, table);
    };
    const int R = a.g.R;
    if (R <= 16) go(std::integral_constant<int, 1>(), std::true_type());
    else if (R <= 32) go(std::integral_constant<int, 1>(), std::false_type());
    else if (R <= 64) go(std::integral_constant<int, 2>(), std::false_type());
    else go(std::integral_constant<int, 4>(), std::false_type());
    STMOE_LAUNCHED();
    return STMOE_OK;
}

}  // namespace lora
}  // namespace stmoe
