// Low-rank adapters over bf16 rows in whole 16-byte chunks: the products of lora.hip on
// the bf16 matrix instruction (16 x 16 x 32).
//
// One operand of every product is bf16 and exact; the fp32 one (v, u) is split into three
// bf16 pieces, the value's rounding and the roundings of what is left twice: its 24 bits.
// (Two hold 16, which a bf16 result shows where its terms cancel; the third costs the product
// over the rank 1 to 3%: 8192 x 4096, rank 64, 35.0 us with two, 35.7 with three.)
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

// N pieces of eight values.  A number that rounds to an infinity has the largest bf16 number
// for its first piece; of an infinity or NaN nothing is left.
template <int N>
__device__ __forceinline__ void split(const float (&x)[8], bf16x8 (&p)[N]) {
    constexpr float most = 3.38953138925153547590470800371487866880e38f;     // 2^128 (1 - 2^-8)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool number = fabsf(x[i]) < INFINITY;
        float left = number ? fminf(fmaxf(x[i], -most), most) : x[i];
        const float beyond = number ? x[i] - left : 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const __bf16 b = __bf16(left);
            p[k][i] = b;
            left = number ? left - float(b) : 0.f;
            if (k == 0) left += beyond;
        }
    }
}

// The numbers of an operand, zeros in the place of infinities and NaN: what pieces after the
// first are multiplied with where a product came out as NaN.  An infinity against a piece of 0
// or of the other sign than the value would be NaN or take the infinity back.  Looking for NaN
// costs the products nothing that shows (8192 tokens, rank 64, both launches: 68.3 and 68.4 us).
__device__ __forceinline__ bf16x8 numbers(bf16x8 m) {
    union {
        bf16x8 v;
        uint32_t w[4];
    } u;
    u.v = m;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        uint32_t w = u.w[d];
        asm volatile("" : "+v"(w));        // made where it is used: kept beside m it costs registers
        u.w[d] = ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
    }
    return u.v;
}

// Columns of eight rows as operands: fragment j has column j of rows 0 to 7.
__device__ __forceinline__ bf16x8 column(const u32x4 (&rows)[8], int j) {
    u32x4 q;
#pragma unroll
    for (int d = 0; d < 4; ++d)
        q[d] = __builtin_amdgcn_perm(rows[2 * d + 1][j / 2], rows[2 * d][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return operand(q);
}

// Eight values of a row of R from r on, 0 beyond it; the sum of its parts (one or an even
// number), two at a time.
__device__ __forceinline__ void load8(const float* row, int64_t part, int parts, int r, int R, float (&v)[8]) {
    if (R % 8 == 0) {
        const float* at = row + (r < R ? r : 0);
        f32x4 lo = *reinterpret_cast<const f32x4*>(at), hi = *reinterpret_cast<const f32x4*>(at + 4);
        if (parts > 1) {
            lo += *reinterpret_cast<const f32x4*>(at + part);
            hi += *reinterpret_cast<const f32x4*>(at + part + 4);
            for (int p = 2; p < parts; p += 2) {
                const float* a0 = at + p * part;
                const float* a1 = a0 + part;
                const f32x4 l0 = *reinterpret_cast<const f32x4*>(a0), h0 = *reinterpret_cast<const f32x4*>(a0 + 4);
                const f32x4 l1 = *reinterpret_cast<const f32x4*>(a1), h1 = *reinterpret_cast<const f32x4*>(a1 + 4);
                lo += l0 + l1;
                hi += h0 + h1;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = r < R ? lo[i] : 0.f;
            v[4 + i] = r < R ? hi[i] : 0.f;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    for (int p = 0; p < parts; ++p, row += part)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r + i < R) v[i] += row[r + i];
}

// v = x A^T.  16 NT tokens a workgroup (a tile, or a part of one) and, with several
// parts, some of the columns; a wave takes every fourth 64 columns.  Rows go through
// LDS, each wave's own: eight consecutive lanes load 128 bytes of one, where the matrix
// instruction's operand has a row a lane, and loads in that order get 16 bytes a cycle
// and CU out of the cache (4096 tokens x 4096, rank 16: 12.4 us so, 18.1 without LDS).
// Bound by the rows from HBM and, at larger ranks, as much again of A out of the L2s for
// every 32 tokens: 8192 x 4096, rank 64, 28.6 us, 2.3 TB/s of rows (64 tokens a workgroup
// 27.8 in two parts, which cost the next launch more; 16 tokens 32.7).
template <int RT, int NT>
__global__ __launch_bounds__(kThreads) void lora_shrink_bf16_kernel(ShrinkArgs a) {
    constexpr int TOK = 16 * NT, LD = 16 * RT + 4, ROWS = 16 * (NT + RT);
    union Lds {
        char rows[kWaves][ROWS][128];
        float red[2][TOK][LD];
    };
    __shared__ __attribute__((aligned(16))) Lds lds;
    __shared__ int64_t token[TOK];
    Tile tile;
    const int sub = a.g.plan.size / TOK, k0 = (blockIdx.x % sub) * TOK;
    if (!tile_of(a.g, blockIdx.x / sub, tile) || tile.adapter < 0 || k0 >= tile.count) return;
    const int count = tile.count - k0 < TOK ? tile.count - k0 : TOK, first = tile.first + k0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int rank = rank_of(a.g, tile.adapter);
    // lane: chunk lane & 7 of row 8 i + lane / 8.  Tokens and ranks beyond the last ones
    // take another's values: their sums are their own
    const char* row[2 * (NT + RT)];
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) {
        const int k = 8 * i + (lane >> 3);
        const int64_t t = a.g.plan.order[first + (k < count ? k : 0)];
        row[i] = reinterpret_cast<const char*>(a.x) + 2 * (t * a.ld);
        if (wave == 0 && (lane & 7) == 0) token[k] = t;
    }
    const char* m = reinterpret_cast<const char*>(a.m[tile.adapter]);
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) {
        const int r = 8 * i + (lane >> 3);
        row[2 * NT + i] = m + 2 * (int64_t(r < rank ? r : 0) * a.C);
    }
    f32x4 acc[NT][RT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const u32x4 zero = {0u, 0u, 0u, 0u};
    struct Chunk {
        u32x4 v[2 * (NT + RT)];
    };
    auto load = [&](int h0, Chunk& v) __attribute__((always_inline)) {
        const int h = h0 + 8 * (lane & 7);
        if (h0 + 64 <= a.C) {              // whole chunks without a branch around each load
#pragma unroll
            for (int i = 0; i < 2 * (NT + RT); ++i) v.v[i] = *reinterpret_cast<const u32x4*>(row[i] + 2 * int64_t(h));
        } else {
#pragma unroll
            for (int i = 0; i < 2 * (NT + RT); ++i)
                v.v[i] = h < a.C ? *reinterpret_cast<const u32x4*>(row[i] + 2 * int64_t(h)) : zero;   // C is a multiple of 8
        }
    };
    // chunk k of row r is at place k ^ r / 2 % 8: 16 lanes read 16 rows without a conflict
    char* const mine = lds.rows[wave][0];
    const int wr = (lane >> 3) * 128 + ((lane & 7) ^ (lane >> 4)) * 16;
    const int rd = c * 128 + (q ^ (c >> 1)) * 16;
    auto use = [&](const Chunk& v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2 * (NT + RT); ++i) *reinterpret_cast<u32x4*>(mine + 1024 * i + (i % 2 ? wr ^ 64 : wr)) = v.v[i];
        // a wave's LDS accesses complete in order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 x[NT], w[RT];
#pragma unroll
            for (int i = 0; i < NT; ++i) x[i] = operand(*reinterpret_cast<const u32x4*>(mine + 2048 * i + (rd ^ 64 * u)));
#pragma unroll
            for (int i = 0; i < RT; ++i) w[i] = operand(*reinterpret_cast<const u32x4*>(mine + 2048 * (NT + i) + (rd ^ 64 * u)));
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int i = 0; i < NT; ++i) acc[i][j] = mfma(w[j], x[i], acc[i][j]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // the next columns are on their way while these are used
    const int step = 64 * kWaves * int(gridDim.y);
    int h0 = 64 * (blockIdx.y * kWaves + wave);
    if (rank > 0 && h0 < a.C) {
        Chunk v0, v1;
        load(h0, v0);
        for (;;) {
            h0 += step;
            if (h0 < a.C) load(h0, v1);
            use(v0);
            if (h0 >= a.C) break;
            h0 += step;
            if (h0 < a.C) load(h0, v0);
            use(v1);
            if (h0 >= a.C) break;
        }
    }
    // the waves' sums, two and two
    __syncthreads();
    auto at = [&](int b, int i, int j) { return reinterpret_cast<f32x4*>(&lds.red[b][16 * i + c][16 * j + 4 * q]); };
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
    // 4 RT threads a token, four ranks each
#pragma unroll
    for (int i = threadIdx.x; i < TOK * 4 * RT; i += kThreads) {
        const int k = i / (4 * RT), r = 4 * (i % (4 * RT));
        if (k >= count || r >= R) continue;
        float* to = out + token[k] * R + r;
        const f32x4 p = *reinterpret_cast<const f32x4*>(&lds.red[0][k][r]), o = *reinterpret_cast<const f32x4*>(&lds.red[1][k][r]);
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = r + j < rank ? s * (p[j] + o[j]) : 0.f;
        if (R % 4 == 0) {
            *reinterpret_cast<f32x4*>(to) = v;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (r + j < R) to[j] = v[j];
        }
    }
}

// y = base + s v B.  A tile of up to 16 NS tokens and 512 columns a workgroup, 128 a
// wave, whose lane (c, q) holds columns 8 c .. + 7 of ranks 8 q .. + 7 (of every 32) as
// the column operand, that of instruction j being columns 8 c + j: it gets columns 8 c
// .. + 7 of tokens 4 q .. + 3, so that 16 lanes load and store 256 bytes of a row.  v's
// pieces are made once for the workgroup, in LDS.  With a rank of 16 at most the lanes q =
// 2, 3 hold the same ranks as q = 0, 1, against the second piece of v.  Bound by base and
// y: 8192 x 4096 bf16, rank 64, 35.7 us, 3.8 TB/s of them (with two pieces 35.0, and so 39
// for 128 tokens a workgroup and 49 with columns as the row operand, 16 bytes of each of 64
// rows a store); 4096 x 4096, rank 16, 19.3 us, 3.5 TB/s.
template <int KS, bool PACK, bool YBF, int NS>
__global__ __launch_bounds__(kThreads, KS <= 2 && YBF ? 3 : NS == 1 ? 2 : 1) void lora_expand_bf16_kernel(ExpandArgs a) {
    constexpr int P = 3, NM = PACK ? 2 : KS * P, W = YBF ? 1 : 2;
    __shared__ u32x4 vf[NS][NM][64];
    __shared__ __attribute__((aligned(16))) int32_t token[16 * NS];
    Tile tile;
    if (!tile_of(a.g, blockIdx.y, tile)) return;
    const int R = a.g.R, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int64_t part = int64_t(a.g.T) * R;
    const int32_t* order = a.g.plan.order + tile.first;
    if (a.v_out && a.parts > 1 && tile.adapter >= 0) sum_parts(a, order, tile.count, blockIdx.x, gridDim.x);
    if (tile.adapter < 0 && a.base == a.y) return;
    // tokens beyond the last one: the first, whose row is not stored again
    if (threadIdx.x < 16 * NS) token[threadIdx.x] = order[int(threadIdx.x) < tile.count ? threadIdx.x : 0];
    const int o = (blockIdx.x * kWaves + wave) * 128 + 8 * c, oc = o < a.C ? o : 0;    // columns beyond the last: not stored
    const u32x4 zero = {0u, 0u, 0u, 0u};
    auto load_base = [&](const int4& t, u32x4 (&b)[4][W]) __attribute__((always_inline)) {
        const int ts[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < W; ++w)
                b[i][w] = a.base ? reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.base) +
                                                                  (YBF ? 2 : 4) * (ts[i] * a.ld_base + oc))[w]
                                 : zero;
    };
    auto tokens = [&](int k) __attribute__((always_inline)) { return *reinterpret_cast<const int4*>(token + 16 * k + 4 * q); };
    bf16x8 mf[KS][8];
    u32x4 b0[4][W], b1[4][W];
    // the first tokens' base, beside what the product waits for
    int4 t0, t1;
    {
        int ts[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ts[i] = order[4 * q + i < tile.count ? 4 * q + i : 0];
        t0 = make_int4(ts[0], ts[1], ts[2], ts[3]);
    }
    float s = 0.f;
    if (tile.adapter >= 0) {
        const int rank = rank_of(a.g, tile.adapter);
        const char* m = reinterpret_cast<const char*>(a.m[tile.adapter]);
        s = a.scaled && a.g.scales ? a.g.scales[tile.adapter] : 1.f;
        u32x4 rows[KS][8];
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // ranks beyond the last one count as zeros, columns are not stored
                const int r = 32 * k + 8 * (PACK ? q & 1 : q) + i;
                const int64_t at = int64_t(r < rank ? r : 0) * a.C + oc;
                rows[k][i] = rank > 0 ? *reinterpret_cast<const u32x4*>(m + 2 * at) : zero;
            }
        load_base(t0, b0);
#pragma unroll
        for (int i = threadIdx.x; i < 64 * NS * KS; i += kThreads) {
            const int l = i & 63, k = (i >> 6) % KS, n = (i >> 6) / KS, lq = l >> 4, lt = 16 * n + (l & 15);
            if (16 * n >= tile.count) break;
            float v[8];
            load8(a.v + int64_t(order[lt < tile.count ? lt : 0]) * R, part, a.parts, 32 * k + 8 * (PACK ? lq & 1 : lq), R, v);
            bf16x8 p[P];
            split(v, p);
            if constexpr (PACK) {
                *reinterpret_cast<bf16x8*>(&vf[n][0][l]) = lq < 2 ? p[0] : p[1];
                *reinterpret_cast<bf16x8*>(&vf[n][1][l]) = lq < 2 ? p[2] : operand(zero);
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) *reinterpret_cast<bf16x8*>(&vf[n][P * k + j][l]) = p[j];
            }
        }
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            if (rank < (PACK ? 16 : 32 * (k + 1)))
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (32 * k + 8 * (PACK ? q & 1 : q) + i >= rank) rows[k][i] = zero;
#pragma unroll
            for (int j = 0; j < 8; ++j) mf[k][j] = column(rows[k], j);
        }
    } else {
        load_base(t0, b0);
    }
    __syncthreads();
    auto finish = [&](int k, const int4& t, const u32x4 (&b)[4][W]) __attribute__((always_inline)) {
        f32x4 acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (tile.adapter >= 0) {
#pragma unroll
            for (int i = NM - 1; i >= 0; --i) {
                const bf16x8 v = operand(vf[k][i][lane]);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = mfma(v, mf[PACK ? 0 : i / P][j], acc[j]);
            }
            bool nan = false;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                nan |= __builtin_isunordered(acc[j][0], acc[j][1]) || __builtin_isunordered(acc[j][2], acc[j][3]);
            if (__any(nan))
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = NM - 1; i >= 0; --i) {
                        const bf16x8 m = mf[PACK ? 0 : i / P][j];
                        const bool whole = PACK ? i == 0 && q < 2 : i % P == 0;
                        acc[j] = mfma(operand(vf[k][i][lane]), whole ? m : numbers(m), acc[j]);
                    }
                }
        }
        const int ts[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (16 * k + 4 * q + i >= tile.count || o >= a.C) continue;
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = YBF ? (j % 2 ? bf16_hi(b[i][0][j / 2]) : bf16_lo(b[i][0][j / 2]))
                                    : __uint_as_float(b[i][W == 2 ? j / 4 : 0][j % 4]);
                y[j] = tile.adapter >= 0 ? f + s * acc[j][i] : f;
            }
            char* out = reinterpret_cast<char*>(a.y) + (YBF ? 2 : 4) * (ts[i] * a.ld + o);
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
    };
    // the next tokens' base is on its way while these are finished
#pragma unroll
    for (int k = 0; k < NS; k += 2) {
        if (16 * k >= tile.count) break;
        if (k + 1 < NS) load_base(t1 = tokens(k + 1), b1);
        finish(k, t0, b0);
        if (k + 1 >= NS || 16 * (k + 1) >= tile.count) break;
        if (k + 2 < NS) load_base(t0 = tokens(k + 2), b0);
        finish(k + 1, t1, b1);
    }
}

// d = u^T x of a tile of tokens (a gradient, or its sum of an adapter with several
// tiles).  512 columns and up to 64 ranks a workgroup, 128 columns a wave, 32 tokens at
// a time: the lane (c, q) loads columns 8 c .. + 7 of tokens 8 q .. + 7, the column
// operand of instruction j being columns 8 c + j, and gets them of ranks 4 q .. + 3.  u's three pieces are made once for the
// workgroup, in LDS, 128 tokens at a time.  Bound by the rows: both gradients of 4096 x
// 4096 each way, rank 16, in 19.7 us, 3.4 TB/s and 8 MB of sums of tiles on top.
constexpr int kStage = 4;          // times 32 tokens

template <int RT>
__global__ __launch_bounds__(kThreads) void lora_outer_bf16_kernel(OuterArgs ox, OuterArgs oy) {
    constexpr int P = 3;
    __shared__ u32x4 uf[kStage][RT][P][64];
    __shared__ __attribute__((aligned(16))) int32_t order[tile_tokens(kTables - 1) + 64 * kStage];
    const OuterArgs a = one_of(blockIdx.z & 1, ox, oy);
    const int rt0 = (blockIdx.z >> 1) * 64;
    Tile tile;
    if (!tile_of(a.g, blockIdx.y, tile)) return;
    if (tile.adapter < 0 || int(blockIdx.x) * 128 * kWaves >= a.C) return;
    const int R = a.g.R, rank = rank_of(a.g, tile.adapter);
    if (rt0 >= rank) return;
    // tokens beyond the last one (loads go up to two stages past a stage's first, which is
    // below the count): the first, whose values are not used
    for (int i = threadIdx.x; i < tile.count + 64 * kStage; i += kThreads)
        order[i] = a.g.plan.order[tile.first + (i < tile.count ? i : 0)];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int h0 = (blockIdx.x * kWaves + wave) * 128, h = h0 + 8 * c;
    const char* x = reinterpret_cast<const char*>(a.x) + 2 * int64_t(h < a.C ? h : 0);   // columns beyond the last: not stored
    const u32x4 zero = {0u, 0u, 0u, 0u};
    f32x4 acc[RT][8];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // thread: rank c of tile i, tokens 8 q .. + 7 of the wave's 32
    float u[RT][8];
    auto load_u = [&](int k0) __attribute__((always_inline)) {
        const int p0 = k0 + 32 * wave + 8 * q;
        const int4 t0 = *reinterpret_cast<const int4*>(order + p0), t1 = *reinterpret_cast<const int4*>(order + p0 + 4);
        const int t[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = rt0 + 16 * i + c;
#pragma unroll
            for (int k = 0; k < 8; ++k) u[i][k] = a.u[int64_t(t[k]) * R + (r < R ? r : 0)];
#pragma unroll
            for (int k = 0; k < 8; ++k) u[i][k] = p0 + k < tile.count && r < rank ? u[i][k] : 0.f;
        }
    };
    auto load_x = [&](int k0, u32x4 (&rows)[8]) __attribute__((always_inline)) {
        const int p0 = k0 + 8 * q;
        const int4 t0 = *reinterpret_cast<const int4*>(order + p0), t1 = *reinterpret_cast<const int4*>(order + p0 + 4);
        const int t[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) rows[k] = *reinterpret_cast<const u32x4*>(x + 2 * (t[k] * a.ld));
    };
    u32x4 rows[2][8];
    __syncthreads();
    load_u(0);
    load_x(0, rows[0]);
    load_x(32, rows[1]);
    for (int k0 = 0; k0 < tile.count; k0 += 32 * kStage) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            bf16x8 p[P];
            split(u[i], p);
#pragma unroll
            for (int j = 0; j < P; ++j) *reinterpret_cast<bf16x8*>(&uf[wave][i][j][lane]) = p[j];
        }
        load_u(k0 + 32 * kStage);
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kStage; ++n) {
            if (k0 + 32 * n >= tile.count) break;
            bf16x8 xf[8];
            if (k0 + 32 * (n + 1) > tile.count)
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k0 + 32 * n + 8 * q + k >= tile.count) rows[n & 1][k] = zero;
#pragma unroll
            for (int j = 0; j < 8; ++j) xf[j] = column(rows[n & 1], j);
            // two loads of 32 tokens are on their way while these are used
            load_x(k0 + 32 * (n + 2), rows[n & 1]);
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int p = P - 1; p >= 0; --p) {
                    const bf16x8 b = operand(uf[n][i][p][lane]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[i][j] = mfma(b, xf[j], acc[i][j]);
                }
        }
    }
    const int tiles = a.g.plan.base[tile.adapter + 1] - a.g.plan.base[tile.adapter];
    const float s = a.scaled && a.g.scales ? a.g.scales[tile.adapter] : 1.f;
    float* d = tiles == 1 ? a.d[tile.adapter]
                          : a.part + int64_t(outer_slot(tile.first, a.g.plan.size, tile.piece == tiles - 1)) * R * a.C;
    if (h >= a.C) return;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = rt0 + 16 * i + 4 * q + k;
            if (r >= rank) continue;
#pragma unroll
            for (int j = 0; j < 8; j += 2) nan |= __builtin_isunordered(acc[i][j][k], acc[i][j + 1][k]);
            f32x4* out = reinterpret_cast<f32x4*>(d + int64_t(r) * a.C + h);
            out[0] = f32x4{s * acc[i][0][k], s * acc[i][1][k], s * acc[i][2][k], s * acc[i][3][k]};
            out[1] = f32x4{s * acc[i][4][k], s * acc[i][5][k], s * acc[i][6][k], s * acc[i][7][k]};
        }
    // sums that are NaN, perhaps of an infinite x against a piece of u (numbers()): again in fp32
    if (!__any(nan)) return;
#pragma unroll 1
    for (int i = 0; i < RT; ++i) {
        float sum[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[k][j] = 0.f;
        const int r0 = rt0 + 16 * i + 4 * q;
#pragma unroll 1
        for (int p = 0; p < tile.count; ++p) {
            const int64_t t = order[p];
            const u32x4 row = *reinterpret_cast<const u32x4*>(x + 2 * (t * a.ld));
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float v = r0 + k < rank ? a.u[t * R + r0 + k] : 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[k][j] += v * (j % 2 ? bf16_hi(row[j / 2]) : bf16_lo(row[j / 2]));
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (r0 + k >= rank) continue;
            float* out = d + int64_t(r0 + k) * a.C + h;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (out[j] != out[j]) out[j] = s * sum[k][j];
        }
    }
}

}  // namespace

int outer_bf16(const OuterArgs (&a)[2], int table, hipStream_t s) {
    const int R = a[0].g.R, C = a[0].C > a[1].C ? a[0].C : a[1].C, n = a[0].g.n;
    const dim3 grid(unsigned((C + 128 * kWaves - 1) / (128 * kWaves)), unsigned(plan_layout(a[0].g.T, n).max_tiles[table]),
                    R > 64 ? 4 : 2);
    const auto go = [&](auto rt) {
        hipLaunchKernelGGL((lora_outer_bf16_kernel<rt()>), grid, dim3(kThreads), 0, s, a[0], a[1]);
    };
    if (R <= 16) go(std::integral_constant<int, 1>());
    else if (R <= 32) go(std::integral_constant<int, 2>());
    else go(std::integral_constant<int, 4>());
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int shrink_bf16(const ShrinkArgs& o, int table, hipStream_t s) {
    ShrinkArgs a = o;
    a.g = with_table(o.g, table);
    const int tiles = plan_layout(a.g.T, a.g.n).max_tiles[table];
    const auto go = [&](auto rt, auto nt) {
        const dim3 grid(unsigned(tiles * (tile_tokens(table) / (16 * nt()))), unsigned(a.parts));
        hipLaunchKernelGGL((lora_shrink_bf16_kernel<rt(), nt()>), grid, dim3(kThreads), 0, s, a);
    };
    const auto with = [&](auto rt) {
        if (table == 0) go(rt, std::integral_constant<int, 1>());
        else go(rt, std::integral_constant<int, 2>());
    };
    const int R = a.g.R;
    if (R <= 16) with(std::integral_constant<int, 1>());
    else if (R <= 32) with(std::integral_constant<int, 2>());
    else if (R <= 64) with(std::integral_constant<int, 4>());
    else with(std::integral_constant<int, 8>());
    STMOE_LAUNCHED();
    return STMOE_OK;
}

int expand_bf16(const ExpandArgs& o, int table, bool ybf, hipStream_t s) {
    ExpandArgs a = o;
    a.g = with_table(o.g, table);
    const unsigned cols = unsigned((a.C + 128 * kWaves - 1) / (128 * kWaves));
    const int R = a.g.R;
    const auto with = [&](auto ks, auto pack, auto ns) {
        const dim3 grid(cols, unsigned(plan_layout(a.g.T, a.g.n).max_tiles[table]));
        if (ybf) hipLaunchKernelGGL((lora_expand_bf16_kernel<ks(), pack(), true, ns()>), grid, dim3(kThreads), 0, s, a);
        else hipLaunchKernelGGL((lora_expand_bf16_kernel<ks(), pack(), false, ns()>), grid, dim3(kThreads), 0, s, a);
    };
    const auto go = [&](auto ks, auto pack) {
        if (table == 0) with(ks, pack, std::integral_constant<int, 1>());
        else with(ks, pack, std::integral_constant<int, 4>());
    };
    if (R <= 16) go(std::integral_constant<int, 1>(), std::true_type());
    else if (R <= 32) go(std::integral_constant<int, 1>(), std::false_type());
    else if (R <= 64) go(std::integral_constant<int, 2>(), std::false_type());
    else go(std::integral_constant<int, 4>(), std::false_type());
    STMOE_LAUNCHED();
    return STMOE_OK;
}

}  // namespace lora
}  // namespace stmoe
