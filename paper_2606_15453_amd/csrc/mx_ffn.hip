// Expert FFN (Section 2) over experts packed as microscaled 4-bit floats
// (mx_format.h), for one token to whole prompts:
//   y[t] = sum_k w[t][k] W_down e (silu(W_gate e x[t]) * (W_up e x[t])) + shared experts.
//
// The weights' values are exact in bf16, so both projections run on the bf16
// matrix instructions with fp32 accumulation: a lane's 16 code bytes become
// the row operand in registers, tokens are the columns.  fp32 values (x, and
// the activations when y is fp32) are split into two bf16 pieces, the value's
// rounding and the rounding of what is left: 16 significant bits, two
// instructions per operand.
#include "mx_format.h"

namespace stmoe {
namespace {

using namespace mx;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kPlanThreads = 1024;
constexpr int kMaxShared = 8;
constexpr int kMaxT = 65536;
constexpr int kMaxGroups = kMaxE + kMaxShared;

struct MxArgs {
    const void* x;                  // [T][H]
    const int32_t* idx;             // [T][K]
    const float* w;                 // [T][K]
    const void* const* eptr;        // [E]
    const void* const* sptr;        // [ns]
    void* y;                        // [T][H]
    int T, K, H, I, E, ns, ks;      // ks = K + ns: entries per token
    int tm;                         // tokens per tile
    int tsplits;                    // parts of the down launch's contraction
    // workspace
    int32_t* order;                 // [expert][T] its entries (t * ks + k)
    int32_t* cnt;                   // [expert] how many
    int4* tiles;                    // (expert, first place in its order, tokens, -)
    int32_t* ntiles;
    uint16_t* act;                  // [entry][piece][I] bf16 pieces
    void* part;                     // [part][entry][H] terms of y
    // decode steps (T <= 16)
    struct DecodeSlot* slots;       // by ascending expert, the shared ones last
    int32_t* nslots;
    int32_t* arrived;               // [row block of H] workgroups of the down launch that are done
    float* split;                   // [row block][split][256] their sums
    unsigned long long* n_experts;  // counts distinct routed experts (timed decode layers), or null
};

// A distinct expert of a decode step and, per token, the entry that selects it.
struct DecodeSlot {
    int32_t g;
    uint8_t k[kMaxB];               // kNone: the token does not select it
};
constexpr int kNone = 255;

// Column operand: eight consecutive values of a row as bf16 pieces.
template <bool F32>
struct Pieces;
template <>
struct Pieces<false> {
    static constexpr int N = 1;
    bf16x8 p[1];
};
template <>
struct Pieces<true> {
    static constexpr int N = 2;
    bf16x8 p[2];
};

// A value as two bf16 numbers; infinities and NaN (and what rounds to
// infinity) keep to the first.  The difference is that of the rounded value:
// fused with the product that gave v, it would depend on how the compiler
// arranged the caller, and a token's bits on the tile it falls into.
__device__ __forceinline__ void split(float v, __bf16& hi, __bf16& lo) {
#pragma clang fp contract(off)
    hi = __bf16(v);
    const float h = float(hi);
    lo = __builtin_isfinite(h) ? __bf16(v - h) : __bf16(0.f);
}

// Eight consecutive values as loaded.
template <bool F32>
struct Raw {
    uint4 q[F32 ? 2 : 1];
};

template <bool F32>
__device__ __forceinline__ Raw<F32> load_raw(const void* x, size_t at, bool in) {
    Raw<F32> r;
    const uint4* s = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(x) + at * (F32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) r.q[i] = in ? s[i] : make_uint4(0u, 0u, 0u, 0u);
    return r;
}

__device__ __forceinline__ Pieces<false> pieces(const Raw<false>& r) {
    union {
        uint4 q;
        bf16x8 v;
    } u;
    u.q = r.q[0];
    return Pieces<false>{{u.v}};
}

__device__ __forceinline__ Pieces<true> pieces(const Raw<true>& r) {
    Pieces<true> o;
    const uint32_t w[8] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w, r.q[1].x, r.q[1].y, r.q[1].z, r.q[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        __bf16 h, l;
        split(__uint_as_float(w[i]), h, l);
        o.p[0][i] = h;
        o.p[1][i] = l;
    }
    return o;
}

// g / (1 + exp(-g)) with the hardware's exponential and reciprocal (2^-23 of
// their values; the exponent's product rounds to 2^-24 of |g|, so silu is off
// by less than 2e-6 of itself down to g = -20 and negligible below).
__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)); }

// The expert of an entry, or -1 where it names none or repeats an earlier
// entry of its token (the first one counts).
__device__ __forceinline__ int entry_expert(const MxArgs& a, int t, int k) {
    if (k >= a.K) return a.E + (k - a.K);
    const int32_t* row = a.idx + size_t(t) * a.K;
    const int e = row[k];
    if (e < 0 || e >= a.E) return -1;
    for (int j = 0; j < k; ++j)
        if (row[j] == e) return -1;
    return e;
}

// A barrier for what passes through LDS alone: __syncthreads would also wait
// for the stores to memory under way (3 us for 1024 scattered ones).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The tiles of at most tm tokens, experts in order (one workgroup; cnt in LDS).
__device__ __forceinline__ void list_tiles(const MxArgs& a, const int* cnt, int* tile) {
    const int tid = threadIdx.x, G = a.E + a.ns;
    if (tid < 64) {
        // running sums of the tile counts, 64 experts at a time
        int before = 0, used = 0;
        for (int g0 = 0; g0 < G; g0 += 64) {
            const int g = g0 + tid, c = g < G ? cnt[g] : 0;
            int v = (c + a.tm - 1) / a.tm;
            used += __popcll(__ballot(c > 0 && g < a.E));
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(v, d, 64);
                if (tid >= d) v += o;
            }
            if (g < G) tile[g + 1] = before + v;
            before += __shfl(v, 63, 64);
        }
        if (tid == 0) {
            tile[0] = 0;
            *a.ntiles = before;
            if (a.n_experts) *a.n_experts += (unsigned long long)(used);
        }
    }
    __syncthreads();
    for (int g = tid >> 4; g < G; g += kPlanThreads >> 4)
        for (int j = tid & 15; j * a.tm < cnt[g]; j += 16)
            a.tiles[tile[g] + j] = make_int4(g, j * a.tm, min(a.tm, cnt[g] - j * a.tm), 0);
}

__global__ __launch_bounds__(kPlanThreads) void mx_tiles_kernel(MxArgs a) {
    __shared__ int cnt[kMaxGroups], tile[kMaxGroups + 1];
    for (int g = threadIdx.x; g < a.E + a.ns; g += kPlanThreads) cnt[g] = a.cnt[g];
    __syncthreads();
    list_tiles(a, cnt, tile);
}

// One expert's entries per workgroup, by token: order[g * T ..] and cnt[g].  A
// thread compares its token's KU entries (FOUR: K is a multiple of four and
// they are loaded four at a time) and takes the first that names the expert;
// a wave's place is its lanes' ballot, the waves' places meet in LDS.
template <int KU, bool FOUR>
__global__ __launch_bounds__(kPlanThreads) void mx_order_kernel(MxArgs a) {
    constexpr int W = kPlanThreads / 64;
    __shared__ int found[2][W];
    const int g = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t* out = a.order + size_t(g) * a.T;
    if (g >= a.E) {
        for (int t = threadIdx.x; t < a.T; t += kPlanThreads) out[t] = t * a.ks + a.K + (g - a.E);
        if (threadIdx.x == 0) a.cnt[g] = a.T;
        return;
    }
    int before = 0;
    for (int t0 = 0, par = 0; t0 < a.T; t0 += kPlanThreads, par ^= 1) {
        const int t = t0 + threadIdx.x;
        const int32_t* row = a.idx + size_t(min(t, a.T - 1)) * a.K;
        int k = -1;
#pragma unroll
        for (int j = KU - (FOUR ? 4 : 1); j >= 0; j -= FOUR ? 4 : 1) {
            // beyond K the last entry again, which does not count there
            if constexpr (FOUR) {
                const int4 e = *reinterpret_cast<const int4*>(row + min(j, a.K - 4));
                const int f = e.x == g ? j : e.y == g ? j + 1 : e.z == g ? j + 2 : e.w == g ? j + 3 : -1;
                k = f >= 0 && j < a.K ? f : k;
            } else {
                k = row[min(j, a.K - 1)] == g && j < a.K ? j : k;
            }
        }
        if (t >= a.T) k = -1;
        const unsigned long long m = __ballot(k >= 0);
        if (lane == 0) found[par][wave] = __popcll(m);
        lds_barrier();
        int base = before;
#pragma unroll
        for (int v = 0; v < W; ++v) {
            const int c = found[par][v];
            base += v < wave ? c : 0;
            before += c;
        }
        if (k >= 0) out[base + __popcll(m & ((1ull << lane) - 1ull))] = t * a.ks + k;
    }
    if (threadIdx.x == 0) a.cnt[g] = before;
}

// All experts' entries and the tiles by one workgroup, 1024 tokens at a time.
// An expert's tokens are bits of a mask in LDS, a token's place the number of
// bits below its own; a bit that its thread finds set is a repeated expert.
// For up to 1024 entries: 4 us, where the two launches above take 3 us each;
// its CU needs 4 us for every 1024 tokens (4096 tokens of top-8: 25 us).
// The KU entries are handled side by side, without branches, so that their LDS
// accesses overlap; entries that name no expert meet a word of their own.
template <int KU>
__global__ __launch_bounds__(kPlanThreads) void mx_plan_kernel(MxArgs a) {
    constexpr int W = kPlanThreads / 32;                    // words of a mask
    __shared__ uint32_t mask[kMaxE + 2][W];                 // the last two: nobody's

    __shared__ uint16_t below[kMaxE][W];
    __shared__ int cnt[kMaxGroups], tile[kMaxGroups + 1];
    const int tid = threadIdx.x, G = a.E + a.ns;
    const bool four = a.K % 4 == 0 && reinterpret_cast<uintptr_t>(a.idx) % 16 == 0;
    for (int g = tid; g < G; g += kPlanThreads) cnt[g] = g < a.E ? 0 : a.T;
    int e[KU];
    auto load = [&](int t) __attribute__((always_inline)) {
        const int32_t* row = a.idx + size_t(t < a.T ? t : 0) * a.K;
#pragma unroll
        for (int j = 0; j < KU; j += 4) {
            int4 v = make_int4(-1, -1, -1, -1);
            if (four) {
                if (j < a.K) v = *reinterpret_cast<const int4*>(row + j);
            } else {
                if (j < a.K) v.x = row[j];
                if (j + 1 < a.K) v.y = row[j + 1];
                if (j + 2 < a.K) v.z = row[j + 2];
                if (j + 3 < a.K) v.w = row[j + 3];
            }
            e[j] = t < a.T ? v.x : -1;
            e[j + 1] = t < a.T ? v.y : -1;
            e[j + 2] = t < a.T ? v.z : -1;
            e[j + 3] = t < a.T ? v.w : -1;
        }
    };
    load(tid);
    for (int t0 = 0; t0 < a.T; t0 += kPlanThreads) {
        const int t = t0 + tid, w = tid >> 5;
        for (int i = tid; i < a.E * W; i += kPlanThreads) mask[0][i] = 0u;
        lds_barrier();
        uint32_t* word[KU];
        bool mine[KU];
#pragma unroll
        for (int j = 0; j < KU; ++j) {
            mine[j] = e[j] >= 0 && e[j] < a.E;
            word[j] = mine[j] ? &mask[e[j]][w] : &mask[kMaxE][tid & 63];
        }
        const uint32_t bit = 1u << (tid & 31);
        uint32_t was[KU];
#pragma unroll
        for (int j = 0; j < KU; ++j) was[j] = atomicOr(word[j], mine[j] ? bit : 0u);
#pragma unroll
        for (int j = 0; j < KU; ++j) mine[j] &= !(was[j] & bit);
        if (t0 + kPlanThreads < a.T) load(t + kPlanThreads);
        lds_barrier();
        // 32 lanes: an expert's words
        for (int g = w; g < a.E; g += W) {
            const int l = tid & 31, c = __builtin_popcount(mask[g][l]);
            int v = c;
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up(v, d, 32);
                if (l >= d) v += o;
            }
            below[g][l] = uint16_t(v - c);
        }
        lds_barrier();
        int at[KU], to[KU];
#pragma unroll
        for (int j = 0; j < KU; ++j) {
            const int g = mine[j] ? int(word[j] - &mask[0][0]) / W : 0;
            to[j] = g;
            at[j] = cnt[g] + below[g][w] + __builtin_popcount(mask[g][w] & (bit - 1u));
        }
#pragma unroll
        for (int j = 0; j < KU; ++j)
            if (mine[j]) a.order[size_t(to[j]) * a.T + at[j]] = t * a.ks + j;
        if (t < a.T)
            for (int s = 0; s < a.ns; ++s) a.order[size_t(a.E + s) * a.T + t] = t * a.ks + a.K + s;
        lds_barrier();
        if (tid < a.E) cnt[tid] += below[tid][W - 1] + __builtin_popcount(mask[tid][W - 1]);
        lds_barrier();
    }
    list_tiles(a, cnt, tile);
}

// fp32 hidden states as two bf16 pieces per row: [T][2][H].
__global__ __launch_bounds__(kThreads) void mx_split_kernel(const float* x, int64_t n4, int H4, uint16_t* o) {
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n4; i += int64_t(gridDim.x) * kThreads) {
        const float4 v = reinterpret_cast<const float4*>(x)[i];
        const int64_t t = i / H4;
        union {
            __bf16 b[4];
            uint2 q;
        } hi, lo;
        split(v.x, hi.b[0], lo.b[0]);
        split(v.y, hi.b[1], lo.b[1]);
        split(v.z, hi.b[2], lo.b[2]);
        split(v.w, hi.b[3], lo.b[3]);
        reinterpret_cast<uint2*>(o)[i + t * H4] = hi.q;
        reinterpret_cast<uint2*>(o)[i + t * H4 + H4] = lo.q;
    }
}

// A blob as a buffer: its address and size in scalar registers, a uniform
// offset and the lane's, and nothing read beyond its end.  (A load through a
// generic pointer would count as an LDS access too, and every wait for LDS
// would wait for the weights in flight.)
typedef __amdgpu_buffer_rsrc_t BlobRef;

__device__ __forceinline__ BlobRef expert_blob(const MxArgs& a, const Blob& L, int g) {
    const void* p = g < a.E ? a.eptr[g] : a.sptr[g - a.E];
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(uint32_t(L.total)), 0x00027000);
}

__device__ __forceinline__ u32x4 load_codes(BlobRef r, uint32_t at, uint32_t lane) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, int(lane * 16u), int(at), 0);
}


// ---------------------------------------------------------------- prompts
//
// A workgroup multiplies 256 weight rows (128 of gate and the same of up, or
// 256 of down) with a tile of up to 16 NT tokens of one expert.  Each wave
// holds 64 rows: their codes go from global memory to its registers and are
// decoded there, once for all tokens of the tile; the tokens' columns pass
// through LDS, 128 at a time, double-buffered.  A column's 256 bytes lie as 16
// chunks of eight values, chunk i in place i ^ (token % 16), so that the 16
// lanes of a read, one chunk of 16 tokens, meet 16 different places.
template <bool UP, int NP, int NT, bool F32>
__device__ __forceinline__ void tile_product(const MxArgs& a, const int4 tl, int bk, int sp, u32x4* xs, int* ent) {
    constexpr int TM = 16 * NT;
    constexpr int RB = 4;                                   // row blocks per wave
    constexpr int CH = kTileCols / 8;                       // chunks per column
    const uint32_t lane = threadIdx.x & 63;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Blob L = blob(a.H, a.I);
    const BlobRef ref = expert_blob(a, L, tl.x);
    const int C = UP ? a.H : a.I, R = UP ? a.I : a.H;
    const int KT = col_tiles(C), KG = col_groups(C), NB = row_blocks(R);
    if (tid < TM) ent[tid] = a.order[size_t(tl.x) * a.T + tl.y + min(tid, tl.z - 1)];
    // the wave's row blocks; beyond the matrix the last one again, not stored
    uint32_t wc[RB], wsc[RB];
    int rb[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        rb[i] = UP ? bk * 8 + wave * 2 + (i & 1) : bk * 16 + wave * 4 + i;
        const int b = min(rb[i], NB - 1);
        const size_t co = UP ? (i < 2 ? L.gate : L.up) : L.down, so = UP ? (i < 2 ? L.gate_s : L.up_s) : L.down_s;
        wc[i] = uint32_t(co) + uint32_t(b * KT) * kTileBytes;
        wsc[i] = uint32_t(so) + uint32_t(b * KG) * kGroupBytes;
    }
    __syncthreads();
    // thread: chunk tid % 16 of tokens tid / 16 + 16 j
    const u32x4* cols = reinterpret_cast<const u32x4*>(UP ? a.x : a.act);
    uint32_t src[NT];                                       // in chunks
    const int chunk = tid % CH;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int e = ent[tid / CH + 16 * j];
        src[j] = uint32_t(UP ? e / a.ks : e) * uint32_t(NP * C / 8);
    }
    const int put = tid / CH * CH + (chunk ^ (tid / CH & 15));
    u32x4 xr[NT], wn[RB];
    uint32_t sn[RB];
    // iteration it: piece it % NP of column tile it / NP.  Chunks beyond the
    // row's end read its first one: their codes are zero, and if the row holds
    // a NaN or an infinity its results are not finite without it too.
    auto load = [&](int it) __attribute__((always_inline)) {
        const int kt = it / NP, p = it - kt * NP;
        const int at = kt * kTileCols + chunk * 8;
        const uint32_t off = uint32_t(p * C + (at < C ? at : 0)) / 8;
#pragma unroll
        for (int j = 0; j < NT; ++j) xr[j] = cols[src[j] + off];
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            wn[i] = load_codes(ref, wc[i] + uint32_t(kt) * kTileBytes, lane);
            sn[i] = __builtin_amdgcn_raw_buffer_load_b8(
                ref, int(lane * 4u), int(wsc[i] + uint32_t(kt / kGroupTiles) * kGroupBytes + uint32_t(kt % kGroupTiles)), 0);
        }
    };
    f32x4 acc[RB][NT];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int c = int(lane & 15), q = int(lane >> 4);
    // the workgroup's share of the contraction
    const int it0 = UP ? 0 : KT * sp / a.tsplits * NP, iters = UP ? KT * NP : KT * (sp + 1) / a.tsplits * NP;
    load(it0);
#pragma unroll
    for (int j = 0; j < NT; ++j) xs[(it0 & 1) * TM * CH + put + j * 16 * CH] = xr[j];
    for (int it = it0; it < iters; ++it) {
        u32x4 w[RB];
        float sc[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            w[i] = wn[i];
            sc[i] = scale_of(sn[i]);
        }
        __syncthreads();
        if (it + 1 < iters) load(it + 1);
        const u32x4* buf = xs + (it & 1) * TM * CH + c * CH;
        union Column {
            u32x4 u;
            bf16x8 v;
        } b[2][NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) b[0][n].u = buf[n * 16 * CH + ((q * 4) ^ c)];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            // the next columns are on their way while these are used
            if (s < 3) {
#pragma unroll
                for (int n = 0; n < NT; ++n) b[(s + 1) & 1][n].u = buf[n * 16 * CH + ((q * 4 + s + 1) ^ c)];
            }
            bf16x8 wv[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) wv[i] = decode8(w[i][s], sc[i]);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < RB; ++i)
                    acc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], b[s & 1][n].v, acc[i][n], 0, 0, 0);
        }
        if (it + 1 < iters) {
#pragma unroll
            for (int j = 0; j < NT; ++j) xs[((it + 1) & 1) * TM * CH + put + j * 16 * CH] = xr[j];
        }
    }
    // lane: token 16 n + c, rows 4 q .. 4 q + 3 of each block
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (16 * n + c >= tl.z) continue;
        const int e = ent[16 * n + c];
        if constexpr (UP) {
            constexpr int NH = Pieces<F32>::N;
#pragma unroll
            for (int i = 0; i < RB / 2; ++i) {
                const int row = rb[i] * kTileRows + 4 * q;
                if (row >= a.I) continue;
                union {
                    __bf16 h[4];
                    uint2 v;
                } o[NH];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float g = acc[i][n][r], v = silu(g) * acc[i + 2][n][r];
                    if constexpr (F32) split(v, o[0].h[r], o[1].h[r]);
                    else o[0].h[r] = __bf16(v);
                }
#pragma unroll
                for (int p = 0; p < NH; ++p)
                    *reinterpret_cast<uint2*>(a.act + (size_t(e) * NH + p) * a.I + row) = o[p].v;
            }
        } else {
            const int t = e / a.ks, k = e - t * a.ks;
            const float w = k < a.K ? a.w[size_t(t) * a.K + k] : 1.f;
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                const int row = rb[i] * kTileRows + 4 * q;
                if (row >= a.H) continue;
                const f32x4 d = acc[i][n];
                const size_t at = (size_t(sp) * a.T * a.ks + e) * a.H + row;
                if constexpr (F32) {
                    *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.part) + at) =
                        make_float4(w * d[0], w * d[1], w * d[2], w * d[3]);
                } else {
                    union {
                        __bf16 b[4];
                        uint2 v;
                    } o;
#pragma unroll
                    for (int r = 0; r < 4; ++r) o.b[r] = __bf16(w * d[r]);
                    *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.part) + at) = o.v;
                }
            }
        }
    }
}

template <bool UP, int NP, int NT, bool F32>
__global__ __launch_bounds__(kThreads, 3) void mx_tile_kernel(MxArgs a, int nb) {
    constexpr int TM = 16 * NT;
    __shared__ u32x4 xs[2][TM * kTileCols / 8];
    __shared__ int ent[TM];
    // consecutive work on one XCD (workgroup i runs on XCD i % 8): the row
    // blocks of a tile and the tiles of an expert share its L2
    const int work = *a.ntiles * nb, per = (work + 7) / 8;
    const int id = int(blockIdx.x % 8) * per + int(blockIdx.x / 8);
    if (int(blockIdx.x / 8) >= per || id >= work) return;
    const int tix = id / nb, rest = id - tix * nb, sp = UP ? 0 : rest % a.tsplits, bk = UP ? rest : rest / a.tsplits;
    const int4 tl = a.tiles[tix];
    if constexpr (NT > 1) {
        // an expert's last tile, if at most half full, in half the instructions
        if (tl.z <= TM / 2) return tile_product<UP, NP, NT / 2, F32>(a, tl, bk, sp, xs[0], ent);
    }
    tile_product<UP, NP, NT, F32>(a, tl, bk, sp, xs[0], ent);
}

// y[t] = the sum of its entries' terms, in the entries' order, in fp32.  With
// bf16 y and an undivided contraction the terms are bf16 (TF false): each is
// rounded once, by 2^-8 of itself at most, as y is, which halves what the down
// launch writes and this one reads.
template <bool TF, bool YF>
__global__ __launch_bounds__(kThreads) void mx_sum_kernel(MxArgs a, int nb) {
    constexpr int V = 8;
    const int t = blockIdx.x / nb;
    const int h = ((blockIdx.x - t * nb) * kThreads + threadIdx.x) * V;
    if (h >= a.H) return;
    float s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.f;
    for (int sp = 0; sp < a.tsplits; ++sp) {
#pragma unroll 4
        for (int k = 0; k < a.ks; ++k) {
            if (entry_expert(a, t, k) < 0) continue;
            const size_t at = ((size_t(sp) * a.T + t) * a.ks + k) * a.H + h;
            if constexpr (TF) {
                const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.part) + at);
                const float4 u = p[0], v = p[1];
                s[0] += u.x; s[1] += u.y; s[2] += u.z; s[3] += u.w;
                s[4] += v.x; s[5] += v.y; s[6] += v.z; s[7] += v.w;
            } else {
                const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.part) + at);
                s[0] += bf16_lo(v.x); s[1] += bf16_hi(v.x); s[2] += bf16_lo(v.y); s[3] += bf16_hi(v.y);
                s[4] += bf16_lo(v.z); s[5] += bf16_hi(v.z); s[6] += bf16_lo(v.w); s[7] += bf16_hi(v.w);
            }
        }
    }
    if constexpr (YF) {
        float4* o = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.y) + size_t(t) * a.H + h);
        o[0] = make_float4(s[0], s[1], s[2], s[3]);
        o[1] = make_float4(s[4], s[5], s[6], s[7]);
    } else {
        union {
            __bf16 b[8];
            uint4 v;
        } o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.b[i] = __bf16(s[i]);
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.y) + size_t(t) * a.H + h) = o.v;
    }
}

// ---------------------------------------------------------------- decode steps
//
// Up to 16 tokens are the columns of one matrix instruction whatever they
// select, so each selected expert is read once, and the down projection is one
// product over the selected experts' concatenated rows: the gate weight goes
// into the activation, a wave adds a slot's product to a token that selects
// the slot, and nothing is gathered.  Both launches are bound by the weights'
// bytes; they split the contraction over the waves of a workgroup (and, down,
// over workgroups) so that every CU has enough of them in flight.

constexpr int kUnitTiles = 2;       // tiles a wave takes at a time: 2 KiB of codes and 128 scales
constexpr int kDownWaves = 8;

struct Unit {
    u32x4 c[kUnitTiles];
    uint32_t s;                     // the tiles' scale bytes
};

// Unit u of a row block whose codes and scales begin at c and s.  A missing
// last tile repeats the one before it (its columns' operands are zero).
__device__ __forceinline__ Unit load_unit(BlobRef ref, uint32_t c, uint32_t s, int u, int KT, uint32_t lane) {
    Unit r;
    const int t = u * kUnitTiles, t1 = t + 1 < KT ? t + 1 : t;
    r.c[0] = load_codes(ref, c + uint32_t(t) * kTileBytes, lane);
    r.c[1] = load_codes(ref, c + uint32_t(t1) * kTileBytes, lane);
    const uint32_t v = __builtin_amdgcn_raw_buffer_load_b16(
        ref, int(lane * 4u), int(s + uint32_t(t / kGroupTiles) * kGroupBytes + uint32_t(t % kGroupTiles)), 0);
    r.s = t1 == t ? v & 0xffu : v;
    return r;
}

template <bool XF, bool YF>
__global__ __launch_bounds__(kThreads) void mx_up_decode(MxArgs a, int nrb) {
    __shared__ uint32_t present[kMaxE / 32];
    __shared__ int entry[kMaxB * kMaxK];
    __shared__ float red[kWaves][2][4][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slot = blockIdx.x / nrb, rb = blockIdx.x % nrb;
    // the slot's expert: the slot-th of those present, then the shared ones
    if (tid < kMaxE / 32) present[tid] = 0u;
    int mine = tid < a.T * a.K ? a.idx[tid] : -1;
    if (mine >= a.E) mine = -1;
    entry[tid] = mine;
    __syncthreads();
    if (mine >= 0) atomicOr(&present[mine >> 5], 1u << (mine & 31));
    __syncthreads();
    int total = 0, g = -1;
    for (int i = 0; i < kMaxE / 32; ++i) {
        uint32_t m = __builtin_amdgcn_readfirstlane(present[i]);
        const int c = __builtin_popcount(m);
        if (slot >= total && slot < total + c) {
            for (int j = slot - total; j > 0; --j) m &= m - 1u;
            g = 32 * i + __builtin_ctz(m);
        }
        total += c;
    }
    if (blockIdx.x == 0) {
        if (tid == 0) {
            *a.nslots = total + a.ns;
            if (a.n_experts) *a.n_experts += (unsigned long long)(total);
        }
        for (int i = tid; i < row_blocks(a.H); i += kThreads) a.arrived[i] = 0;
    }
    if (g < 0) {
        if (slot - total >= a.ns) return;
        g = a.E + slot - total;
    }
    const Blob L = blob(a.H, a.I);
    const BlobRef ref = expert_blob(a, L, g);
    const int KT = col_tiles(a.H), KG = col_groups(a.H), KU = (KT + kUnitTiles - 1) / kUnitTiles;
    const uint32_t gc = uint32_t(L.gate) + uint32_t(rb * KT) * kTileBytes;
    const uint32_t uc = uint32_t(L.up) + uint32_t(rb * KT) * kTileBytes;
    const uint32_t gs = uint32_t(L.gate_s) + uint32_t(rb * KG) * kGroupBytes;
    const uint32_t us = uint32_t(L.up_s) + uint32_t(rb * KG) * kGroupBytes;
    Unit ng{}, nu{};
    if (wave < KU) {
        ng = load_unit(ref, gc, gs, wave, KT, lane);
        nu = load_unit(ref, uc, us, wave, KT, lane);
    }
    // lane: token c; its first entry that selects the expert
    const int c = lane & 15, q = lane >> 4;
    int k = kNone;
    if (c < a.T) {
        if (g >= a.E) k = a.K + g - a.E;
        else
            for (int j = a.K - 1; j >= 0; --j)
                if (entry[c * a.K + j] == g) k = j;
    }
    const bool live = k != kNone;
    if (rb == 0 && tid < kMaxB) {
        if (tid == 0) a.slots[slot].g = g;
        a.slots[slot].k[tid] = uint8_t(k);
    }
    const size_t xrow = live ? size_t(c) * a.H : 0;
    f32x4 ag = {0.f, 0.f, 0.f, 0.f}, au = {0.f, 0.f, 0.f, 0.f};
    for (int u = wave; u < KU; u += kWaves) {
        const Unit cg = ng, cu = nu;
        // the unit's columns before the next weights: loads return in order,
        // and the wait for the columns then leaves the weights in flight
        Raw<XF> xr[kUnitTiles][4];
#pragma unroll
        for (int j = 0; j < kUnitTiles; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int at = (u * kUnitTiles + j) * kTileCols + q * kBlock + s * 8;
                xr[j][s] = load_raw<XF>(a.x, xrow + at, live && at < a.H);
            }
        if (u + kWaves < KU) {
            ng = load_unit(ref, gc, gs, u + kWaves, KT, lane);
            nu = load_unit(ref, uc, us, u + kWaves, KT, lane);
        }
#pragma unroll
        for (int j = 0; j < kUnitTiles; ++j) {
            const float sg = scale_of(cg.s >> (8 * j) & 0xffu), su = scale_of(cu.s >> (8 * j) & 0xffu);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const Pieces<XF> xv = pieces(xr[j][s]);
                const bf16x8 gv = decode8(cg.c[j][s], sg), uv = decode8(cu.c[j][s], su);
#pragma unroll
                for (int p = 0; p < Pieces<XF>::N; ++p) {
                    ag = __builtin_amdgcn_mfma_f32_16x16x32_bf16(gv, xv.p[p], ag, 0, 0, 0);
                    au = __builtin_amdgcn_mfma_f32_16x16x32_bf16(uv, xv.p[p], au, 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        red[wave][0][r][lane] = ag[r];
        red[wave][1][r][lane] = au[r];
    }
    __syncthreads();
    // wave r: rows 4 q + r of the block
    float gsum = 0.f, usum = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
        gsum += red[v][0][wave][lane];
        usum += red[v][1][wave][lane];
    }
    const int row = rb * kTileRows + 4 * q + wave;
    if (!live || row >= a.I) return;
    const float w = k < a.K ? a.w[c * a.K + k] : 1.f;
    const float h = silu(gsum) * usum * w;
    constexpr int NP = Pieces<YF>::N;
    __bf16* o = reinterpret_cast<__bf16*>(a.act) + size_t(c * a.ks + k) * NP * a.I + row;
    if constexpr (YF) {
        __bf16 hi, lo;
        split(h, hi, lo);
        o[0] = hi;
        o[a.I] = lo;
    } else {
        o[0] = __bf16(h);
    }
}

// PC: up to eight tokens with two pieces each: the pieces are columns too.
template <bool YF, bool PC>
__global__ __launch_bounds__(64 * kDownWaves) void mx_down_decode(MxArgs a, int splits) {
    constexpr int NP = Pieces<YF>::N, MP = PC ? 1 : NP;     // pieces; instructions per operand
    __shared__ const void* base[kMaxE + kMaxShared];
    __shared__ uint8_t sk[kMaxE + kMaxShared][kMaxB];
    __shared__ float red[kDownWaves][4][64];
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rb = blockIdx.x / splits, sp = blockIdx.x % splits;
    const int S = *a.nslots;
    for (int s = tid; s < S; s += 64 * kDownWaves) {
        const DecodeSlot d = a.slots[s];
        base[s] = d.g < a.E ? a.eptr[d.g] : a.sptr[d.g - a.E];
#pragma unroll
        for (int t = 0; t < kMaxB; ++t) sk[s][t] = d.k[t];
    }
    __syncthreads();
    const Blob L = blob(a.H, a.I);
    const int KT = col_tiles(a.I), KG = col_groups(a.I), KU = (KT + kUnitTiles - 1) / kUnitTiles;
    const uint32_t co = uint32_t(L.down) + uint32_t(rb * KT) * kTileBytes;
    const uint32_t so = uint32_t(L.down_s) + uint32_t(rb * KG) * kGroupBytes;
    // unit u of all slots' (uniform within a wave)
    auto load = [&](int u) __attribute__((always_inline)) {
        const int s = u / KU;
        const uint64_t p = reinterpret_cast<uint64_t>(base[s]);
        const uint64_t w = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(p >> 32)))) << 32 |
                           uint32_t(__builtin_amdgcn_readfirstlane(int(p)));
        const BlobRef ref =
            __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(w), 0, int(uint32_t(L.total)), 0x00027000);
        return load_unit(ref, co, so, u - s * KU, KT, lane);
    };
    const int c = lane & 15, q = lane >> 4;
    const int t = PC ? c >> 1 : c, pc = PC ? c & 1 : 0;
    const int units = S * KU, step = splits * kDownWaves;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    Unit nx{};
    int u = sp * kDownWaves + wave;
    if (u < units) nx = load(u);
    for (; u < units; u += step) {
        const Unit cur = nx;
        const int slot = u / KU, t0 = (u - slot * KU) * kUnitTiles;
        const int k = sk[slot][t];
        const bool live = k != kNone;
        const size_t arow = live ? (size_t(t * a.ks + k) * NP + pc) * a.I : 0;
        Raw<false> h[kUnitTiles][4][MP];
#pragma unroll
        for (int j = 0; j < kUnitTiles; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int p = 0; p < MP; ++p) {
                    const int at = (t0 + j) * kTileCols + q * kBlock + s * 8;
                    h[j][s][p] = load_raw<false>(a.act, arow + size_t(p) * a.I + at, live && at < a.I);
                }
        if (u + step < units) nx = load(u + step);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kUnitTiles; ++j) {
            const float sd = scale_of(cur.s >> (8 * j) & 0xffu);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bf16x8 dv = decode8(cur.c[j][s], sd);
#pragma unroll
                for (int p = 0; p < MP; ++p)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dv, pieces(h[j][s][p]).p[0], acc, 0, 0, 0);
            }
        }
        // only to the tokens that select the slot: a NaN among its weights stays theirs
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[r] += live ? acc[r] : 0.f;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) red[wave][r][lane] = sum[r];
    __syncthreads();
    const int r = wave & 3;
    float v = 0.f;
#pragma unroll
    for (int x = 0; x < kDownWaves; ++x) v += red[x][r][lane];
    if (splits > 1) {
        // the row block's last workgroup adds the others' sums, in their order;
        // stores and loads at device scope, the count after the stores are done
        float* mine = a.split + (size_t(rb) * splits + sp) * 256;
        if (wave < 4) __hip_atomic_store(&mine[r * 64 + lane], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0)
            last = __hip_atomic_fetch_add(&a.arrived[rb], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == splits - 1;
        __syncthreads();
        if (!last || wave >= 4) return;
        v = 0.f;
        for (int x = 0; x < splits; ++x)
            v += __hip_atomic_load(&a.split[(size_t(rb) * splits + x) * 256 + r * 64 + lane], __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
    }
    if (wave >= 4) return;
    if constexpr (PC) v += __shfl_xor(v, 1, 64);
    const int row = rb * kTileRows + 4 * q + r;
    if (t >= a.T || pc || row >= a.H) return;
    if constexpr (YF) reinterpret_cast<float*>(a.y)[size_t(t) * a.H + row] = v;
    else reinterpret_cast<__bf16*>(a.y)[size_t(t) * a.H + row] = __bf16(v);
}

struct MxLayout {
    int tm, max_tiles, tsplits, slots, splits;
    size_t order, cnt, tiles, ntiles, act, part, xs, plan, nslots, arrived, split, total;
};

// Workgroups of the down launch per row block: 512 in all.
int down_splits(int H) {
    const int rb = row_blocks(H);
    return rb >= 512 ? 1 : (512 + rb - 1) / rb < 16 ? (512 + rb - 1) / rb : 16;
}

// Tokens per tile: by the tokens an expert gets on average.
int tile_tokens(int T, int K, int E) {
    const int mean = T * K / E;
    return mean > 32 ? 64 : mean > 16 ? 32 : 16;
}

// Parts of the down launch's contraction: enough for 768 workgroups (three per
// CU) if half of the experts' last tiles are filled, of four column tiles at least.
int tile_splits(int tm, size_t n, int E, int ns, int H, int I) {
    const size_t wg = (n / tm + (E + ns) / 2 + 1) * size_t((H + 255) / 256);
    const int want = wg >= 768 ? 1 : int(768 / wg), most = col_tiles(I) / 4;
    return want < 1 ? 1 : most < 1 ? 1 : want < most ? want : most;
}

MxLayout mx_layout(int T, int K, int E, int H, int I, int ns, int dtype, int ydtype) {
    MxLayout y{};
    const size_t n = size_t(T) * (K + ns);
    size_t off = 0;
    auto take = [&](size_t b) { const size_t at = off; off = (off + b + 255) / 256 * 256; return at; };
    y.act = take(n * (ydtype == STMOE_F32 ? 2 : 1) * I * sizeof(uint16_t));
    if (T <= kMaxB) {
        y.slots = (E < T * K ? E : T * K) + ns;
        y.splits = down_splits(H);
        y.plan = take(size_t(y.slots) * sizeof(DecodeSlot));
        y.nslots = take(sizeof(int32_t));
        y.arrived = take(size_t(row_blocks(H)) * sizeof(int32_t));
        y.split = take(size_t(row_blocks(H)) * y.splits * 256 * sizeof(float));
    } else {
        y.tm = tile_tokens(T, K, E);
        // a full tile takes tm entries; each expert has at most one that is not full
        const size_t most = n / y.tm + E + ns;
        y.max_tiles = int(most < n ? most : n);
        y.order = take(size_t(E + ns) * T * sizeof(int32_t));
        y.cnt = take(size_t(E + ns) * sizeof(int32_t));
        y.tiles = take(size_t(y.max_tiles) * sizeof(int4));
        y.ntiles = take(sizeof(int32_t));
        y.tsplits = tile_splits(y.tm, n, E, ns, H, I);
        y.part = take(n * y.tsplits * H * (ydtype == STMOE_F32 || y.tsplits > 1 ? 4 : 2));
        if (dtype == STMOE_F32) y.xs = take(size_t(T) * H * 2 * sizeof(uint16_t));
    }
    y.total = off;
    return y;
}

template <bool XF, bool YF>
int launch_decode(const MxArgs& a, const MxLayout& L, hipStream_t s, hipEvent_t ev_mid) {
    const int rb = row_blocks(a.I);
    hipLaunchKernelGGL((mx_up_decode<XF, YF>), dim3(unsigned(rb * L.slots)), dim3(kThreads), 0, s, a, rb);
    STMOE_LAUNCHED();
    if (ev_mid) STMOE_HIP(hipEventRecord(ev_mid, s));
    const dim3 grid(unsigned(row_blocks(a.H) * L.splits)), block(64 * kDownWaves);
    if constexpr (YF) {
        if (a.T <= kMaxB / 2) {
            hipLaunchKernelGGL((mx_down_decode<YF, true>), grid, block, 0, s, a, L.splits);
            STMOE_LAUNCHED();
            return STMOE_OK;
        }
    }
    hipLaunchKernelGGL((mx_down_decode<YF, false>), grid, block, 0, s, a, L.splits);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

template <bool XF, bool YF, int NT>
int launch_tiles(const MxArgs& a, const MxLayout& L, hipStream_t s, hipEvent_t ev_mid) {
    // rounded up to the eight XCDs
    const auto grid = [&](int nb) { return dim3(unsigned((int64_t(L.max_tiles) * nb + 7) / 8 * 8)); };
    const int ub = (a.I + 127) / 128, db = (a.H + 255) / 256 * L.tsplits;
    const int sb = (a.H + kThreads * 8 - 1) / (kThreads * 8);
    const dim3 sgrid(unsigned(a.T) * unsigned(sb)), block(kThreads);
    hipLaunchKernelGGL((mx_tile_kernel<true, XF ? 2 : 1, NT, YF>), grid(ub), block, 0, s, a, ub);
    STMOE_LAUNCHED();
    if (ev_mid) STMOE_HIP(hipEventRecord(ev_mid, s));
    if (YF || L.tsplits > 1) {
        hipLaunchKernelGGL((mx_tile_kernel<false, YF ? 2 : 1, NT, true>), grid(db), block, 0, s, a, db);
        STMOE_LAUNCHED();
        hipLaunchKernelGGL((mx_sum_kernel<true, YF>), sgrid, block, 0, s, a, sb);
    } else {
        hipLaunchKernelGGL((mx_tile_kernel<false, 1, NT, false>), grid(db), block, 0, s, a, db);
        STMOE_LAUNCHED();
        hipLaunchKernelGGL((mx_sum_kernel<false, false>), sgrid, block, 0, s, a, sb);
    }
    STMOE_LAUNCHED();
    return STMOE_OK;
}

template <bool XF, bool YF>
int launch_prompt(const MxArgs& args, const MxLayout& L, uint16_t* xs, hipStream_t s, hipEvent_t ev_mid) {
    MxArgs a = args;
    const dim3 block(kPlanThreads);
    if (a.T * a.K <= 1024) {
        if (a.K <= 8) hipLaunchKernelGGL((mx_plan_kernel<8>), dim3(1), block, 0, s, a);
        else hipLaunchKernelGGL((mx_plan_kernel<16>), dim3(1), block, 0, s, a);
    } else {
        const dim3 grid(unsigned(a.E + a.ns));
        const bool four = a.K % 4 == 0 && reinterpret_cast<uintptr_t>(a.idx) % 16 == 0;
        if (four && a.K <= 8) hipLaunchKernelGGL((mx_order_kernel<8, true>), grid, block, 0, s, a);
        else if (four) hipLaunchKernelGGL((mx_order_kernel<16, true>), grid, block, 0, s, a);
        else if (a.K <= 8) hipLaunchKernelGGL((mx_order_kernel<8, false>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((mx_order_kernel<16, false>), grid, block, 0, s, a);
        STMOE_LAUNCHED();
        hipLaunchKernelGGL(mx_tiles_kernel, dim3(1), block, 0, s, a);
    }
    STMOE_LAUNCHED();
    if constexpr (XF) {
        const int64_t n4 = int64_t(a.T) * a.H / 4, wg = (n4 + kThreads - 1) / kThreads;
        hipLaunchKernelGGL(mx_split_kernel, dim3(unsigned(wg < 8192 ? wg : 8192)), dim3(kThreads), 0, s,
                           reinterpret_cast<const float*>(a.x), n4, a.H / 4, xs);
        STMOE_LAUNCHED();
        a.x = xs;
    }
    if (L.tm == 64) return launch_tiles<XF, YF, 4>(a, L, s, ev_mid);
    if (L.tm == 32) return launch_tiles<XF, YF, 2>(a, L, s, ev_mid);
    return launch_tiles<XF, YF, 1>(a, L, s, ev_mid);
}

}  // namespace

// Internal entry of the decode-layer orchestration too (no argument checks).
// `ev_mid` is recorded between the gate/up and the down work.
int mx_ffn_launch(const void* x, const int32_t* idx, const float* w, int T, int K, int H, int I, int E, int dtype,
                  int ydtype, const void* const* eptr, const void* const* sptr, int n_shared, void* y, void* ws,
                  hipStream_t s, unsigned long long* n_experts, hipEvent_t ev_mid) {
    const MxLayout L = mx_layout(T, K, E, H, I, n_shared, dtype, ydtype);
    char* base = reinterpret_cast<char*>(ws);
    MxArgs a{};
    a.x = x;
    a.idx = idx;
    a.w = w;
    a.eptr = eptr;
    a.sptr = sptr;
    a.y = y;
    a.T = T;
    a.K = K;
    a.H = H;
    a.I = I;
    a.E = E;
    a.ns = n_shared;
    a.ks = K + n_shared;
    a.tm = L.tm;
    a.tsplits = L.tsplits;
    a.order = reinterpret_cast<int32_t*>(base + L.order);
    a.cnt = reinterpret_cast<int32_t*>(base + L.cnt);
    a.tiles = reinterpret_cast<int4*>(base + L.tiles);
    a.ntiles = reinterpret_cast<int32_t*>(base + L.ntiles);
    a.act = reinterpret_cast<uint16_t*>(base + L.act);
    a.slots = reinterpret_cast<DecodeSlot*>(base + L.plan);
    a.nslots = reinterpret_cast<int32_t*>(base + L.nslots);
    a.arrived = reinterpret_cast<int32_t*>(base + L.arrived);
    a.split = reinterpret_cast<float*>(base + L.split);
    a.part = base + L.part;
    a.n_experts = n_experts;
    const bool xf = dtype == STMOE_F32, yf = ydtype == STMOE_F32;
    if (T <= kMaxB) {
        if (xf) return yf ? launch_decode<true, true>(a, L, s, ev_mid) : launch_decode<true, false>(a, L, s, ev_mid);
        return yf ? launch_decode<false, true>(a, L, s, ev_mid) : launch_decode<false, false>(a, L, s, ev_mid);
    }
    uint16_t* xs = reinterpret_cast<uint16_t*>(base + L.xs);
    if (xf) return yf ? launch_prompt<true, true>(a, L, xs, s, ev_mid) : launch_prompt<true, false>(a, L, xs, s, ev_mid);
    return yf ? launch_prompt<false, true>(a, L, xs, s, ev_mid) : launch_prompt<false, false>(a, L, xs, s, ev_mid);
}

}  // namespace stmoe

using namespace stmoe;

extern "C" size_t moe_expert_ffn_mx_workspace_bytes(int T, int K, int E, int H, int I, int n_shared, int dtype,
                                                    int ydtype) {
    if (T < 0 || T > kMaxT || E < 1 || E > kMaxE || K < 1 || K > E || K > kMaxK || H < 8 || H % 8 || H > kMaxH ||
        I < 8 || I % 8 || I > kMaxI || n_shared < 0 || n_shared > kMaxShared)
        return 0;
    if ((dtype != STMOE_BF16 && dtype != STMOE_F32) || (ydtype != STMOE_BF16 && ydtype != STMOE_F32)) return 0;
    return mx_layout(T < 1 ? 1 : T, K, E, H, I, n_shared, dtype, ydtype).total;
}

extern "C" int moe_expert_ffn_mx(const void* x, const int32_t* topk_idx, const float* topk_w, int T, int K, int H,
                                 int I, int E, int dtype, int ydtype, const void* const* expert_ptrs,
                                 const void* const* shared_ptrs, int n_shared, void* y, void* ws, size_t ws_bytes,
                                 void* stream) {
    clear_error();
    STMOE_CHECK(T >= 0 && T <= kMaxT, "T must be in [0, 65536]");
    STMOE_CHECK(E >= 1 && E <= kMaxE, "E must be in [1, 256]");
    STMOE_CHECK(K >= 1 && K <= E && K <= kMaxK, "K must be in [1, min(E, 16)]");
    STMOE_CHECK(H >= 8 && H % 8 == 0 && H <= kMaxH, "H must be a multiple of 8 in [8, 16384]");
    STMOE_CHECK(I >= 8 && I % 8 == 0 && I <= kMaxI, "I must be a multiple of 8 in [8, 65536]");
    STMOE_CHECK(n_shared >= 0 && n_shared <= kMaxShared, "n_shared must be in [0, 8]");
    STMOE_CHECK(dtype == STMOE_BF16 || dtype == STMOE_F32, "dtype must be STMOE_BF16 or STMOE_F32");
    STMOE_CHECK(ydtype == STMOE_BF16 || ydtype == STMOE_F32, "ydtype must be STMOE_BF16 or STMOE_F32");
    if (T == 0) return STMOE_OK;
    STMOE_CHECK(x && topk_idx && topk_w && expert_ptrs && y && ws, "null pointer");
    STMOE_CHECK(n_shared == 0 || shared_ptrs, "shared_ptrs is required when n_shared > 0");
    STMOE_CHECK(ws_bytes >= moe_expert_ffn_mx_workspace_bytes(T, K, E, H, I, n_shared, dtype, ydtype),
                "workspace too small");
    STMOE_CHECK((reinterpret_cast<uintptr_t>(x) & 15) == 0 && (reinterpret_cast<uintptr_t>(y) & 15) == 0 &&
                    (reinterpret_cast<uintptr_t>(ws) & 255) == 0,
                "x and y must be 16-byte and ws 256-byte aligned");
    return mx_ffn_launch(x, topk_idx, topk_w, T, K, H, I, E, dtype, ydtype, expert_ptrs, shared_ptrs, n_shared, y, ws,
                         as_stream(stream), nullptr, nullptr);
}
