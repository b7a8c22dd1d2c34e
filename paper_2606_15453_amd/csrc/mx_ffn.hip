// Expert FFN (Section 2) over experts packed as microscaled 4-bit floats
// (mx_format.h), for one token to whole prompts:
//   y[t] = sum_k w[t][k] W_down e (silu(W_gate e x[t]) * (W_up e x[t])) + shared experts.
//
// The weights' values are exact in bf16, so both projections run on the bf16
// matrix instructions with fp32 accumulation: a lane's 16 code bytes become
// the row operand in registers, tokens are the columns.  fp32 values (x, and
// the activations when y is fp32) are split into three bf16 pieces, the
// value's rounding and twice the rounding of what is left, which hold its 24
// bits: three instructions per operand.  With bf16 y two pieces are taken of
// both: 2^-16 of themselves at most, where rounding y costs 2^-8.  (One piece of
// the activations lost as much as that rounding itself: 0.0024 of y off against
// 0.0017; with two, decode steps take up to 3% longer and 4096 tokens 19%.)
#include "mx_format.h"

namespace stmoe {
namespace {

using namespace mx;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kPlanThreads = 1024;
constexpr int kPlanEntries = 256;
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
    float* part;                    // [part][entry][H] terms of y
    // decode steps (T <= 16)
    struct DecodeSlot* slots;       // by ascending expert, the shared ones last
    int32_t* nslots;
    int smax;                       // slots at most
    float* split;                   // [chunk][4 row blocks of H][token][row] sums of the down launch
    unsigned long long* n_experts;  // counts distinct routed experts (timed decode layers), or null
};

// Pieces of an fp32 value: of x, of an activation.
template <bool XF, bool YF>
constexpr int kPiecesX = XF ? (YF ? 3 : 2) : 1;
template <bool YF>
constexpr int kPiecesH = YF ? 3 : 2;
inline size_t pieces_h(int ydtype) { return ydtype == STMOE_F32 ? kPiecesH<true> : kPiecesH<false>; }

// Column operand: eight consecutive values of a row as bf16 pieces.
template <int N>
struct Pieces {
    bf16x8 p[N];
};

// A value as N bf16 numbers; infinities and NaN (and what rounds to infinity)
// keep to the first.  The differences are those of the rounded values: fused
// with the product that gave v, they would depend on how the compiler arranged
// the caller, and a token's bits on the tile it falls into.
template <int N>
__device__ __forceinline__ void split(float v, __bf16 (&o)[N]) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        o[i] = __bf16(v);
        const float f = float(o[i]);
        v = __builtin_isfinite(f) ? v - f : 0.f;
    }
}

// Eight consecutive values as loaded.
template <bool F32>
struct Raw {
    u32x4 q[F32 ? 2 : 1];
};

__device__ __forceinline__ bf16x8 as_operand(u32x4 q) {
    union {
        u32x4 q;
        bf16x8 v;
    } u;
    u.q = q;
    return u.v;
}

template <int N>
__device__ __forceinline__ Pieces<N> pieces(const Raw<(N > 1)>& r) {
    Pieces<N> o;
    if constexpr (N == 1) {
        o.p[0] = as_operand(r.q[0]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 b[N];
            split(__uint_as_float(r.q[i / 4][i % 4]), b);
#pragma unroll
            for (int p = 0; p < N; ++p) o.p[p][i] = b[p];
        }
    }
    return o;
}

// g / (1 + exp(-g)) with the hardware's exponential and reciprocal (2^-23 of
// their values; the exponent's product rounds to 2^-24 of |g|, so silu is off
// by less than 2e-6 of itself down to g = -20 and negligible below).
__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)); }

// Which of token t's entries count, as bits (one token per wave): those that name
// an expert and are the first of the token to name it, and the shared experts'.
__device__ __forceinline__ uint32_t valid_entries(const MxArgs& a, int t) {
    const int lane = threadIdx.x & 63;
    const int e = lane < a.K ? a.idx[size_t(t) * a.K + lane] : -1;
    bool first = e >= 0 && e < a.E;
    for (int j = 0; j < a.K; ++j) first &= !((j < lane) & (__builtin_amdgcn_readlane(e, j) == e));
    return uint32_t(__ballot(first)) | ((1u << a.ns) - 1u) << a.K;
}

// A barrier for what passes through LDS alone: __syncthreads would also wait
// for the stores to memory under way (3 us for 1024 scattered ones).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Nothing that uses the values is moved before this.
template <class A, class B>
__device__ __forceinline__ void hold(A& a, B& b) { asm volatile("" : "+v"(a), "+v"(b)); }

// The tiles of at most tm tokens, experts in order (one workgroup; cnt in LDS).
__device__ __forceinline__ void list_tiles(const MxArgs& a, const int* cnt, int* tile) {
    const int tid = threadIdx.x, G = a.E + a.ns;
    if (tid < 64) {
        // running sums of the tile counts, 64 experts at a time
        int before = 0;
        for (int g0 = 0; g0 < G; g0 += 64) {
            const int g = g0 + tid, c = g < G ? cnt[g] : 0;
            int v = (c + a.tm - 1) / a.tm;
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
// a wave's place is its lanes' ballot, the waves' places meet in LDS.  Bound by
// the latency of its barriers, 1024 tokens after another, the next ones' entries
// on their way: 5.4 us for 4096 tokens and 128 experts.
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
    int before = 0, e[KU];
    // beyond K the last entry again, which does not count there
    auto load = [&](int t) __attribute__((always_inline)) {
        const int32_t* row = a.idx + size_t(min(t, a.T - 1)) * a.K;
#pragma unroll
        for (int j = 0; j < KU; j += FOUR ? 4 : 1) {
            if constexpr (FOUR) {
                const int4 v = *reinterpret_cast<const int4*>(row + min(j, a.K - 4));
                e[j] = v.x;
                e[j + 1] = v.y;
                e[j + 2] = v.z;
                e[j + 3] = v.w;
            } else {
                e[j] = row[min(j, a.K - 1)];
            }
        }
    };
    load(threadIdx.x);
    for (int t0 = 0, par = 0; t0 < a.T; t0 += kPlanThreads, par ^= 1) {
        const int t = t0 + threadIdx.x;
        int k = -1;
#pragma unroll
        for (int j = KU - 1; j >= 0; --j) k = (e[j] == g) & (j < a.K) ? j : k;
        load(t + kPlanThreads);
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

// All experts' entries and the tiles by one workgroup, a thread per token, for at
// most kPlanEntries entries: it saves a launch (whole calls against the two
// launches above: 20 tokens of top-2 16.2 and 16.8 us, 37 of top-3 27.4 and 28.0;
// beyond 300 entries it no longer did).  An expert's tokens are bits of a mask in
// LDS, a token's place the number of bits below its own; a bit that its thread
// finds set is a repeated expert.  The KU entries are handled side by side,
// without branches, so that their LDS accesses overlap; entries that name no
// expert meet words of their own.
template <int KU>
__global__ __launch_bounds__(kPlanThreads) void mx_plan_kernel(MxArgs a) {
    constexpr int W = kPlanEntries / 32;                    // words of a mask
    __shared__ uint32_t mask[kMaxE + 2][W];                 // the last two: nobody's
    __shared__ uint16_t below[kMaxE][W];
    __shared__ int cnt[kMaxGroups], tile[kMaxGroups + 1];
    const int tid = threadIdx.x, t = tid, w = min(tid >> 5, W - 1);
    const bool four = a.K % 4 == 0 && reinterpret_cast<uintptr_t>(a.idx) % 16 == 0;
    const int32_t* row = a.idx + size_t(t < a.T ? t : 0) * a.K;
    int e[KU];
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
    for (int i = tid; i < a.E * W; i += kPlanThreads) mask[0][i] = 0u;
    lds_barrier();
    uint32_t* word[KU];
    bool mine[KU];
#pragma unroll
    for (int j = 0; j < KU; ++j) {
        mine[j] = e[j] >= 0 && e[j] < a.E;
        word[j] = mine[j] ? &mask[e[j]][w] : &mask[kMaxE][tid % (2 * W)];
    }
    const uint32_t bit = 1u << (tid & 31);
    uint32_t was[KU];
#pragma unroll
    for (int j = 0; j < KU; ++j) was[j] = atomicOr(word[j], mine[j] ? bit : 0u);
#pragma unroll
    for (int j = 0; j < KU; ++j) mine[j] &= !(was[j] & bit);
    lds_barrier();
    // W lanes: an expert's words
    for (int g = tid / W; g < a.E; g += kPlanThreads / W) {
        const int l = tid % W, c = __builtin_popcount(mask[g][l]);
        int v = c;
        for (int d = 1; d < W; d <<= 1) {
            const int o = __shfl_up(v, d, W);
            if (l >= d) v += o;
        }
        below[g][l] = uint16_t(v - c);
        if (l == W - 1) cnt[g] = v;
    }
    if (tid < a.ns) cnt[a.E + tid] = a.T;
    lds_barrier();
    int at[KU], to[KU];
#pragma unroll
    for (int j = 0; j < KU; ++j) {
        const int g = mine[j] ? int(word[j] - &mask[0][0]) / W : 0;
        to[j] = g;
        at[j] = below[g][w] + __builtin_popcount(mask[g][w] & (bit - 1u));
    }
#pragma unroll
    for (int j = 0; j < KU; ++j)
        if (mine[j]) a.order[size_t(to[j]) * a.T + at[j]] = t * a.ks + j;
    if (t < a.T)
        for (int s = 0; s < a.ns; ++s) a.order[size_t(a.E + s) * a.T + t] = t * a.ks + a.K + s;
    list_tiles(a, cnt, tile);
}

// fp32 hidden states as bf16 pieces, row by row: [T][N][H].
template <int N>
__global__ __launch_bounds__(kThreads) void mx_split_kernel(const float* x, int64_t n4, int H4, uint16_t* o) {
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n4; i += int64_t(gridDim.x) * kThreads) {
        const float4 v = reinterpret_cast<const float4*>(x)[i];
        const int64_t t = i / H4, at = t * N * H4 + (i - t * H4);
        union {
            __bf16 b[4];
            uint2 q;
        } u[N];
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            __bf16 b[N];
            split(f[c], b);
#pragma unroll
            for (int p = 0; p < N; ++p) u[p].b[c] = b[p];
        }
#pragma unroll
        for (int p = 0; p < N; ++p) reinterpret_cast<uint2*>(o)[at + int64_t(p) * H4] = u[p].q;
    }
}

// A blob as a buffer: its address and size in scalar registers, a uniform
// offset and the lane's, and nothing read beyond its end.  (A load through a
// generic pointer would count as an LDS access too, and every wait for LDS
// would wait for the weights in flight.)
typedef __amdgpu_buffer_rsrc_t BlobRef;

__device__ __forceinline__ BlobRef blob_ref(const void* p, const Blob& L) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(uint32_t(L.total)), 0x00027000);
}

__device__ __forceinline__ BlobRef expert_blob(const MxArgs& a, const Blob& L, int g) {
    return blob_ref(g < a.E ? a.eptr[g] : a.sptr[g - a.E], L);
}

// ONCE: read by one workgroup only, past the caches (gate and up of
// DeepSeek-V2-Lite sizes, 16 tokens: 40.0 us through them, 34.0 past them; of
// Mixtral sizes, one token: 26.2 and 23.5).
template <bool ONCE>
__device__ __forceinline__ u32x4 load_codes(BlobRef r, uint32_t at, uint32_t lane) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, int(lane * 16u), int(at), ONCE ? 2 : 0);
}

// The scales of the group of column tiles that holds this one, and this one's.
// (As a byte it would be extended where two stages' values meet, and waited
// for there.)
__device__ __forceinline__ uint32_t load_scales(BlobRef r, uint32_t at, int tile, uint32_t lane) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, int(lane * 4u), int(at + uint32_t(tile / kGroupTiles) * kGroupBytes), 0);
}
__device__ __forceinline__ float scale_in(uint32_t group, int tile) { return scale_of(group >> 8 * (tile % kGroupTiles) & 0xffu); }

// ---------------------------------------------------------------- prompts
//
// A workgroup multiplies 256 weight rows (128 of gate and the same of up, or
// 256 of down) with a tile of up to 16 NT tokens of one expert.  Each wave
// holds 64 rows: their codes go from global memory to its registers and are
// decoded there, once for all tokens of the tile; the tokens' columns pass
// through LDS, 128 at a time, double-buffered.  A column's 256 bytes lie as 16
// chunks of eight values, chunk i in place i ^ (token % 16), so that the 16
// lanes of a read, one chunk of 16 tokens, meet 16 different places.
// Bound by the matrix instructions for many tokens (Qwen3-30B sizes, 4096 tokens,
// bf16 y, medians of a trace: up 213 us, 970 TFLOP/s, where the library's 8192^3
// product reaches 1213 on the same card; down, two pieces, 211 us, 980 TFLOP/s of
// instructions), by the weights' bytes for few (64 tokens: 210 MB in 39.5 us, 5.3
// TB/s).
// The experts' terms of y go to memory in fp32, whatever y's type: they are parts of
// its sum, and a column of y may be far smaller than the columns beside it (fp16
// terms over a power of two per 64 columns took 4096 tokens from 424 to 404 us a
// call and lost every column 2^-25 of its neighbours' size).
//
// NP: pieces of the columns, NH: of the activations (up).
template <bool UP, int NP, int NT, int NH>
__device__ __forceinline__ void tile_product(const MxArgs& a, const int4 tl, int bk, int sp, u32x4* xs, int* ent) {
    constexpr int TM = 16 * NT;
    constexpr int RB = 4;                                   // row blocks per wave
    constexpr int CH = kTileCols / 8;                       // chunks per column
    constexpr int SZ = NP * TM * CH;                        // chunks of a buffer
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
    uint32_t src[NT];                                       // in chunks of one piece
    const int chunk = tid % CH;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int e = ent[tid / CH + 16 * j];
        src[j] = uint32_t(UP ? e / a.ks : e) * uint32_t(C / 8);
    }
    const int put = tid / CH * CH + (chunk ^ (tid / CH & 15));
    struct Stage {
        u32x4 x[NP][NT], w[RB];
        uint32_t s[RB];
    } st[2];
    // Chunks beyond the row's end read its first one and are kept as zeros: their
    // codes are zero, but that times an infinity is NaN.
    auto load = [&](Stage& d, int kt) __attribute__((always_inline)) {
        const int at = kt * kTileCols + chunk * 8;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const uint32_t off = uint32_t(p * C + (at < C ? at : 0)) / 8;
#pragma unroll
            for (int j = 0; j < NT; ++j) d.x[p][j] = cols[size_t(src[j]) * NP + off];
        }
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            d.w[i] = load_codes<false>(ref, wc[i] + uint32_t(kt) * kTileBytes, lane);
            d.s[i] = load_scales(ref, wsc[i], kt, lane);
        }
    };
    f32x4 acc[RB][NT];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int c = int(lane & 15), q = int(lane >> 4);
    auto keep = [&](const Stage& d, int kt) __attribute__((always_inline)) {
        const uint32_t in = kt * kTileCols + chunk * 8 < C ? ~0u : 0u;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int j = 0; j < NT; ++j) xs[(kt & 1) * SZ + p * TM * CH + put + j * 16 * CH] = d.x[p][j] & in;
    };
    auto multiply = [&](const u32x4 (&w)[RB], const uint32_t (&scales)[RB], int kt) __attribute__((always_inline)) {
        const u32x4* buf = xs + (kt & 1) * SZ + c * CH;
        float sc[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) sc[i] = scale_in(scales[i], kt);
        bf16x8 b[2][NP][NT];
        auto fetch = [&](int s) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    b[s & 1][p][n] = as_operand(buf[p * TM * CH + n * 16 * CH + ((q * 4 + s) ^ c)]);
        };
        fetch(0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            // the next columns are on their way while these are used
            if (s < 3) fetch(s + 1);
            bf16x8 wv[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) wv[i] = decode8(w[i][s], sc[i]);
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < RB; ++i)
                        acc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i], b[s & 1][p][n], acc[i][n], 0, 0, 0);
        }
    };
    // the workgroup's share of the contraction
    const int first = UP ? 0 : KT * sp / a.tsplits, last = UP ? KT : KT * (sp + 1) / a.tsplits;
    load(st[0], first);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (NT == 1) {
        // few products per column tile: bound by the loads, two of them ahead (20
        // tokens, H 2048, I 1408, 16 experts: 29.4 us a call, 31.8 with one; with
        // 32 tokens a tile the two are equal)
        const auto step = [&](Stage& now, Stage& next, int kt) __attribute__((always_inline)) {
            lds_barrier();
            multiply(now.w, now.s, kt);
            load(now, kt + 2);
            __builtin_amdgcn_sched_barrier(0);
            keep(next, kt + 1);
        };
        load(st[1], min(first + 1, last - 1));              // (not behind a branch, see pipeline)
        __builtin_amdgcn_sched_barrier(0);
        keep(st[0], first);
        int kt = first;
        for (; kt + 3 < last; kt += 2) {
            step(st[0], st[1], kt);
            step(st[1], st[0], kt + 1);
        }
        lds_barrier();
        multiply(st[0].w, st[0].s, kt);
        if (kt + 2 < last) load(st[0], kt + 2);
        if (kt + 1 < last) {
            keep(st[1], kt + 1);
            lds_barrier();
            multiply(st[1].w, st[1].s, kt + 1);
        }
        if (kt + 2 < last) {
            keep(st[0], kt + 2);
            lds_barrier();
            multiply(st[0].w, st[0].s, kt + 2);
        }
    } else {
        keep(st[0], first);
        for (int kt = first; kt < last; ++kt) {
            u32x4 w[RB];
            uint32_t sc[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                w[i] = st[0].w[i];
                sc[i] = st[0].s[i];
            }
            lds_barrier();
            if (kt + 1 < last) load(st[0], kt + 1);
            multiply(w, sc, kt);
            if (kt + 1 < last) keep(st[0], kt + 1);
        }
    }
    // lane: token 16 n + c, rows 4 q .. 4 q + 3 of each block
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (16 * n + c >= tl.z) continue;
        const int e = ent[16 * n + c];
        if constexpr (UP) {
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
                    __bf16 b[NH];
                    split(silu(acc[i][n][r]) * acc[i + 2][n][r], b);
#pragma unroll
                    for (int p = 0; p < NH; ++p) o[p].h[r] = b[p];
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
                *reinterpret_cast<f32x4*>(a.part + (size_t(sp) * a.T * a.ks + e) * a.H + row) = w * acc[i][n];
            }
        }
    }
}

// cut: workgroups that share a tile's tokens (down).
// Three waves per SIMD (168 registers); four where they cost no spills in the loop
// and pay: 1024 tokens of top-4, tiles of 32, 85.6 us a call, 89.6 with three.
template <bool UP, int NP, int NT, int NH>
__global__ __launch_bounds__(kThreads, NP == 1 && NT == 2 ? 4 : 3) void mx_tile_kernel(MxArgs a, int nb, int cut) {
    constexpr int TM = 16 * NT;
    __shared__ u32x4 xs[2][NP * TM * kTileCols / 8];
    __shared__ int ent[TM];
    // consecutive work on one XCD (workgroup i runs on XCD i % 8): the row
    // blocks of a tile and the tiles of an expert share its L2
    const int work = *a.ntiles * nb, per = (work + 7) / 8;
    const int id = int(blockIdx.x % 8) * per + int(blockIdx.x / 8);
    if (int(blockIdx.x / 8) >= per || id >= work) return;
    const int tix = id / nb, rest = id - tix * nb, sp = UP ? 0 : rest % a.tsplits;
    int bk = UP ? rest : rest / a.tsplits;
    int4 tl = a.tiles[tix];
    if (!UP && cut > 1) {
        const int piece = bk % cut;
        bk /= cut;
        tl.y += piece * TM;
        tl.z = min(tl.z - piece * TM, TM);
        if (tl.z <= 0) return;
    }
    if constexpr (NT > 1) {
        // an expert's last tile, if at most half full, in half the instructions
        if (tl.z <= TM / 2) return tile_product<UP, NP, NT / 2, NH>(a, tl, bk, sp, xs[0], ent);
    }
    tile_product<UP, NP, NT, NH>(a, tl, bk, sp, xs[0], ent);
}

// y[t] = the sum of its entries' terms, in the entries' order, in fp32.  Bound by
// the terms' bytes (4096 tokens of top-8, H 2048: 285 MB in 44.9 us, 6.3 TB/s).
template <bool YF>
__global__ __launch_bounds__(kThreads) void mx_sum_kernel(MxArgs a, int nb) {
    constexpr int V = 8;
    const int t = blockIdx.x / nb;
    const int h = ((blockIdx.x - t * nb) * kThreads + threadIdx.x) * V;
    const uint32_t valid = valid_entries(a, t);
    if (h >= a.H) return;
    float s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.f;
    for (int sp = 0; sp < a.tsplits; ++sp) {
#pragma unroll 4
        for (int k = 0; k < a.ks; ++k) {
            // the other entries' bits cleared: a branch would keep their loads apart
            const uint32_t mask = 0u - (valid >> k & 1u);
            const size_t e = (size_t(sp) * a.T + t) * a.ks + k;
            const u32x4* p = reinterpret_cast<const u32x4*>(a.part + e * a.H + h);
            const u32x4 u = p[0] & mask, v = p[1] & mask;
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] += __uint_as_float(i < 4 ? u[i & 3] : v[i & 3]);
        }
    }
    if constexpr (YF) {
        float4* o = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.y) + size_t(t) * a.H + h);
        o[0] = make_float4(s[0], s[1], s[2], s[3]);
        o[1] = make_float4(s[4], s[5], s[6], s[7]);
    } else {
        union {
            __bf16 b[V];
            uint4 q;
        } o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.b[i] = __bf16(s[i]);
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.y) + size_t(t) * a.H + h) = o.q;
    }
}

// ---------------------------------------------------------------- decode steps
//
// Up to 16 tokens are the columns of one matrix instruction whatever they
// select, so each selected expert is read once, and the down projection is one
// product over the selected experts' concatenated rows: the gate weight goes
// into the activation, a wave adds a slot's product to a token that selects
// the slot, and nothing is gathered.
//
// Both launches are bound by the weights' bytes.  Their workgroups stay: each
// takes an equal run of the row blocks to compute, its waves share the
// contraction and keep their columns in registers, so that the loop loads
// weights alone, the next row block's while the present one's are used.
// Medians of a trace, Mixtral sizes, one token: up 125 MB in 23.4 us and down 62 MB
// in 14.0 + 4.6 (join); DeepSeek-V2-Lite sizes, 16 tokens: 161 MB in 34.2, 81 MB in
// 26.0 + 4.9 (29.4, 21.5 and 4.4 the shortest).  About 6 us of each launch pass
// before the first weights arrive (selection, pointers, weights, one after the
// other) and after the last; in between the up launch streams 7 TB/s, the down
// launch, whose waves' sums meet in LDS for every four row blocks, 5.

// A distinct expert of a decode step and, per token, the entry that selects it.
struct DecodeSlot {
    const void* blob;
    uint8_t k[kMaxB];               // kNone: the token does not select it
};
constexpr int kNone = 255;

// Rows of values as a buffer (below 2 GiB): what is not wanted is asked for
// beyond its end, which gives zeros.  Loads behind a branch inside a loop would
// make the compiler wait for every load in flight where their values meet.
__device__ __forceinline__ BlobRef rows_ref(const void* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(bytes), 0x00027000);
}

template <bool F32>
__device__ __forceinline__ Raw<F32> load_row(BlobRef rows, uint32_t at, bool in) {
    Raw<F32> r;
    const uint32_t off = in ? at * (F32 ? 4u : 2u) : 0x80000000u;
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) r.q[i] = __builtin_amdgcn_raw_buffer_load_b128(rows, int(off + 16u * i), 0, 0);
    return r;
}

// Work items lo, lo + step .. below hi (at least one), the next one's loads
// (into the other of two stages) under way while one is used.  ready(i) comes
// before the next loads, so that what it loads is waited for without them.
// Three things would make every use wait for the loads that are to overlap it:
// loads behind a branch of the loop, loads that the compiler puts off to save
// registers, and uses that it draws forward before them (pin).
template <class S, class Load, class Ready, class Use>
__device__ __forceinline__ void pipeline(S (&st)[2], int lo, int hi, int step, Load load, Ready ready, Use use) {
    const auto both = [&](S& now, S& next, int i, int s) __attribute__((always_inline)) {
        load(next, i + step);
        __builtin_amdgcn_sched_barrier(0);
        now.pin();
        use(now, i, s);
        __builtin_amdgcn_sched_barrier(0);
    };
    load(st[0], lo);
    int i = lo;
    for (; i + 2 * step < hi; i += 2 * step) {
        ready(i);
        both(st[0], st[1], i, 0);
        ready(i + step);
        both(st[1], st[0], i + step, 1);
    }
    ready(i);
    if (i + step < hi) {
        both(st[0], st[1], i, 0);
        ready(i + step);
        use(st[1], i + step, 1);
    } else {
        use(st[0], i, 0);
    }
}

// Where workgroup wg of n's equal share of the items begins (items n < 2^32: at
// most 4.4 million items of 512 workgroups).  In a scalar register, with what
// depends on it: a buffer load whose offset is not becomes a loop over lanes.
__device__ __forceinline__ int share(uint32_t items, uint32_t wg, uint32_t n) {
    return __builtin_amdgcn_readfirstlane(int(items * wg / n));
}

// The slots of a decode step in LDS: routed experts ascending, then the shared.
struct SlotTable {
    const void* blob[kMaxGroups];
    alignas(16) uint8_t k[kMaxGroups][kMaxB];
    uint32_t present[kMaxE / 32];
    int entry[kMaxB * kMaxK];

    __device__ __forceinline__ BlobRef ref(int s, const Blob& L) const {
        const uint64_t p = reinterpret_cast<uint64_t>(blob[s]);
        const uint64_t u = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(p >> 32)))) << 32 |
                           uint32_t(__builtin_amdgcn_readfirstlane(int(p)));
        return blob_ref(reinterpret_cast<const void*>(u), L);
    }
};

// Builds the table from the selection (at least 256 threads, one per entry);
// returns the number of slots.
template <int N>
__device__ __forceinline__ int make_slots(const MxArgs& a, SlotTable& tab) {
    const int tid = threadIdx.x;
    if (tid < kMaxE / 32) tab.present[tid] = 0u;
    for (int s = tid; s < kMaxGroups; s += N) *reinterpret_cast<uint4*>(tab.k[s]) = make_uint4(~0u, ~0u, ~0u, ~0u);
    int mine = tid < a.T * a.K ? a.idx[tid] : -1;
    if (mine >= a.E) mine = -1;
    const void* blob = mine >= 0 ? a.eptr[mine] : nullptr;
    if (tid < kMaxB * kMaxK) tab.entry[tid] = mine;
    lds_barrier();
    if (mine >= 0) atomicOr(&tab.present[mine >> 5], 1u << (mine & 31));
    // the first of a token's entries that names the expert
    const int t = tid / a.K, k = tid - t * a.K;
    bool first = mine >= 0;
#pragma unroll
    for (int j = 0; j < kMaxK; ++j) {
        const int e = tab.entry[min(t * a.K + j, kMaxB * kMaxK - 1)];
        first &= !((j < k) & (e == mine));
    }
    lds_barrier();
    int total = 0, at = 0;
#pragma unroll
    for (int i = 0; i < kMaxE / 32; ++i) {
        const uint32_t m = tab.present[i];
        const int below = max(0, min(32, mine - 32 * i));       // experts of this word before this one
        at += __builtin_popcount(m & uint32_t((1ull << below) - 1ull));
        total += __builtin_popcount(m);
    }
    total = __builtin_amdgcn_readfirstlane(total);
    if (first) {
        tab.blob[at] = blob;
        tab.k[at][t] = uint8_t(k);
    }
    for (int i = tid; i < a.ns * a.T; i += N) tab.k[total + i / a.T][i % a.T] = uint8_t(a.K + i / a.T);
    if (tid < a.ns) tab.blob[total + tid] = a.sptr[tid];
    lds_barrier();
    return total + a.ns;
}

// What the down launch needs, by the first workgroup.
template <int N>
__device__ __forceinline__ void publish_slots(const MxArgs& a, const SlotTable& tab, int S) {
    for (int s = threadIdx.x; s < S; s += N) {
        a.slots[s].blob = tab.blob[s];
        for (int t = 0; t < kMaxB; ++t) a.slots[s].k[t] = tab.k[s][t];
    }
    if (threadIdx.x == 0) {
        *a.nslots = S;
        if (a.n_experts) *a.n_experts += (unsigned long long)(S - a.ns);
    }
}

// A run of (slot, row block) of gate and up rows per workgroup.  Wave w holds
// the columns of the tiles from w TPW on, of every token: a token that does not
// select the slot is a column that is not stored.
template <int NH, int NW, int TPW>
__global__ __launch_bounds__(64 * NW) void mx_up_decode(MxArgs a) {
    constexpr int N = 64 * NW;
    __shared__ SlotTable tab;
    __shared__ float gate_w[kMaxB * kMaxK];
    __shared__ float red[2][NW][8][64];
    const uint32_t lane = threadIdx.x & 63;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid < a.T * a.K) gate_w[tid] = a.w[tid];
    const int KT = col_tiles(a.H), KG = col_groups(a.H), NB = row_blocks(a.I);
    const int c = int(lane & 15), q = int(lane >> 4);
    const int kt0 = wave * TPW;
    const BlobRef rows = rows_ref(a.x, uint32_t(a.T * a.H) * 2u);
    Raw<false> x[TPW][4];
#pragma unroll
    for (int j = 0; j < TPW; ++j)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int col = (kt0 + j) * kTileCols + q * kBlock + s * 8;
            x[j][s] = load_row<false>(rows, uint32_t(c * a.H + col), c < a.T && col < a.H);
        }
    const int S = make_slots<N>(a, tab);
    if (blockIdx.x == 0) publish_slots<N>(a, tab, S);
    const Blob L = blob(a.H, a.I);
    const int lo = share(S * NB, blockIdx.x, gridDim.x), hi = share(S * NB, blockIdx.x + 1, gridDim.x);
    if (lo >= hi) return;
    struct Stage {
        u32x4 w[2][TPW];
        uint32_t s[2];
        __device__ __forceinline__ void pin() {
#pragma unroll
            for (int j = 0; j < TPW; ++j) hold(w[0][j], w[1][j]);
            hold(s[0], s[1]);
        }
    } st[2];
    // A tile beyond the last one is the last one again, with columns of zeros.
    // TPW tiles never lie in two groups of scales.
    auto load = [&](Stage& d, int item) __attribute__((always_inline)) {
        const int slot = __builtin_amdgcn_readfirstlane(item / NB), rb = item - slot * NB;
        const BlobRef ref = tab.ref(slot, L);
        const uint32_t wc = uint32_t(rb * KT) * kTileBytes;
        const uint32_t sc = uint32_t(rb * KG + kt0 / kGroupTiles) * kGroupBytes;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int j = 0; j < TPW; ++j)
                d.w[m][j] = load_codes<true>(ref, uint32_t(m ? L.up : L.gate) + wc + uint32_t(min(kt0 + j, KT - 1)) * kTileBytes, lane);
            d.s[m] = __builtin_amdgcn_raw_buffer_load_b32(ref, int(lane * 4u), int(uint32_t(m ? L.up_s : L.gate_s) + sc), 0);
        }
    };
    auto multiply = [&](const Stage& d, f32x4 (&acc)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TPW; ++j)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const bf16x8 wv = decode8(d.w[m][j][s], scale_in(d.s[m], kt0 + j));
                    acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, as_operand(x[j][s].q[0]), acc[m], 0, 0, 0);
                }
            }
    };
    auto finish = [&](const f32x4 (&acc)[2], int item, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) red[buf][wave][m * 4 + r][lane] = acc[m][r];
        lds_barrier();
        if (wave >= 4) return;
        // wave r: rows 4 q + r of the block
        float gsum = 0.f, usum = 0.f;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            gsum += red[buf][v][wave][lane];
            usum += red[buf][v][4 + wave][lane];
        }
        const int slot = item / NB, row = (item - slot * NB) * kTileRows + 4 * q + wave, k = tab.k[slot][c];
        if (k == kNone || row >= a.I) return;
        const float w = k < a.K ? gate_w[c * a.K + k] : 1.f;
        __bf16 b[NH];
        split(silu(gsum) * usum * w, b);
        __bf16* o = reinterpret_cast<__bf16*>(a.act) + size_t(c * a.ks + k) * NH * a.I + row;
#pragma unroll
        for (int p = 0; p < NH; ++p) o[size_t(p) * a.I] = b[p];
    };
    // waves without columns add zeros
    if (kt0 >= KT) {
        const f32x4 none[2] = {};
        for (int item = lo; item < hi; ++item) finish(none, item, (item - lo) & 1);
        return;
    }
    pipeline(
        st, lo, hi, 1, load, [](int) {},
        [&](const Stage& d, int item, int buf) __attribute__((always_inline)) {
            f32x4 acc[2] = {};
            multiply(d, acc);
            finish(acc, item, buf);
        });
}

// fp32 hidden states, or more than 32 column tiles: a row block of one expert
// per workgroup, whose four waves take every fourth tile and load its columns
// with it, of the tokens that select the expert.
template <int NX, int NH>
__global__ __launch_bounds__(kThreads) void mx_up_wide(MxArgs a, int nrb) {
    __shared__ SlotTable tab;
    __shared__ float red[kWaves][8][64];
    const uint32_t lane = threadIdx.x & 63;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slot = blockIdx.x / nrb, rb = int(blockIdx.x % nrb);
    const int S = make_slots<kThreads>(a, tab);
    if (blockIdx.x == 0) publish_slots<kThreads>(a, tab, S);
    if (slot >= S) return;
    const Blob L = blob(a.H, a.I);
    const BlobRef ref = tab.ref(slot, L);
    const int KT = col_tiles(a.H), KG = col_groups(a.H);
    const int c = int(lane & 15), q = int(lane >> 4), k = tab.k[slot][c];
    const bool live = k != kNone;
    const BlobRef rows = rows_ref(a.x, uint32_t(a.T * a.H) * (NX > 1 ? 4u : 2u));
    const uint32_t wc = uint32_t(rb * KT) * kTileBytes, sc = uint32_t(rb * KG) * kGroupBytes;
    struct Stage {
        u32x4 w[2];
        uint32_t s[2];
        Raw<(NX > 1)> x[4];
        __device__ __forceinline__ void pin() {
            hold(w[0], w[1]);
            hold(s[0], s[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                hold(x[2 * i].q[0], x[2 * i + 1].q[0]);
                if constexpr (NX > 1) hold(x[2 * i].q[1], x[2 * i + 1].q[1]);
            }
        }
    } st[2];
    auto load = [&](Stage& d, int kt) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            d.w[m] = load_codes<true>(ref, uint32_t(m ? L.up : L.gate) + wc + uint32_t(kt) * kTileBytes, lane);
            d.s[m] = load_scales(ref, uint32_t(m ? L.up_s : L.gate_s) + sc, kt, lane);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int col = kt * kTileCols + q * kBlock + s * 8;
            d.x[s] = load_row<(NX > 1)>(rows, uint32_t(c * a.H + col), live && col < a.H);
        }
    };
    f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
    auto use = [&](const Stage& d, int kt, int) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const Pieces<NX> xv = pieces<NX>(d.x[s]);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const bf16x8 wv = decode8(d.w[m][s], scale_in(d.s[m], kt));
#pragma unroll
                for (int p = 0; p < NX; ++p)
                    acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xv.p[p], acc[m], 0, 0, 0);
            }
        }
    };
    if (wave < KT) pipeline(st, wave, KT, kWaves, load, [](int) {}, use);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave][m * 4 + r][lane] = acc[m][r];
    lds_barrier();
    // wave r: rows 4 q + r of the block
    float gsum = 0.f, usum = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
        gsum += red[v][wave][lane];
        usum += red[v][4 + wave][lane];
    }
    const int row = rb * kTileRows + 4 * q + wave;
    if (!live || row >= a.I) return;
    const float w = k < a.K ? a.w[c * a.K + k] : 1.f;
    __bf16 b[NH];
    split(silu(gsum) * usum * w, b);
    __bf16* o = reinterpret_cast<__bf16*>(a.act) + size_t(c * a.ks + k) * NH * a.I + row;
#pragma unroll
    for (int p = 0; p < NH; ++p) o[size_t(p) * a.I] = b[p];
}

// A run of (chunk of column tiles, group of R row blocks) of the down rows per
// workgroup.  A chunk is NW U tiles of the selected experts' concatenated
// rows, U per wave, whose activations the wave holds while it goes through the
// row blocks.  With one chunk the sums are y, else the chunks' sums go to the
// join launch.  PC: few tokens, whose pieces are columns too.
// (Four waves per SIMD: with 142 registers for three pieces only one workgroup
// would fit a CU.)
template <int NH, bool PC, bool YF, int NW, int U, int R>
__global__ __launch_bounds__(64 * NW, 4) void mx_down_decode(MxArgs a, int direct) {
    constexpr int MP = PC ? 1 : NH;                         // instructions per operand
    constexpr int N = 64 * NW, OUT = R * 256;
    constexpr int PER = ((PC ? kMaxB / NH : kMaxB) * R * kTileRows + N - 1) / N;
    __shared__ SlotTable tab;
    __shared__ float red[2][NW][OUT];
    const uint32_t lane = threadIdx.x & 63;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int S = *a.nslots;
    for (int s = tid; s < a.smax; s += N) {
        const DecodeSlot d = a.slots[s];
        tab.blob[s] = d.blob;
#pragma unroll
        for (int t = 0; t < kMaxB; ++t) tab.k[s][t] = d.k[t];
    }
    lds_barrier();
    const Blob L = blob(a.H, a.I);
    const int KT = col_tiles(a.I), KG = col_groups(a.I), NB = row_blocks(a.H), groups = (NB + R - 1) / R;
    const int units = S * KT, chunks = max(1, (units + NW * U - 1) / (NW * U));
    const int lo = share(chunks * groups, blockIdx.x, gridDim.x), hi = share(chunks * groups, blockIdx.x + 1, gridDim.x);
    if (lo >= hi) return;
    const int c = int(lane & 15), q = int(lane >> 4);
    const int t = PC ? c / NH : c, pc = PC ? c % NH : 0;
    struct Stage {
        u32x4 w[U][R];
        uint32_t s[U][R];
        int kt[U];
        __device__ __forceinline__ void pin() {
#pragma unroll
            for (int i = 0; i < U * R; ++i) hold(w[i / R][i % R], s[i / R][i % R]);
        }
    } st[2];
    auto load = [&](Stage& d, int item) __attribute__((always_inline)) {
        const int chunk = __builtin_amdgcn_readfirstlane(item / groups), grp = item - chunk * groups;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            // beyond the last tile: no loads where there is one item mostly,
            // else the last one again, which no token adds
            int u = (chunk * NW + wave) * U + j;
            if (U > 1 && u >= units) continue;
            u = min(u, units - 1);
            const int slot = __builtin_amdgcn_readfirstlane(u / KT), kt = u - slot * KT;
            const BlobRef ref = tab.ref(slot, L);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const uint32_t b = uint32_t(min(grp * R + i, NB - 1));
                d.w[j][i] = load_codes<true>(ref, uint32_t(L.down) + (b * uint32_t(KT) + uint32_t(kt)) * kTileBytes, lane);
                d.s[j][i] = load_scales(ref, uint32_t(L.down_s) + b * uint32_t(KG) * kGroupBytes, kt, lane);
            }
            d.kt[j] = kt;
        }
    };
    const BlobRef rows = rows_ref(a.act, uint32_t(a.T * a.ks * NH) * uint32_t(a.I) * 2u);
    Raw<false> h[U][4][MP];
    bool live[U];
    auto columns = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = (chunk * NW + wave) * U + j, slot = u / KT, kt = u - slot * KT;
            const int k = u < units ? tab.k[slot][t] : kNone;
            live[j] = k != kNone;
            const uint32_t row = uint32_t((t * a.ks + k) * NH + pc) * uint32_t(a.I);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int col = kt * kTileCols + q * kBlock + x * 8;
#pragma unroll
                for (int y = 0; y < MP; ++y)
                    h[j][x][y] = load_row<false>(rows, row + uint32_t(y * a.I + col), live[j] && col < a.I);
            }
        }
    };
    // Where a sum is put (chunks): the columns of a row permuted by row and row
    // block, so that half a wave meets 32 banks both here, where it has two rows of
    // 16 columns, and in finish, where it has 16 rows of two row blocks.
    const int put = U > 1 ? int(lane) : int(lane) ^ (int(lane) >> 5) << 1;
    auto multiply = [&](const Stage& d, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < U; ++j) {
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const bf16x8 wv = decode8(d.w[j][i][x], scale_in(d.s[j][i], d.kt[j]));
#pragma unroll
                    for (int y = 0; y < MP; ++y)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, as_operand(h[j][x][y].q[0]), acc, 0, 0, 0);
                }
                // only to the tokens that select the slot: a NaN among its weights stays theirs
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] += live[j] ? acc[r] : 0.f;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) red[buf][wave][i * 256 + r * 64 + (put ^ (U > 1 ? 0 : r * 4 + (i & 1)))] = sum[r];
        }
    };
    // the sums of the waves, and of a token's pieces
    auto finish = [&](int item, int buf) __attribute__((always_inline)) {
        lds_barrier();
        const auto store = [&](int tok, int row, float v) __attribute__((always_inline)) {
            if constexpr (YF) reinterpret_cast<float*>(a.y)[size_t(tok) * a.H + row] = v;
            else reinterpret_cast<__bf16*>(a.y)[size_t(tok) * a.H + row] = __bf16(v);
        };
        if constexpr (U > 1) {
            // one row block, a thread per row and column
            static_assert(PC && (NH == 2 || NH == 3), "a token's pieces are two or three columns");
            if (tid >= OUT) return;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) v += red[buf][w][tid];
            float more = __shfl_down(v, 1, 64);
            if constexpr (NH == 3) more += __shfl_down(v, 2, 64);
            v += more;
            const int row = item * kTileRows + 4 * q + tid / 64;
            if (t < a.T && !pc && row < a.H) store(t, row, v);
            return;
        }
        // [token][row block][row]: of the tokens that are there, so that few of them
        // have few sums to write and to join (Mixtral sizes, one token: the down
        // launch at its shortest 15.5 us with all 16 columns' sums, 13.8 with these)
        float v[PER];
#pragma unroll
        for (int z = 0; z < PER; ++z) {
            const int o = tid + z * N, row = o % kTileRows, i = o / kTileRows % R, tok = o / (R * kTileRows);
            v[z] = 0.f;
            if (tok >= a.T) break;
            const float* p = &red[buf][0][i * 256 + row % 4 * 64 + row / 4 * 16];
            const int to = row % 4 * 4 + row / 8 * 2 + (i & 1);
#pragma unroll
            for (int x = 0; x < (PC ? NH : 1); ++x)
#pragma unroll
                for (int w = 0; w < NW; ++w) v[z] += p[w * OUT + ((PC ? NH * tok + x : tok) ^ to)];
        }
#pragma unroll
        for (int z = 0; z < PER; ++z) {
            const int o = tid + z * N, row = (item * R + o / kTileRows % R) * kTileRows + o % kTileRows;
            const int tok = o / (R * kTileRows);
            if (tok >= a.T) break;
            if (!direct) a.split[size_t(item) * (a.T * R * kTileRows) + o] = v[z];
            else if (row < a.H) store(tok, row, v[z]);
        }
    };
    if (units == 0) {
        // nothing selected: the sums are zero
#pragma unroll
        for (int o = tid; o < NW * OUT; o += N) red[0][o / OUT][o % OUT] = 0.f;
        for (int item = lo; item < hi; ++item) finish(item, 0);
        return;
    }
    const auto use = [&](const Stage& d, int item, int buf) __attribute__((always_inline)) {
        multiply(d, buf);
        finish(item, buf);
    };
    if constexpr (U > 1) {
        // one chunk, and one item up to H 4096
        columns(0);
        for (int item = lo; item < hi; ++item) {
            load(st[0], item);
            use(st[0], item, (item - lo) & 1);
        }
    } else {
        int held = -1;                                      // the chunk whose columns are held
        pipeline(
            st, lo, hi, 1, load,
            [&](int item) __attribute__((always_inline)) {
                const int chunk = item / groups;
                if (chunk != held) columns(held = chunk);
            },
            use);
    }
}

// y from the chunks' sums, in their order: 256 of a chunk's sums per workgroup,
// four threads each.
template <bool YF, int TILES, int R>
__global__ __launch_bounds__(1024) void mx_join_kernel(MxArgs a) {
    __shared__ float red[4][256];
    const int tid = threadIdx.x, o = int(blockIdx.x) * 256 + (tid & 255), part = tid >> 8;
    const int groups = (row_blocks(a.H) + R - 1) / R, units = *a.nslots * col_tiles(a.I);
    const int chunks = max(1, (units + TILES - 1) / TILES), n = groups * R * kTileRows * a.T;
    float v = 0.f;
    if (o < n) {
#pragma unroll 8
        for (int x = part; x < chunks; x += 4) v += a.split[size_t(x) * n + o];
    }
    red[part][tid & 255] = v;
    __syncthreads();
    const int t = o / (R * kTileRows) % a.T, row = (o / (R * kTileRows * a.T) * R + o / kTileRows % R) * kTileRows + o % kTileRows;
    if (part || o >= n || row >= a.H) return;
    const float s = (red[0][tid] + red[1][tid]) + (red[2][tid] + red[3][tid]);
    if constexpr (YF) reinterpret_cast<float*>(a.y)[size_t(t) * a.H + row] = s;
    else reinterpret_cast<__bf16*>(a.y)[size_t(t) * a.H + row] = __bf16(s);
}

// The down launch's forms: pieces as columns and up to 48 column tiles, which is
// what sixteen waves hold in registers, in one chunk, whose sums are y (at that
// border, one token, H 2048, I 768, top 8: a call 12.9 us, 13.7 with chunks; H
// 4096, I 1408, top 4, bf16 y: 16.8 and 18.3), else chunks of eight tiles (two row
// blocks at a time, or four waves: up to 10% slower; sixteen waves: within 3%).
constexpr int kOneWaves = 16, kOneU = 3, kOneR = 1;
constexpr int kRunWaves = 8, kRunU = 1, kRunR = 4;

struct MxLayout {
    int tm, max_tiles, tsplits, slots, units;
    size_t order, cnt, tiles, ntiles, act, part, xs, plan, nslots, split, total;
};

// Tokens per tile: 64 where an expert gets more than 32 on average, both x and
// y are bf16 and that leaves 1536 workgroups of the up launch (two rounds of
// three per CU); else 32 above 12 on average, else 16.  Measured in us with
// tiles of 16, 32 and 64 (H 2048, I 768, 64 experts, top 4 unless said):
//    128 tokens   41    41    45       512 tokens   59    63    68
//    256          49    49    52      2048         152   137   148  (960 workgroups)
//   4096, 128 experts, top 8, bf16:   472 with 32, 463 with 64; fp32: 862, 803, 890
//    512, H 4096, I 14336, 8 experts, top 2, bf16:  663 with 32, 531 with 64
// 12 is where 32 gets ahead with large experts (64 tokens of the last shape 201 and
// 171 us); with small ones 16 stays ahead until about 40 (160 fp32 tokens, H 1000, I
// 520, top 3 of 13: 30 and 40 us).
int tile_tokens(int T, int K, int E, int ns, int I, bool bf16) {
    const int mean = T * K / E;
    const int64_t wg = (int64_t(T) * (K + ns) / 64 + (E + ns) / 2) * ((I + 127) / 128);
    return mean > 32 && bf16 && wg >= 1536 ? 64 : mean > 12 ? 32 : 16;
}

// Parts of the down launch's contraction: enough for 768 workgroups (three per
// CU) if half of the experts' last tiles are filled, of four column tiles at
// least (32 tokens, H 1024, I 8192, 8 experts: 74 us unsplit, 44 split; 20
// tokens, H 2048, I 1408, 16 experts: 32 and 29).
constexpr size_t kDownWgs = 768;
int most_splits(int I) { return col_tiles(I) < 8 ? 1 : col_tiles(I) / 4; }
int tile_splits(int tm, size_t n, int E, int ns, int H, int I) {
    const size_t wg = (n / tm + (E + ns) / 2 + 1) * size_t((H + 255) / 256);
    const int want = wg >= kDownWgs ? 1 : int(kDownWgs / wg), most = most_splits(I);
    return want < most ? want : most;
}

// Rows of terms for n entries: n times tile_splits, or what fewer entries in more
// parts need.  With floor(n / tm) >= (n + 1) / tm - 1 the parts are at most
// 768 tm / ((n + 1 + (E + ns) / 2 tm) H / 256), and that times n grows with n.
size_t term_rows(int tm, size_t n, int E, int ns, int H, int I) {
    const size_t den = (n + 1 + size_t((E + ns) / 2) * tm) * size_t((H + 255) / 256);
    const size_t parts = (kDownWgs * tm * n + den - 1) / den, most = n * most_splits(I);
    return parts < n ? n : parts < most ? parts : most;
}

// Its bytes grow with T (a workspace for many tokens serves fewer): a prompt's are
// those of 16 tokens at least, and its parts are sized for the largest number of
// tokens up to T that needs most.
MxLayout mx_layout(int T, int K, int E, int H, int I, int ns, int dtype, int ydtype) {
    MxLayout y{};
    const size_t n = size_t(T) * (K + ns);
    size_t off = 0;
    auto take = [&](size_t b) { const size_t at = off; off = (off + b + 255) / 256 * 256; return at; };
    y.act = take(n * pieces_h(ydtype) * I * sizeof(uint16_t));
    if (T <= kMaxB) {
        y.slots = (E < T * K ? E : T * K) + ns;
        y.units = y.slots * col_tiles(I);
        y.plan = take(size_t(y.slots) * sizeof(DecodeSlot));
        y.nslots = take(sizeof(int32_t));
        const size_t chunks = (size_t(y.units) + kRunWaves * kRunU - 1) / (kRunWaves * kRunU);
        y.split = take(chunks * ((row_blocks(H) + kRunR - 1) / kRunR * kRunR) * kTileRows * T * sizeof(float));
    } else {
        y.tm = tile_tokens(T, K, E, ns, I, dtype == STMOE_BF16 && ydtype == STMOE_BF16);
        // a full tile takes tm entries; each expert has at most one that is not full
        const size_t most = n / y.tm + E + ns;
        y.max_tiles = int(most < n ? most : n);
        y.order = take(size_t(E + ns) * T * sizeof(int32_t));
        y.cnt = take(size_t(E + ns) * sizeof(int32_t));
        const size_t small = n / 16 + E + ns;               // tiles of 16 tokens
        y.tiles = take((small < n ? small : n) * sizeof(int4));
        y.ntiles = take(sizeof(int32_t));
        y.tsplits = tile_splits(y.tm, n, E, ns, H, I);
        y.part = take(term_rows(y.tm, n, E, ns, H, I) * H * sizeof(float));
        if (dtype == STMOE_F32) y.xs = take(size_t(T) * H * (ydtype == STMOE_F32 ? 3 : 2) * sizeof(uint16_t));
    }
    const size_t step = T <= kMaxB ? 0 : mx_layout(kMaxB, K, E, H, I, ns, dtype, ydtype).total;
    y.total = off > step ? off : step;
    return y;
}

// Row blocks in turn with the columns in registers, for bf16 x of up to 32 column
// tiles, which is what eight waves of four hold (16 tokens of top-8 of 64, I 1536,
// whole calls: H 512 31.7 us, 40.1 with mx_up_wide; 1024 44.1 and 49.8; 2048 65.6
// and 71.6; 4096 113 and 117; one token the same with both).  Four waves take 1, 2 or 4 tiles each (with 4 throughout H
// 512 34.6 us, 1024 45.3), eight 4; as many workgroups as stay side by side on the
// 256 CUs, but up to 1024 row blocks of four waves one each (one token, H 2048, I
// 1536: 18.0 us, 19.4 on 512).
template <int NX, int NH>
void launch_up_decode(const MxArgs& a, const MxLayout& L, hipStream_t s) {
    const int KT = col_tiles(a.H), NB = row_blocks(a.I);
    const int64_t items = int64_t(L.slots) * NB;
    const auto grid = [&](int most) { return dim3(unsigned(items < most ? items : most)); };
    if (NX > 1 || KT > 32) hipLaunchKernelGGL((mx_up_wide<NX, NH>), dim3(unsigned(items)), dim3(kThreads), 0, s, a, NB);
    else if (KT <= 4) hipLaunchKernelGGL((mx_up_decode<NH, 4, 1>), grid(1024), dim3(256), 0, s, a);
    else if (KT <= 8) hipLaunchKernelGGL((mx_up_decode<NH, 4, 2>), grid(1024), dim3(256), 0, s, a);
    else if (KT <= 16) hipLaunchKernelGGL((mx_up_decode<NH, 4, 4>), grid(items <= 1024 ? 1024 : 512), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((mx_up_decode<NH, 8, 4>), grid(256), dim3(512), 0, s, a);
}

template <int NH, bool PC, bool YF>
int launch_down_decode(const MxArgs& a, const MxLayout& L, hipStream_t s) {
    const int NB = row_blocks(a.H);
    if constexpr (PC) {
        if (L.units <= kOneWaves * kOneU) {
            hipLaunchKernelGGL((mx_down_decode<NH, PC, YF, kOneWaves, kOneU, kOneR>), dim3(unsigned(NB < 256 ? NB : 256)),
                               dim3(64 * kOneWaves), 0, s, a, 1);
            STMOE_LAUNCHED();
            return STMOE_OK;
        }
    }
    const int64_t chunks = (L.units + kRunWaves * kRunU - 1) / (kRunWaves * kRunU);
    const int64_t work = chunks * ((NB + kRunR - 1) / kRunR);
    hipLaunchKernelGGL((mx_down_decode<NH, PC, YF, kRunWaves, kRunU, kRunR>), dim3(unsigned(work < 512 ? work : 512)),
                       dim3(64 * kRunWaves), 0, s, a, chunks == 1);
    STMOE_LAUNCHED();
    if (chunks > 1) {
        const int64_t sums = int64_t((NB + kRunR - 1) / kRunR * kRunR) * kTileRows * a.T;
        hipLaunchKernelGGL((mx_join_kernel<YF, kRunWaves * kRunU, kRunR>), dim3(unsigned((sums + 255) / 256)), dim3(1024), 0, s, a);
        STMOE_LAUNCHED();
    }
    return STMOE_OK;
}

template <bool XF, bool YF>
int launch_decode(const MxArgs& a, const MxLayout& L, hipStream_t s, hipEvent_t ev_mid) {
    constexpr int NX = kPiecesX<XF, YF>, NH = kPiecesH<YF>;
    launch_up_decode<NX, NH>(a, L, s);
    STMOE_LAUNCHED();
    if (ev_mid) STMOE_HIP(hipEventRecord(ev_mid, s));
    // few tokens (up to five of fp32 y, eight of bf16) have the pieces of a column as
    // columns of one instruction (one token, H 2048, I 768, top 8, fp32 y: a call 13.1
    // us, 14.8 with three instructions; five tokens 27.8 and 29.9; eight of bf16 y, H
    // 2048, I 128, top 6: 13.0 and 14.3)
    if (a.T * NH <= kMaxB) return launch_down_decode<NH, true, YF>(a, L, s);
    return launch_down_decode<NH, false, YF>(a, L, s);
}

template <bool XF, bool YF, int NT>
int launch_tiles(const MxArgs& a, const MxLayout& L, hipStream_t s) {
    // rounded up to the eight XCDs
    const auto grid = [&](int nb) { return dim3(unsigned((int64_t(L.max_tiles) * nb + 7) / 8 * 8)); };
    const int ub = (a.I + 127) / 128, db = (a.H + 255) / 256 * L.tsplits;
    const int sb = (a.H + kThreads * 8 - 1) / (kThreads * 8);
    const dim3 sgrid(unsigned(a.T) * unsigned(sb)), block(kThreads);
    constexpr int NH = kPiecesH<YF>;
    hipLaunchKernelGGL((mx_tile_kernel<true, kPiecesX<XF, YF>, NT, NH>), grid(ub), block, 0, s, a, ub, 1);
    STMOE_LAUNCHED();
    // tiles of 64 tokens in two halves: both pieces of 64 columns would leave two
    // workgroups a CU (4096 tokens of top-8 507 us a call, 519 whole; 512 tokens of
    // Mixtral sizes 539 and 572)
    constexpr int DT = NT == 4 ? 2 : NT, CUT = NT / DT;
    hipLaunchKernelGGL((mx_tile_kernel<false, NH, DT, NH>), grid(db * CUT), block, 0, s, a, db * CUT, CUT);
    STMOE_LAUNCHED();
    hipLaunchKernelGGL((mx_sum_kernel<YF>), sgrid, block, 0, s, a, sb);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

template <bool XF, bool YF>
int launch_prompt(const MxArgs& args, const MxLayout& L, uint16_t* xs, hipStream_t s) {
    MxArgs a = args;
    const dim3 block(kPlanThreads);
    if (a.T * a.K <= kPlanEntries) {
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
        hipLaunchKernelGGL((mx_split_kernel<kPiecesX<XF, YF>>), dim3(unsigned(wg < 8192 ? wg : 8192)), dim3(kThreads), 0, s,
                           reinterpret_cast<const float*>(a.x), n4, a.H / 4, xs);
        STMOE_LAUNCHED();
        a.x = xs;
    }
    if constexpr (!XF && !YF) {
        if (L.tm == 64) return launch_tiles<XF, YF, 4>(a, L, s);
    }
    if (L.tm == 32) return launch_tiles<XF, YF, 2>(a, L, s);
    return launch_tiles<XF, YF, 1>(a, L, s);
}

// The launches count a piece of the activations in 16-byte chunks of 32 bits; three
// pieces are held to the same bytes.
bool too_large(int T, int K, int I, int ns, int ydtype) {
    return size_t(T) * (K + ns) * (ydtype == STMOE_F32 ? 3 : 1) * I / 8 > size_t(1) << 32;
}

}  // namespace

// Internal entry of the decode-layer orchestration too (no argument checks).
// `n_experts` and `ev_mid` (recorded between the gate/up and the down work) are for
// decode steps, T <= kMaxB; a prompt ignores them.
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
    a.smax = L.slots;
    a.split = reinterpret_cast<float*>(base + L.split);
    a.part = reinterpret_cast<float*>(base + L.part);
    a.n_experts = n_experts;
    const bool xf = dtype == STMOE_F32, yf = ydtype == STMOE_F32;
    if (T <= kMaxB) {
        if (xf) return yf ? launch_decode<true, true>(a, L, s, ev_mid) : launch_decode<true, false>(a, L, s, ev_mid);
        return yf ? launch_decode<false, true>(a, L, s, ev_mid) : launch_decode<false, false>(a, L, s, ev_mid);
    }
    uint16_t* xs = reinterpret_cast<uint16_t*>(base + L.xs);
    if (xf) return yf ? launch_prompt<true, true>(a, L, xs, s) : launch_prompt<true, false>(a, L, xs, s);
    return yf ? launch_prompt<false, true>(a, L, xs, s) : launch_prompt<false, false>(a, L, xs, s);
}

}  // namespace stmoe

using namespace stmoe;

extern "C" size_t moe_expert_ffn_mx_workspace_bytes(int T, int K, int E, int H, int I, int n_shared, int dtype,
                                                    int ydtype) {
    if (T < 0 || T > kMaxT || E < 1 || E > kMaxE || K < 1 || K > E || K > kMaxK || H < 8 || H % 8 || H > kMaxH ||
        I < 8 || I % 8 || I > kMaxI || n_shared < 0 || n_shared > kMaxShared)
        return 0;
    if ((dtype != STMOE_BF16 && dtype != STMOE_F32) || (ydtype != STMOE_BF16 && ydtype != STMOE_F32)) return 0;
    if (too_large(T, K, I, n_shared, ydtype)) return 0;
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
    STMOE_CHECK(!too_large(T, K, I, n_shared, ydtype), "the tokens' activations exceed 64 GiB");
    STMOE_CHECK(x && topk_idx && topk_w && expert_ptrs && y && ws, "null pointer");
    STMOE_CHECK(n_shared == 0 || shared_ptrs, "shared_ptrs is required when n_shared > 0");
    STMOE_CHECK(ws_bytes >= moe_expert_ffn_mx_workspace_bytes(T, K, E, H, I, n_shared, dtype, ydtype),
                "workspace too small");
    STMOE_CHECK((reinterpret_cast<uintptr_t>(x) & 15) == 0 && (reinterpret_cast<uintptr_t>(y) & 15) == 0 &&
                    (reinterpret_cast<uintptr_t>(ws) & 255) == 0,
                "x and y must be 16-byte and ws 256-byte aligned");
    STMOE_CHECK((reinterpret_cast<uintptr_t>(topk_idx) & 3) == 0 && (reinterpret_cast<uintptr_t>(topk_w) & 3) == 0 &&
                    (reinterpret_cast<uintptr_t>(expert_ptrs) & 7) == 0 && (reinterpret_cast<uintptr_t>(shared_ptrs) & 7) == 0,
                "topk_idx, topk_w and the pointer arrays must be aligned to their elements");
    return mx_ffn_launch(x, topk_idx, topk_w, T, K, H, I, E, dtype, ydtype, expert_ptrs, shared_ptrs, n_shared, y, ws,
                         as_stream(stream), nullptr, nullptr);
}
