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
    // workspace
    int32_t* order;                 // [T * ks] entries (t * ks + k) by expert
    int4* tiles;                    // (expert, first position, tokens, -)
    int32_t* ntiles;
    uint16_t* act;                  // [position][piece][I] bf16 pieces
    float* part;                    // [entry][H]
    unsigned long long* n_experts;  // counts distinct routed experts (timed decode layers), or null
};

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
// infinity) keep to the first.
__device__ __forceinline__ void split(float v, __bf16& hi, __bf16& lo) {
    hi = __bf16(v);
    const float h = float(hi);
    lo = __builtin_isfinite(h) ? __bf16(v - h) : __bf16(0.f);
}

template <bool F32>
__device__ __forceinline__ Pieces<F32> load8(const void* x, size_t at, bool in) {
    Pieces<F32> r;
    if constexpr (!F32) {
        union {
            uint4 q;
            bf16x8 v;
        } u;
        u.q = in ? *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(x) + at) : make_uint4(0, 0, 0, 0);
        r.p[0] = u.v;
    } else {
        float v[8];
        const float* s = reinterpret_cast<const float*>(x) + at;
        const float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 a = in ? *reinterpret_cast<const float4*>(s) : z, b = in ? *reinterpret_cast<const float4*>(s + 4) : z;
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 h, l;
            split(v[i], h, l);
            r.p[0][i] = h;
            r.p[1][i] = l;
        }
    }
    return r;
}

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

// Entries by expert and the tiles of at most tm tokens: one workgroup.  The
// order within an expert is that of the atomics; a token's results do not
// depend on its place.
__global__ __launch_bounds__(kPlanThreads) void mx_plan_kernel(MxArgs a) {
    __shared__ int cnt[kMaxGroups], base[kMaxGroups], tile[kMaxGroups];
    const int G = a.E + a.ns, n = a.T * a.ks;
    for (int g = threadIdx.x; g < G; g += kPlanThreads) cnt[g] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int e = entry_expert(a, i / a.ks, i % a.ks);
        if (e >= 0) atomicAdd(&cnt[e], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int at = 0, nt = 0, used = 0;
        for (int g = 0; g < G; ++g) {
            used += g < a.E && cnt[g] > 0;
            base[g] = at;
            tile[g] = nt;
            at += cnt[g];
            nt += (cnt[g] + a.tm - 1) / a.tm;
        }
        *a.ntiles = nt;
        if (a.n_experts) *a.n_experts += (unsigned long long)(used);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < G; g += kPlanThreads)
        for (int j = 0; j * a.tm < cnt[g]; ++j)
            a.tiles[tile[g] + j] = make_int4(g, base[g] + j * a.tm, min(a.tm, cnt[g] - j * a.tm), 0);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int e = entry_expert(a, i / a.ks, i % a.ks);
        if (e >= 0) a.order[atomicAdd(&base[e], 1)] = i;
    }
}

__device__ __forceinline__ const char* expert_blob(const MxArgs& a, int g) {
    return reinterpret_cast<const char*>(g < a.E ? a.eptr[g] : a.sptr[g - a.E]);
}

// Gate and up rows of one 16-row block and 16 tokens per wave; activations
// silu(g) * u as bf16 pieces.
template <bool XF, bool YF>
__global__ __launch_bounds__(kThreads) void mx_up_direct(MxArgs a, int nb) {
    const int tix = blockIdx.x / nb;
    if (tix >= *a.ntiles) return;
    const int4 tl = a.tiles[tix];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rb = int(blockIdx.x % nb) * kWaves + wave;
    if (rb >= row_blocks(a.I)) return;
    const char* blobp = expert_blob(a, tl.x);
    const Blob L = blob(a.H, a.I);
    const int KT = col_tiles(a.H), KG = col_groups(a.H);
    const char* gc = blobp + L.gate + size_t(rb) * KT * kTileBytes + lane * 16;
    const char* uc = blobp + L.up + size_t(rb) * KT * kTileBytes + lane * 16;
    const char* gs = blobp + L.gate_s + size_t(rb) * KG * kGroupBytes + lane * 4;
    const char* us = blobp + L.up_s + size_t(rb) * KG * kGroupBytes + lane * 4;
    const int c = lane & 15, q = lane >> 4;
    const bool live = c < tl.z;
    const size_t xrow = live ? size_t(a.order[tl.y + c] / a.ks) * a.H : 0;
    f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = {0.f, 0.f, 0.f, 0.f};
    for (int kt = 0; kt < KT; ++kt) {
        const uint4 gq = *reinterpret_cast<const uint4*>(gc + size_t(kt) * kTileBytes);
        const uint4 uq = *reinterpret_cast<const uint4*>(uc + size_t(kt) * kTileBytes);
        const float sg = scale_of(*reinterpret_cast<const uint8_t*>(gs + (kt / kGroupTiles) * kGroupBytes + kt % kGroupTiles));
        const float su = scale_of(*reinterpret_cast<const uint8_t*>(us + (kt / kGroupTiles) * kGroupBytes + kt % kGroupTiles));
        const uint32_t gw[4] = {gq.x, gq.y, gq.z, gq.w}, uw[4] = {uq.x, uq.y, uq.z, uq.w};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = kt * kTileCols + q * kBlock + s * 8;
            const Pieces<XF> xv = load8<XF>(a.x, xrow + k, live && k < a.H);
            const bf16x8 gv = decode8(gw[s], sg), uv = decode8(uw[s], su);
#pragma unroll
            for (int p = 0; p < Pieces<XF>::N; ++p) {
                g = __builtin_amdgcn_mfma_f32_16x16x32_bf16(gv, xv.p[p], g, 0, 0, 0);
                u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(uv, xv.p[p], u, 0, 0, 0);
            }
        }
    }
    // lane: token c, rows 4 q .. 4 q + 3 of the block
    const int row = rb * kTileRows + 4 * q;
    if (!live || row >= a.I) return;
    constexpr int NP = Pieces<YF>::N;
    union {
        __bf16 h[4];
        uint2 v;
    } o[NP];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v = g[i] / (1.f + expf(-g[i])) * u[i];
        if constexpr (YF) split(v, o[0].h[i], o[1].h[i]);
        else o[0].h[i] = __bf16(v);
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
        *reinterpret_cast<uint2*>(a.act + (size_t(tl.y + c) * NP + p) * a.I + row) = o[p].v;
}

// Down rows of one 16-row block and 16 entries per wave, times the gate
// weight, to the entries' partial rows.
template <bool YF>
__global__ __launch_bounds__(kThreads) void mx_down_direct(MxArgs a, int nb) {
    constexpr int NP = Pieces<YF>::N;
    const int tix = blockIdx.x / nb;
    if (tix >= *a.ntiles) return;
    const int4 tl = a.tiles[tix];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rb = int(blockIdx.x % nb) * kWaves + wave;
    if (rb >= row_blocks(a.H)) return;
    const char* blobp = expert_blob(a, tl.x);
    const Blob L = blob(a.H, a.I);
    const int KT = col_tiles(a.I), KG = col_groups(a.I);
    const char* dc = blobp + L.down + size_t(rb) * KT * kTileBytes + lane * 16;
    const char* ds = blobp + L.down_s + size_t(rb) * KG * kGroupBytes + lane * 4;
    const int c = lane & 15, q = lane >> 4;
    const bool live = c < tl.z;
    const size_t arow = live ? size_t(tl.y + c) * NP * a.I : 0;
    f32x4 d = {0.f, 0.f, 0.f, 0.f};
    for (int kt = 0; kt < KT; ++kt) {
        const uint4 dq = *reinterpret_cast<const uint4*>(dc + size_t(kt) * kTileBytes);
        const float sd = scale_of(*reinterpret_cast<const uint8_t*>(ds + (kt / kGroupTiles) * kGroupBytes + kt % kGroupTiles));
        const uint32_t dw[4] = {dq.x, dq.y, dq.z, dq.w};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = kt * kTileCols + q * kBlock + s * 8;
            const bf16x8 dv = decode8(dw[s], sd);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const Pieces<false> h = load8<false>(a.act, arow + size_t(p) * a.I + k, live && k < a.I);
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dv, h.p[0], d, 0, 0, 0);
            }
        }
    }
    const int row = rb * kTileRows + 4 * q;
    if (!live || row >= a.H) return;
    const int entry = a.order[tl.y + c], t = entry / a.ks, k = entry % a.ks;
    const float w = k < a.K ? a.w[size_t(t) * a.K + k] : 1.f;
    *reinterpret_cast<float4*>(a.part + size_t(entry) * a.H + row) = make_float4(w * d[0], w * d[1], w * d[2], w * d[3]);
}

// y[t] = the sum of its entries' rows, in the entries' order.
template <bool YF>
__global__ __launch_bounds__(kThreads) void mx_sum_kernel(MxArgs a) {
    const int t = blockIdx.x;
    unsigned used = 0u;
    for (int k = 0; k < a.ks; ++k)
        if (entry_expert(a, t, k) >= 0) used |= 1u << k;
    for (int h = threadIdx.x * 4; h < a.H; h += kThreads * 4) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < a.ks; ++k) {
            if (!(used >> k & 1u)) continue;
            const float4 v = *reinterpret_cast<const float4*>(a.part + (size_t(t) * a.ks + k) * a.H + h);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        if constexpr (YF) {
            *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.y) + size_t(t) * a.H + h) = s;
        } else {
            union {
                __bf16 b[4];
                uint2 v;
            } o;
            o.b[0] = __bf16(s.x); o.b[1] = __bf16(s.y); o.b[2] = __bf16(s.z); o.b[3] = __bf16(s.w);
            *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.y) + size_t(t) * a.H + h) = o.v;
        }
    }
}

struct MxLayout {
    int tm, max_tiles;
    size_t order, tiles, ntiles, act, part, total;
};

MxLayout mx_layout(int T, int K, int E, int H, int I, int ns, int ydtype) {
    MxLayout y{};
    const size_t n = size_t(T) * (K + ns);
    y.tm = 16;
    const size_t most = (n + y.tm - 1) / y.tm + E + ns;
    y.max_tiles = int(most < n ? most : n);
    size_t off = 0;
    auto take = [&](size_t b) { const size_t at = off; off = (off + b + 255) / 256 * 256; return at; };
    y.order = take(n * sizeof(int32_t));
    y.tiles = take(size_t(y.max_tiles) * sizeof(int4));
    y.ntiles = take(sizeof(int32_t));
    y.act = take(n * (ydtype == STMOE_F32 ? 2 : 1) * I * sizeof(uint16_t));
    y.part = take(n * H * sizeof(float));
    y.total = off;
    return y;
}

template <bool XF, bool YF>
int launch_direct(const MxArgs& a, const MxLayout& L, hipStream_t s, hipEvent_t ev_mid) {
    hipLaunchKernelGGL(mx_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
    STMOE_LAUNCHED();
    const int ub = (row_blocks(a.I) + kWaves - 1) / kWaves, db = (row_blocks(a.H) + kWaves - 1) / kWaves;
    hipLaunchKernelGGL((mx_up_direct<XF, YF>), dim3(unsigned(ub * L.max_tiles)), dim3(kThreads), 0, s, a, ub);
    STMOE_LAUNCHED();
    if (ev_mid) STMOE_HIP(hipEventRecord(ev_mid, s));
    hipLaunchKernelGGL((mx_down_direct<YF>), dim3(unsigned(db * L.max_tiles)), dim3(kThreads), 0, s, a, db);
    STMOE_LAUNCHED();
    hipLaunchKernelGGL((mx_sum_kernel<YF>), dim3(unsigned(a.T)), dim3(kThreads), 0, s, a);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

}  // namespace

// Internal entry of the decode-layer orchestration too (no argument checks).
// `ev_mid` is recorded between the gate/up and the down work.
int mx_ffn_launch(const void* x, const int32_t* idx, const float* w, int T, int K, int H, int I, int E, int dtype,
                  int ydtype, const void* const* eptr, const void* const* sptr, int n_shared, void* y, void* ws,
                  hipStream_t s, unsigned long long* n_experts, hipEvent_t ev_mid) {
    const MxLayout L = mx_layout(T, K, E, H, I, n_shared, ydtype);
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
    a.order = reinterpret_cast<int32_t*>(base + L.order);
    a.tiles = reinterpret_cast<int4*>(base + L.tiles);
    a.ntiles = reinterpret_cast<int32_t*>(base + L.ntiles);
    a.act = reinterpret_cast<uint16_t*>(base + L.act);
    a.part = reinterpret_cast<float*>(base + L.part);
    a.n_experts = n_experts;
    if (dtype == STMOE_F32) return ydtype == STMOE_F32 ? launch_direct<true, true>(a, L, s, ev_mid) : launch_direct<true, false>(a, L, s, ev_mid);
    return ydtype == STMOE_F32 ? launch_direct<false, true>(a, L, s, ev_mid) : launch_direct<false, false>(a, L, s, ev_mid);
}

}  // namespace stmoe

using namespace stmoe;

extern "C" size_t moe_expert_ffn_mx_workspace_bytes(int T, int K, int E, int H, int I, int n_shared, int dtype,
                                                    int ydtype) {
    if (T < 0 || T > kMaxT || E < 1 || E > kMaxE || K < 1 || K > E || K > kMaxK || H < 8 || H % 8 || H > kMaxH ||
        I < 8 || I % 8 || I > kMaxI || n_shared < 0 || n_shared > kMaxShared)
        return 0;
    if ((dtype != STMOE_BF16 && dtype != STMOE_F32) || (ydtype != STMOE_BF16 && ydtype != STMOE_F32)) return 0;
    return mx_layout(T < 1 ? 1 : T, K, E, H, I, n_shared, ydtype).total;
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
