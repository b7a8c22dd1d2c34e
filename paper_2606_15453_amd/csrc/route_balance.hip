// The router over a batch of tokens for training: softmax and top-K of given
// logits, per-expert counts, the balance and z losses, and their gradient.
//
// With p_te the softmax of row t, n the number of live rows, c_e the number of
// selections of expert e and S_e = sum_t p_te over live rows:
//   balance = E sum_e c_e / (n K) * S_e / n        z = sum_t lse_t^2 / n
// and, with counts and n as constants, for upstream gradients g_b, g_z and g_tk
// of the two losses and of the gate weights:
//   d_te = p_te (a_te - sum_j p_tj a_tj) + 2 g_z / n lse_t p_te,
//   a_te = g_b E c_e / (n^2 K) + [e = idx_tk] g_tk            (weights p)
// or, with renormalised weights w_k = softmax over the selected logits, the
// second term of a_te is replaced by w_k (g_tk - sum_j w_j g_tj) on top of d_te.
// Both directions are one pass over the logits, a row in a wave's registers.
#include "gating_dev.h"

namespace stmoe {
namespace {

using gating::kKeyRegs;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxWg = 512;        // workgroups of the forward pass, each with a row of partial sums

struct BalanceArgs {
    const void* logits;            // [T] rows of stride ld
    int64_t T, ld;
    int E, K, renorm;
    const uint8_t* mask;           // [T] or null
    int32_t* idx;                  // [T][K]
    float* w;                      // [T][K]
    int32_t* counts;               // [E]
    int32_t* n;                    // [1]
    float* prob_sum;               // [E] or null
    float* loss;                   // [2]
    // partial sums per workgroup
    float* part_p;                 // [wg][E]
    int32_t* part_c;               // [wg][E]
    float* part_z;                 // [wg]
    int32_t* part_n;               // [wg]
    int wg;
};

// Logits of row t: lane l holds those of l, l + 64, ...
template <bool BF>
__device__ __forceinline__ void load_row(const void* logits, int64_t at, int E, float (&z)[kKeyRegs]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int v = 0; v < kKeyRegs; ++v) {
        const int e = 64 * v + lane;
        z[v] = -INFINITY;
        if (e < E)
            z[v] = BF ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(logits)[at + e]) << 16)
                      : reinterpret_cast<const float*>(logits)[at + e];
    }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
}

// Softmax terms of a row: its largest logit (NaN aside), exp(z - max), their
// sum.  Logits of minus infinity are no candidates; false where a row has none.
__device__ __forceinline__ bool row_softmax(const float (&z)[kKeyRegs], float& top, float (&ex)[kKeyRegs], float& sum) {
    float m = -INFINITY;
    bool any = false;
#pragma unroll
    for (int v = 0; v < kKeyRegs; ++v) {
        m = fmaxf(m, z[v]);
        any |= z[v] != -INFINITY;      // also NaN
    }
    top = wave_max(m);
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < kKeyRegs; ++v) {
        ex[v] = z[v] == -INFINITY ? 0.f : expf(z[v] - top);
        s += ex[v];
    }
    sum = wave_sum(s);
    return __ballot(any) != 0ull;
}

template <bool BF>
__global__ __launch_bounds__(kThreads) void balance_kernel(BalanceArgs a) {
    __shared__ float lp[kWaves][kMaxE];
    __shared__ int32_t lc[kMaxE];
    __shared__ float lz[kWaves];
    __shared__ int32_t ln[kWaves];
    constexpr int V = kKeyRegs;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e < kMaxE; e += kThreads) lc[e] = 0;
    __syncthreads();
    float ps[V], zs = 0.f;
    int n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) ps[v] = 0.f;
    for (int64_t t = int64_t(blockIdx.x) * kWaves + wave; t < a.T; t += int64_t(gridDim.x) * kWaves) {
        float z[V], ex[V], top, sum;
        uint32_t key[V];
        bool ok[V], win[V];
        int pos[V];
        const bool masked = a.mask && !a.mask[t];
        bool live = false;
        if (!masked) {
            load_row<BF>(a.logits, t * a.ld, a.E, z);
            live = row_softmax(z, top, ex, sum);
        }
        int won = 0;
        if (live) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                ok[v] = 64 * v + lane < a.E && z[v] != -INFINITY;
                // NaN ranks below every number and above what is no candidate
                const uint32_t k = gating::order_key(z[v]);
                key[v] = ok[v] ? (k ? k : 1u) : 0u;
            }
            gating::topk_positions(key, ok, a.E, a.K, win, pos);
            float q = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                won += __popcll(__ballot(win[v]));
                q += win[v] ? ex[v] : 0.f;
                ps[v] += ex[v] / sum;
            }
            const float norm = a.renorm ? wave_sum(q) : sum;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (win[v]) {
                    a.idx[t * a.K + pos[v]] = 64 * v + lane;
                    a.w[t * a.K + pos[v]] = ex[v] / norm;
                    atomicAdd(&lc[64 * v + lane], 1);
                }
            const float lse = top + logf(sum);
            zs += lse * lse;
            ++n;
        }
        if (lane >= won && lane < a.K) {
            a.idx[t * a.K + lane] = -1;
            a.w[t * a.K + lane] = 0.f;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) lp[wave][64 * v + lane] = ps[v];
    if (lane == 0) {
        lz[wave] = zs;
        ln[wave] = n;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kThreads) {
        float s = 0.f;
        for (int u = 0; u < kWaves; ++u) s += lp[u][e];
        a.part_p[size_t(blockIdx.x) * a.E + e] = s;
        a.part_c[size_t(blockIdx.x) * a.E + e] = lc[e];
    }
    if (threadIdx.x == 0) {
        float s = 0.f;
        int m = 0;
        for (int u = 0; u < kWaves; ++u) {
            s += lz[u];
            m += ln[u];
        }
        a.part_z[blockIdx.x] = s;
        a.part_n[blockIdx.x] = m;
    }
}

// Sums over the workgroups, in their order, in 64 bits; the losses.
__global__ __launch_bounds__(kThreads) void balance_finish_kernel(BalanceArgs a) {
    __shared__ double red[kThreads];
    __shared__ int nn;
    const int e = threadIdx.x;
    if (e == 0) {
        int n = 0;
        for (int g = 0; g < a.wg; ++g) n += a.part_n[g];
        nn = n;
        *a.n = n;
    }
    __syncthreads();
    const double n = nn > 0 ? nn : 1;
    double term = 0.0;
    if (e < a.E) {
        double p = 0.0;
        int c = 0;
        for (int g = 0; g < a.wg; ++g) {
            p += a.part_p[size_t(g) * a.E + e];
            c += a.part_c[size_t(g) * a.E + e];
        }
        a.counts[e] = c;
        if (a.prob_sum) a.prob_sum[e] = float(p);
        term = a.E * (c / (n * a.K)) * (p / n);
    }
    red[e] = term;
    __syncthreads();
    if (e == 0) {
        double s = 0.0, z = 0.0;
        for (int i = 0; i < a.E; ++i) s += red[i];
        for (int g = 0; g < a.wg; ++g) z += a.part_z[g];
        a.loss[0] = float(s);
        a.loss[1] = float(z / n);
    }
}

struct BalanceGradArgs {
    const void* logits;
    int64_t T, ld, ld_d;
    int E, K, renorm;
    const int32_t *idx, *counts, *n;
    const float *d_w, *d_loss;
    void* d_logits;
};

template <bool BF>
__global__ __launch_bounds__(kThreads) void balance_grad_kernel(BalanceGradArgs a) {
    constexpr int V = kKeyRegs;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float n = float(*a.n > 0 ? *a.n : 1);
    const float gz = 2.f * a.d_loss[1] / n;
    float cf[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        cf[v] = 64 * v + lane < a.E ? a.d_loss[0] * a.E / a.K * float(a.counts[64 * v + lane]) / (n * n) : 0.f;
    for (int64_t t = int64_t(blockIdx.x) * kWaves + wave; t < a.T; t += int64_t(gridDim.x) * kWaves) {
        const int sel = lane < a.K ? a.idx[t * a.K + lane] : -1;
        const float dw = a.d_w && sel >= 0 ? a.d_w[t * a.K + lane] : 0.f;
        float d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = 0.f;
        float z[V], ex[V], top, sum;
        if (__builtin_amdgcn_readfirstlane(sel) >= 0) {
            load_row<BF>(a.logits, t * a.ld, a.E, z);
            row_softmax(z, top, ex, sum);
            float gw[V];
            bool hit[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                gw[v] = 0.f;
                hit[v] = false;
            }
            for (int k = 0; k < a.K; ++k) {
                const int e = __builtin_amdgcn_readlane(sel, k);
                const float g = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(dw), k));
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (e == 64 * v + lane) {
                        gw[v] += g;
                        hit[v] = true;
                    }
            }
            float q = 0.f, qg = 0.f, pa = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                q += hit[v] ? ex[v] : 0.f;
                qg += hit[v] ? ex[v] * gw[v] : 0.f;
            }
            if (a.renorm) {
                q = wave_sum(q);
                qg = wave_sum(qg) / q;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) pa += ex[v] / sum * (cf[v] + (a.renorm ? 0.f : gw[v]));
            pa = wave_sum(pa);
            const float lse = top + logf(sum);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float p = ex[v] / sum;
                d[v] = p * (cf[v] + (a.renorm ? 0.f : gw[v]) - pa + gz * lse);
                if (a.renorm && hit[v]) d[v] += ex[v] / q * (gw[v] - qg);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = 64 * v + lane;
            if (e >= a.E) continue;
            if (BF) reinterpret_cast<__bf16*>(a.d_logits)[t * a.ld_d + e] = __bf16(d[v]);
            else reinterpret_cast<float*>(a.d_logits)[t * a.ld_d + e] = d[v];
        }
    }
}

struct BalanceLayout {
    int wg;
    size_t p, c, z, n, total;
};

BalanceLayout balance_layout(int64_t T, int E) {
    BalanceLayout y{};
    const int64_t wg = (T + kWaves - 1) / kWaves;
    y.wg = int(wg < 1 ? 1 : wg < kMaxWg ? wg : kMaxWg);
    size_t off = 0;
    auto take = [&](size_t b) { const size_t at = off; off = (off + b + 255) / 256 * 256; return at; };
    y.p = take(size_t(y.wg) * E * sizeof(float));
    y.c = take(size_t(y.wg) * E * sizeof(int32_t));
    y.z = take(size_t(y.wg) * sizeof(float));
    y.n = take(size_t(y.wg) * sizeof(int32_t));
    y.total = off;
    return y;
}

int check_router(const char* fn, int64_t T, int64_t ld, int E, int K, int dtype) {
    const char* bad = nullptr;
    if (T < 0 || T > (int64_t(1) << 26)) bad = "T must be in [0, 2^26]";
    else if (E < 1 || E > kMaxE) bad = "E must be in [1, 256]";
    else if (K < 1 || K > E || K > kMaxK) bad = "K must be in [1, min(E, 16)]";
    else if (ld < E || ld > (int64_t(1) << 31)) bad = "the row stride must be in [E, 2^31]";
    else if (dtype != STMOE_BF16 && dtype != STMOE_F32) bad = "dtype must be STMOE_BF16 or STMOE_F32";
    if (!bad) return STMOE_OK;
    set_error(std::string(fn) + ": " + bad);
    return STMOE_EINVAL;
}

}  // namespace
}  // namespace stmoe

using namespace stmoe;

extern "C" size_t moe_route_balance_workspace_bytes(int64_t T, int E) {
    if (T < 0 || T > (int64_t(1) << 26) || E < 1 || E > kMaxE) return 0;
    return balance_layout(T, E).total;
}

extern "C" int moe_route_balance(const void* logits, int64_t T, int64_t ld, int E, int K, int dtype, int renorm,
                                 const uint8_t* mask, int32_t* topk_idx, float* topk_w, int32_t* counts,
                                 int32_t* n_tokens, float* prob_sum, float* loss, void* ws, size_t ws_bytes,
                                 void* stream) {
    clear_error();
    if (int rc = check_router(__func__, T, ld, E, K, dtype)) return rc;
    STMOE_CHECK(counts && n_tokens && loss && ws, "null pointer");
    STMOE_CHECK(T == 0 || (logits && topk_idx && topk_w), "null pointer");
    const BalanceLayout L = balance_layout(T, E);
    STMOE_CHECK(ws_bytes >= L.total, "workspace too small");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(ws) % 256 == 0, "ws must be 256-byte aligned");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(logits) % (dtype == STMOE_BF16 ? 2 : 4) == 0,
                "logits must be aligned to their elements");
    char* base = reinterpret_cast<char*>(ws);
    BalanceArgs a{};
    a.logits = logits;
    a.T = T;
    a.ld = ld;
    a.E = E;
    a.K = K;
    a.renorm = renorm ? 1 : 0;
    a.mask = mask;
    a.idx = topk_idx;
    a.w = topk_w;
    a.counts = counts;
    a.n = n_tokens;
    a.prob_sum = prob_sum;
    a.loss = loss;
    a.part_p = reinterpret_cast<float*>(base + L.p);
    a.part_c = reinterpret_cast<int32_t*>(base + L.c);
    a.part_z = reinterpret_cast<float*>(base + L.z);
    a.part_n = reinterpret_cast<int32_t*>(base + L.n);
    a.wg = L.wg;
    hipStream_t s = as_stream(stream);
    if (dtype == STMOE_BF16) hipLaunchKernelGGL((balance_kernel<true>), dim3(unsigned(L.wg)), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((balance_kernel<false>), dim3(unsigned(L.wg)), dim3(kThreads), 0, s, a);
    STMOE_LAUNCHED();
    hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(kThreads), 0, s, a);
    STMOE_LAUNCHED();
    return STMOE_OK;
}

extern "C" int moe_route_balance_backward(const void* logits, int64_t T, int64_t ld, int E, int K, int dtype,
                                          int renorm, const int32_t* topk_idx, const int32_t* counts,
                                          const int32_t* n_tokens, const float* d_w, const float* d_loss,
                                          void* d_logits, int64_t ld_d, void* stream) {
    clear_error();
    if (int rc = check_router(__func__, T, ld, E, K, dtype)) return rc;
    STMOE_CHECK(ld_d >= E && ld_d <= (int64_t(1) << 31), "the gradient's row stride must be in [E, 2^31]");
    if (T == 0) return STMOE_OK;
    STMOE_CHECK(logits && topk_idx && counts && n_tokens && d_loss && d_logits, "null pointer");
    const uintptr_t esz = dtype == STMOE_BF16 ? 2 : 4;
    STMOE_CHECK(reinterpret_cast<uintptr_t>(logits) % esz == 0 && reinterpret_cast<uintptr_t>(d_logits) % esz == 0,
                "logits and d_logits must be aligned to their elements");
    BalanceGradArgs a{};
    a.logits = logits;
    a.T = T;
    a.ld = ld;
    a.ld_d = ld_d;
    a.E = E;
    a.K = K;
    a.renorm = renorm ? 1 : 0;
    a.idx = topk_idx;
    a.counts = counts;
    a.n = n_tokens;
    a.d_w = d_w;
    a.d_loss = d_loss;
    a.d_logits = d_logits;
    const int64_t wg = (T + kWaves - 1) / kWaves;
    const dim3 grid(unsigned(wg < 2048 ? wg : 2048));
    if (dtype == STMOE_BF16)
        hipLaunchKernelGGL((balance_grad_kernel<true>), grid, dim3(kThreads), 0, as_stream(stream), a);
    else
        hipLaunchKernelGGL((balance_grad_kernel<false>), grid, dim3(kThreads), 0, as_stream(stream), a);
    STMOE_LAUNCHED();
    return STMOE_OK;
}
