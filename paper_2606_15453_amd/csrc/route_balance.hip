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
// Both directions are one pass over the logits.  A row belongs to 16 lanes, a
// row of the vector unit: its sums and maxima are four lane rotations, and a
// wave works on four rows at once, with up to 16 logits of each in a lane's
// registers.  The K winners are taken one by one (largest key, lowest index).
//
// The forward pass is bound by its instructions, those of the K selections above
// all (89 each for eight logits a lane, of which 65 are the vector unit's and 16
// waits between them): 32768 x 128 fp32, top 8, 16.8 us, the median of a trace,
// for 16.8 MB, and as long in bf16.  Its workgroups' sums go to a second launch
// of one workgroup (5.6 us; the last workgroup to arrive doing that in the first
// launch took as long).  The gradient is bound by its bytes and by the load of a
// selected logit, which waits for the selection: 36 MB in 11.2 us, 3.2 TB/s.
#include <type_traits>

#include "common.h"

namespace stmoe {
namespace {

constexpr int kWaves = 16;
constexpr int kThreads = 64 * kWaves;
constexpr int kRowLanes = 16;
constexpr int kRows = 64 / kRowLanes;      // rows a wave works on
constexpr int kMaxWg = 256;                // workgroups of the forward pass, each with a row of partial sums
// Rows that a lane adds up, in 32 bits, before the sums in 64: beyond 2^19 tokens
// there are more than kMaxWg workgroups instead.  Equal rows' rounding errors do not cancel
// (4096 of them are up to 4e-5 off, 32 at most 2e-6).  2^24 x 128 bf16, top 8, takes
// 5.46 ms, 5.26 in 256 workgroups; 2^26 x 8 3.7 and 5.1.
constexpr int kChain = 32;
constexpr int kGradThreads = 256;

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

// Rotations within the 16 lanes of a row.
template <int N>
__device__ __forceinline__ uint32_t rotate(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(int(v), int(v), 0x120 + N, 0xf, 0xf, false));
}
template <int N>
__device__ __forceinline__ float rotate(float v) { return __uint_as_float(rotate<N>(__float_as_uint(v))); }

__device__ __forceinline__ float row_sum(float v) {
    v += rotate<8>(v);
    v += rotate<4>(v);
    v += rotate<2>(v);
    return v + rotate<1>(v);
}
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    v = max(v, rotate<8>(v));
    v = max(v, rotate<4>(v));
    v = max(v, rotate<2>(v));
    return max(v, rotate<1>(v));
}
__device__ __forceinline__ uint32_t row_min(uint32_t v) {
    v = min(v, rotate<8>(v));
    v = min(v, rotate<4>(v));
    v = min(v, rotate<2>(v));
    return min(v, rotate<1>(v));
}

// Candidates' order as unsigned keys: larger logit, larger key; -0 and +0 are
// one value; NaN 1, below every number; minus infinity is no candidate: 0.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t u = v == 0.f ? 0u : __float_as_uint(v);
    const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return v != v ? 1u : v == -INFINITY ? 0u : k;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return key == 1u ? __builtin_nanf("") : __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

// Expert of a lane's v-th logit.  VEC: four consecutive ones, loaded at once
// (bf16: 8 bytes a lane; fp32 loads are no faster for it).
template <bool VEC>
__device__ __forceinline__ int expert_at(int v, int l) {
    return VEC ? (v >> 2) * 4 * kRowLanes + 4 * l + (v & 3) : v * kRowLanes + l;
}

// A lane's logits of the row at element `at`; minus infinity beyond E.
template <bool BF, int V, bool VEC>
__device__ __forceinline__ void load_row(const void* logits, int64_t at, int E, int l, float (&z)[V]) {
    if constexpr (VEC) {
#pragma unroll
        for (int v = 0; v < V; v += 4) {
            const int e = expert_at<true>(v, l);
            uint2 q = make_uint2(0xff80ff80u, 0xff80ff80u);
            if (e < E) q = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(logits) + at + e);  // E is a multiple of 4
            z[v] = bf16_lo(q.x);
            z[v + 1] = bf16_hi(q.x);
            z[v + 2] = bf16_lo(q.y);
            z[v + 3] = bf16_hi(q.y);
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = expert_at<false>(v, l);
            z[v] = -INFINITY;
            if (e < E)
                z[v] = BF ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(logits)[at + e]) << 16)
                          : reinterpret_cast<const float*>(logits)[at + e];
        }
    }
}

// exp(z - top) of a candidate; none (0) for minus infinity.  The hardware's
// exponential: the product with log2(e) rounds to 2^-24 of |z - top|, as the
// difference itself does.
__device__ __forceinline__ float term(float z, float top) { return z == -INFINITY ? 0.f : __expf(z - top); }

template <bool BF, int V, bool VEC>
__global__ __launch_bounds__(kThreads) void balance_kernel(BalanceArgs a) {
    __shared__ float lp[kWaves][V * kRowLanes];
    __shared__ int32_t lc[V * kRowLanes];
    __shared__ float lz[kWaves];
    __shared__ int32_t ln[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (kRowLanes - 1), r = lane / kRowLanes;
    for (int e = threadIdx.x; e < V * kRowLanes; e += kThreads) lc[e] = 0;
    __syncthreads();
    float ps[V], zs = 0.f;
    int cs[V], n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ps[v] = 0.f;
        cs[v] = 0;
    }
    const int64_t step = int64_t(gridDim.x) * kWaves * kRows;
    for (int64_t t0 = (int64_t(blockIdx.x) * kWaves + wave) * kRows; t0 < a.T; t0 += step) {
        const int64_t t = t0 + r;
        const bool in = t < a.T;
        float z[V];
        // rows beyond the batch and masked ones have no candidates (the row and
        // its mask are loaded side by side)
        const uint8_t counts = in && a.mask ? a.mask[t] : uint8_t(in);
        load_row<BF, V, VEC>(a.logits, (in ? t : a.T - 1) * a.ld, a.E, l, z);
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = counts ? z[v] : -INFINITY;
        uint32_t key[V], best = 0u;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            key[v] = key_of(z[v]);
            best = max(best, key[v]);
        }
        best = row_max(best);
        const bool live = best != 0u;
        const float top = value_of(best);
        float ex[V], sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ex[v] = live ? term(z[v], top) : 0.f;
            sum += ex[v];
        }
        sum = row_sum(sum);
        const float inv = live ? 1.f / sum : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) ps[v] += ex[v] * inv;
        // lane k of the row keeps winner k
        int mine = -1;
        uint32_t won = 0u;
        for (int k = 0; k < a.K; ++k) {
            if (k) {
                best = 0u;
#pragma unroll
                for (int v = 0; v < V; ++v) best = max(best, key[v]);
                best = row_max(best);
            }
            uint32_t at = ~0u;
#pragma unroll
            for (int v = V - 1; v >= 0; --v) at = key[v] == best ? uint32_t(expert_at<VEC>(v, l)) : at;
            at = best ? row_min(at) : ~0u;
            if (l == k && best) {
                mine = int(at);
                won = best;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = at == uint32_t(expert_at<VEC>(v, l)) ? 0u : key[v];
        }
        // what is left of the candidates
#pragma unroll
        for (int v = 0; v < V; ++v) cs[v] += z[v] != -INFINITY && key[v] == 0u;
        const float wk = mine >= 0 ? term(value_of(won), top) : 0.f;
        const float norm = a.renorm ? 1.f / row_sum(wk) : inv;
        if (in && l < a.K) {
            a.idx[t * a.K + l] = mine;
            a.w[t * a.K + l] = mine >= 0 ? wk * norm : 0.f;
        }
        if (live && l == 0) {
            const float lse = top + logf(sum);
            zs += lse * lse;
            ++n;
        }
    }
    // the wave's four rows, then the waves in order
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ps[v] += __shfl_xor(ps[v], 16, 64);
        ps[v] += __shfl_xor(ps[v], 32, 64);
        cs[v] += __shfl_xor(cs[v], 16, 64);
        cs[v] += __shfl_xor(cs[v], 32, 64);
        if (lane < kRowLanes) {
            lp[wave][expert_at<VEC>(v, l)] = ps[v];
            if (cs[v]) atomicAdd(&lc[expert_at<VEC>(v, l)], cs[v]);
        }
    }
    zs = wave_sum(zs);
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d, 64);
    if (lane == 0) {
        lz[wave] = zs;
        ln[wave] = n;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kThreads) {
        float s = 0.f;
#pragma unroll
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

// Sums over the workgroups in 64 bits, in a fixed order; the losses.  Thread
// (part, expert): every kParts-th workgroup.
__global__ __launch_bounds__(1024) void balance_finish_kernel(BalanceArgs a) {
    __shared__ double sp[1024];
    __shared__ int sc[1024];
    __shared__ double zz[kMaxWg];
    __shared__ int nn[kMaxWg];
    const int tid = threadIdx.x;
    int EP = 32;                           // experts side by side, a power of two
    while (EP < a.E) EP *= 2;
    const int parts = 1024 / EP, e = tid & (EP - 1), part = tid / EP;
    double p = 0.0;
    int c = 0;
    if (e < a.E) {
#pragma unroll 8
        for (int g = part; g < a.wg; g += parts) {
            p += a.part_p[size_t(g) * a.E + e];
            c += a.part_c[size_t(g) * a.E + e];
        }
    }
    sp[tid] = p;
    sc[tid] = c;
    if (tid < kMaxWg) {
        double z = 0.0;
        int n = 0;
        for (int g = tid; g < a.wg; g += kMaxWg) {
            z += a.part_z[g];
            n += a.part_n[g];
        }
        zz[tid] = z;
        nn[tid] = n;
    }
    for (int d = kMaxWg / 2; d; d >>= 1) {
        __syncthreads();
        if (tid < d) {
            zz[tid] += zz[tid + d];
            nn[tid] += nn[tid + d];
        }
    }
    __syncthreads();
    const double n = nn[0] > 0 ? nn[0] : 1;
    double term = 0.0;
    if (part == 0) {
        for (int g = 1; g < parts; ++g) {
            p += sp[g * EP + e];
            c += sc[g * EP + e];
        }
        if (e < a.E) {
            a.counts[e] = c;
            if (a.prob_sum) a.prob_sum[e] = float(p);
            term = a.E * (c / (n * a.K)) * (p / n);
        }
    }
    __syncthreads();
    if (part == 0) sp[e] = term;
    for (int d = EP / 2; d; d >>= 1) {
        __syncthreads();
        if (tid < d) sp[tid] += sp[tid + d];
    }
    if (tid == 0) {
        *a.n = nn[0];
        a.loss[0] = float(sp[0]);
        a.loss[1] = float(zz[0] / n);
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

// The gate weights' part of a row, one term per selected expert, goes through
// LDS to the lanes that hold those experts.
template <bool BF, int V, bool VEC>
__global__ __launch_bounds__(kGradThreads) void balance_grad_kernel(BalanceGradArgs a) {
    __shared__ float sel[kGradThreads / 64][kRows][V * kRowLanes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (kRowLanes - 1), r = lane / kRowLanes;
    float* mysel = sel[wave][r];
#pragma unroll
    for (int v = 0; v < V; ++v) mysel[v * kRowLanes + l] = 0.f;
    const float n = float(*a.n > 0 ? *a.n : 1);
    const float gz = 2.f * a.d_loss[1] / n, cb = a.d_loss[0] * a.E / a.K / n / n;
    float cf[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = expert_at<VEC>(v, l);
        cf[v] = e < a.E ? cb * float(a.counts[e]) : 0.f;
    }
    const int64_t step = int64_t(gridDim.x) * (kGradThreads / 64) * kRows;
    for (int64_t t0 = (int64_t(blockIdx.x) * (kGradThreads / 64) + wave) * kRows; t0 < a.T; t0 += step) {
        const int64_t t = t0 + r;
        const bool in = t < a.T;
        // the row, its selection and the weights' gradients side by side
        const int mine = in && l < a.K ? a.idx[t * a.K + l] : -1;
        float g = a.d_w && in && l < a.K ? a.d_w[t * a.K + l] : 0.f;
        float z[V];
        load_row<BF, V, VEC>(a.logits, (in ? t : a.T - 1) * a.ld, a.E, l, z);
        const bool live = __shfl(mine, r * kRowLanes, 64) >= 0;
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = live ? z[v] : -INFINITY;
        const bool chosen = a.d_w && live && mine >= 0 && mine < a.E;
        float zk = -INFINITY;
        if (chosen) {
            zk = BF ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(a.logits)[t * a.ld + mine]) << 16)
                    : reinterpret_cast<const float*>(a.logits)[t * a.ld + mine];
        }
        // the largest number; a NaN enters by its own term
        uint32_t best = 0u;
#pragma unroll
        for (int v = 0; v < V; ++v) best = max(best, key_of(z[v]));
        const float top = value_of(row_max(best));
        float ex[V], sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ex[v] = live ? term(z[v], top) : 0.f;
            sum += ex[v];
        }
        sum = row_sum(sum);
        const float inv = live ? 1.f / sum : 0.f;
        float pa = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ex[v] *= inv;
            pa += ex[v] * cf[v];
        }
        float base = gz * (live ? top + logf(sum) : 0.f) - row_sum(pa);
        if (a.d_w) {
            // lane k: selected expert k with its weight
            float wk = chosen ? term(zk, top) : 0.f;
            wk *= a.renorm ? 1.f / row_sum(wk) : inv;
            const float wg = row_sum(chosen ? wk * g : 0.f);
            if (!a.renorm) base -= wg;
            if (chosen) mysel[mine] = a.renorm ? wk * (g - wg) : wk * g;
            // a wave's LDS accesses complete in order
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        float d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            d[v] = ex[v] * (cf[v] + base);
            if (a.d_w) d[v] += mysel[expert_at<VEC>(v, l)];
            if (!live) d[v] = 0.f;
        }
        if (a.d_w) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (chosen) mysel[mine] = 0.f;
        }
        if (!in) continue;
        const int64_t o = t * a.ld_d;
        if constexpr (VEC) {
#pragma unroll
            for (int v = 0; v < V; v += 4) {
                const int e = expert_at<true>(v, l);
                if (e >= a.E) continue;
                union {
                    __bf16 b[4];
                    uint2 q;
                } u;
#pragma unroll
                for (int i = 0; i < 4; ++i) u.b[i] = __bf16(d[v + i]);
                *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.d_logits) + o + e) = u.q;
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = expert_at<false>(v, l);
                if (e >= a.E) continue;
                if (BF) reinterpret_cast<__bf16*>(a.d_logits)[o + e] = __bf16(d[v]);
                else reinterpret_cast<float*>(a.d_logits)[o + e] = d[v];
            }
        }
    }
}

struct BalanceLayout {
    int wg;
    size_t p, c, z, n, total;
};

BalanceLayout balance_layout(int64_t T, int E) {
    BalanceLayout y{};
    const int64_t wg = (T + kWaves * kRows - 1) / (kWaves * kRows), chains = (wg + kChain - 1) / kChain;
    y.wg = int(wg < 1 ? 1 : wg < kMaxWg ? wg : chains < kMaxWg ? kMaxWg : chains);
    size_t off = 0;
    auto take = [&](size_t b) { const size_t at = off; off = (off + b + 255) / 256 * 256; return at; };
    y.p = take(size_t(y.wg) * E * sizeof(float));
    y.c = take(size_t(y.wg) * E * sizeof(int32_t));
    y.z = take(size_t(y.wg) * sizeof(float));
    y.n = take(size_t(y.wg) * sizeof(int32_t));
    y.total = off;
    return y;
}

// Calls f(bf16, logits per lane, VEC) for E experts.  VEC: bf16 rows of whole
// groups of four, aligned to them (32768 x 128, shortest launches: 14.5 us with,
// 15.7 without, the gradient 9.8 and 11.2; fp32 15.4 and 15.5, 10.3 and 9.8).
template <class F>
void with_row(int dtype, int E, bool fours, F f) {
    const auto lanes = [&](auto bf, auto vec) {
        if (E <= 64) f(bf, std::integral_constant<int, 4>(), vec);
        else if (E <= 128) f(bf, std::integral_constant<int, 8>(), vec);
        else f(bf, std::integral_constant<int, 16>(), vec);
    };
    const auto any = [&](auto bf) {
        if (E <= 16) f(bf, std::integral_constant<int, 1>(), std::false_type());
        else if (E <= 32) f(bf, std::integral_constant<int, 2>(), std::false_type());
        else lanes(bf, std::false_type());
    };
    if (dtype != STMOE_BF16) any(std::false_type());
    else if (E > 32 && fours) lanes(std::true_type(), std::true_type());
    else any(std::true_type());
}

bool rows_of_four(const void* p, int64_t ld, int E) {
    return E % 4 == 0 && ld % 4 == 0 && reinterpret_cast<uintptr_t>(p) % 8 == 0;
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
    with_row(dtype, E, rows_of_four(logits, ld, E), [&](auto bf, auto v, auto vec) {
        hipLaunchKernelGGL((balance_kernel<bf(), v(), vec()>), dim3(unsigned(L.wg)), dim3(kThreads), 0, s, a);
    });
    STMOE_LAUNCHED();
    hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(1024), 0, s, a);
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
    // 1024 workgroups at most (32768 x 128 fp32, shortest launches: 16.0 us with 256,
    // 10.3, 11.1 with 4096)
    const int64_t per = kGradThreads / 64 * kRows, wg = (T + per - 1) / per;
    const dim3 grid(unsigned(wg < 1024 ? wg : 1024));
    with_row(dtype, E, rows_of_four(logits, ld, E) && rows_of_four(d_logits, ld_d, E), [&](auto bf, auto v, auto vec) {
        hipLaunchKernelGGL((balance_grad_kernel<bf(), v(), vec()>), grid, dim3(kGradThreads), 0, as_stream(stream), a);
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}
