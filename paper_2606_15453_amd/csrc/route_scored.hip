// Routing by scores: softmax or sigmoid of given logits, a bias for balance, the
// best groups of experts, the top K in them and their weights; the weights'
// gradient; the bias's step.
//
// With s the scores of a row and b the bias, c = s + b chooses and s weighs:
//   group's score   the sum of its best group_top choices (1 or 2)
//   selection       the best K experts of the best top_groups groups
//   weights         scale s_k, or scale s_k / sum of the selected s
// and, with the selection as a constant and g_k the weights' gradients, w' = w / scale:
//   sigmoid   d_k = scale g_k s_k (1 - s_k)             d_k = w_k (g_k - sum_j w'_j g_j)(1 - s_k)
//   softmax   d_e = [e = idx_k] w_k g_k - s_e sum w_j g_j    d_k = w_k (g_k - sum_j w'_j g_j)
// (left: weights as they are, right: renormalised).
//
// A choice between two experts is made by the 64-bit values of s + b: in 32 bits
// experts whose choices are 1e-7 apart change places, one row in some hundred.
// A row belongs to 16 lanes, a lane to consecutive experts.
#include <type_traits>

#include "row16.h"

namespace stmoe {
namespace {

using namespace row16;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct ScoredArgs {
    const void* logits;            // [T] rows of stride ld
    int64_t T, ld;
    int E, K, sigmoid, groups, top_groups, group_top, renorm;
    float scale;
    const float* bias;             // [E] or null
    const uint8_t* mask;           // [T] or null
    int32_t* idx;                  // [T][K]
    float* w;                      // [T][K]
    int32_t* counts;               // [E] or null, added to
};

template <bool BF>
__device__ __forceinline__ float logit(const void* p, int64_t at) {
    return BF ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(p)[at]) << 16)
              : reinterpret_cast<const float*>(p)[at];
}

// A lane's logits, experts l V + v, of the row at element `at`; minus infinity beyond E.
template <bool BF, int V>
__device__ __forceinline__ void load_row(const void* logits, int64_t at, int E, int l, float (&z)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = l * V + v;
        z[v] = e < E ? logit<BF>(logits, at + e) : -INFINITY;
    }
}

// Key of a lane's logits' choices in 64 bits; 0 where there is no candidate.
template <int V>
__device__ __forceinline__ void choices64(const ScoredArgs& a, int l, const float (&z)[V], bool scores, uint64_t (&key)[V]) {
    double s[V];
    if (scores && a.sigmoid) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = 1.0 / (1.0 + exp(-double(z[v])));
    } else if (scores) {
        double top = -INFINITY, sum = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v) top = fmax(top, double(z[v]));
        top = largest(top);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[v] = z[v] == -INFINITY ? 0.0 : exp(double(z[v]) - top);
            sum += s[v];
        }
        sum = row16::sum(sum);
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] /= sum;
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = z[v];
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = l * V + v;
        const float b = a.bias && e < a.E ? a.bias[e] : 0.f;
        key[v] = z[v] == -INFINITY || b == -INFINITY ? 0ull : key64(s[v] + double(b));
    }
}

// Drops the candidates outside the best groups.  keys: room for the row's choices
// (LDS); a group's score takes the place of its first one.
template <int V>
__device__ __forceinline__ void keep_groups(const ScoredArgs& a, int l, uint64_t* keys, const uint64_t (&by)[V],
                                            uint64_t (&key)[V]) {
    const int size = a.E / a.groups;
#pragma unroll
    for (int v = 0; v < V; ++v) keys[l * V + v] = by[v];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int g = l; g < a.groups; g += kLanes) {
        uint64_t first = 0, second = 0;
        for (int i = 0; i < size; ++i) {
            const uint64_t k = keys[g * size + i];
            second = max(second, min(first, k));
            first = max(first, k);
        }
        keys[g * size] = a.group_top == 2 && second ? key64(value64(first) + value64(second)) : first;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = l * V + v, g = e < a.E ? e / size : 0;
        const uint64_t mine = keys[g * size];
        int before = 0;
        for (int i = 0; i < a.groups; ++i) {
            const uint64_t other = keys[i * size];
            before += other > mine || (other == mine && i < g);
        }
        if (before >= a.top_groups) key[v] = 0ull;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The K best of a row one by one: lane k gets the k-th (-1: there is none).
template <int V>
__device__ __forceinline__ int select64(int K, int l, uint64_t (&key)[V]) {
    int mine = -1;
    for (int k = 0; k < K; ++k) {
        uint64_t best = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) best = max(best, key[v]);
        best = largest(best);
        uint32_t at = ~0u;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) at = key[v] == best ? uint32_t(l * V + v) : at;
        at = best ? least(at) : ~0u;
        if (l == k) mine = int(at);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = at == uint32_t(l * V + v) ? 0ull : key[v];
    }
    return mine;
}

// Scores whose quotients are the selected sigmoids', which may all be below the
// smallest number: from -64 down 1 + e^z is 1, and e^(z - top) has their ratios.
__device__ __forceinline__ float sigmoid_of_row(float z, bool renorm) {
    const float top = largest(z);
    return renorm && top < -64.f ? expf(z - top) : 1.f / (1.f + expf(-z));
}

template <bool BF, int V>
__global__ __launch_bounds__(kThreads) void route_scored_kernel(ScoredArgs a) {
    __shared__ uint64_t lk[kWaves][kRows][V * kLanes];
    __shared__ int32_t lc[V * kLanes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (kLanes - 1), r = lane / kLanes;
    if (a.counts) {
        for (int e = threadIdx.x; e < V * kLanes; e += kThreads) lc[e] = 0;
        __syncthreads();
    }
    const int64_t step = int64_t(gridDim.x) * kWaves * kRows;
    for (int64_t t0 = (int64_t(blockIdx.x) * kWaves + wave) * kRows; t0 < a.T; t0 += step) {
        const int64_t t = t0 + r;
        const bool in = t < a.T;
        // rows beyond the batch and masked ones have no candidates
        const uint8_t counts = in && a.mask ? a.mask[t] : uint8_t(in);
        float z[V];
        load_row<BF, V>(a.logits, (in ? t : a.T - 1) * a.ld, a.E, l, z);
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = counts ? z[v] : -INFINITY;
        uint64_t key[V];
        choices64<V>(a, l, z, a.bias != nullptr, key);
        if (a.top_groups < a.groups) {
            uint64_t by[V];
            const bool scores = a.bias || a.group_top == 2;
            if (scores != (a.bias != nullptr)) {
                choices64<V>(a, l, z, scores, by);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) by[v] = key[v];
            }
            keep_groups<V>(a, l, lk[wave][r], by, key);
        }
        const int mine = select64<V>(a.K, l, key);
        // lane k: the weight of selected expert k
        float top = 0.f, total = 1.f, s = 0.f;
        const float zk = mine >= 0 ? logit<BF>(a.logits, t * a.ld + mine) : -INFINITY;
        if (a.sigmoid) {
            s = sigmoid_of_row(zk, a.renorm);
            if (mine < 0) s = 0.f;
        } else {
            top = -INFINITY;
#pragma unroll
            for (int v = 0; v < V; ++v) top = fmaxf(top, z[v]);
            top = largest(top);
            total = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) total += z[v] == -INFINITY ? 0.f : __expf(z[v] - top);
            total = row16::sum(total);
            s = mine >= 0 ? expf(zk - top) : 0.f;
        }
        if (a.renorm) total = row16::sum(s);
        if (in && l < a.K) {
            a.idx[t * a.K + l] = mine;
            a.w[t * a.K + l] = mine >= 0 ? a.scale * (s / total) : 0.f;
        }
        if (a.counts && mine >= 0) atomicAdd(&lc[mine], 1);
    }
    if (a.counts) {
        __syncthreads();
        for (int e = threadIdx.x; e < a.E; e += kThreads)
            if (lc[e]) atomicAdd(&a.counts[e], lc[e]);
    }
}

struct ScoredGradArgs {
    const void* logits;
    int64_t T, ld, ld_d;
    int E, K, sigmoid, renorm;
    float scale;
    const int32_t* idx;
    const float* d_w;
    void* d_logits;
};

// The selected experts' parts, one a lane, go through LDS to the lanes that hold
// those experts.
template <bool BF, int V>
__global__ __launch_bounds__(kThreads) void route_scored_grad_kernel(ScoredGradArgs a) {
    __shared__ float sel[kWaves][kRows][V * kLanes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (kLanes - 1), r = lane / kLanes;
    float* mysel = sel[wave][r];
#pragma unroll
    for (int v = 0; v < V; ++v) mysel[v * kLanes + l] = 0.f;
    const bool dense = !a.sigmoid && !a.renorm;
    const int64_t step = int64_t(gridDim.x) * kWaves * kRows;
    for (int64_t t0 = (int64_t(blockIdx.x) * kWaves + wave) * kRows; t0 < a.T; t0 += step) {
        const int64_t t = t0 + r;
        const bool in = t < a.T;
        int mine = in && l < a.K ? a.idx[t * a.K + l] : -1;
        if (mine >= a.E) mine = -1;
        const float g = mine >= 0 ? a.d_w[t * a.K + l] : 0.f;
        const float zk = mine >= 0 ? logit<BF>(a.logits, t * a.ld + mine) : -INFINITY;
        const bool live = row16::largest(mine) >= 0;
        float z[V], total = 1.f, top;
        if (dense) {
            load_row<BF, V>(a.logits, (in ? t : a.T - 1) * a.ld, a.E, l, z);
            top = -INFINITY;
#pragma unroll
            for (int v = 0; v < V; ++v) top = fmaxf(top, z[v]);
            top = largest(top);
            total = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                z[v] = z[v] == -INFINITY ? 0.f : __expf(z[v] - top);
                total += z[v];
            }
            total = row16::sum(total);
        } else {
            top = a.sigmoid ? 0.f : largest(zk);
        }
        // 1 - s of a sigmoid is the sigmoid of -z
        float s, rest = 1.f;
        if (a.sigmoid) {
            s = sigmoid_of_row(zk, a.renorm);
            if (mine < 0) s = 0.f;
            rest = 1.f / (1.f + expf(zk));
        } else {
            s = mine >= 0 ? expf(zk - top) : 0.f;
        }
        if (a.renorm) total = row16::sum(s);
        const float w = mine >= 0 ? s / total : 0.f;
        const float wg = row16::sum(mine >= 0 ? w * g : 0.f);
        const float d = a.scale * w * (a.renorm ? g - wg : g) * rest;
        // added: an expert that a caller names twice counts twice
        if (mine >= 0) atomicAdd(&mysel[mine], d);
        // a wave's LDS accesses complete in order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const float base = dense ? -a.scale * wg / total : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = l * V + v;
            const float y = live ? mysel[e] + (dense ? z[v] * base : 0.f) : 0.f;
            if (in && e < a.E) {
                if (BF) reinterpret_cast<__bf16*>(a.d_logits)[t * a.ld_d + e] = __bf16(y);
                else reinterpret_cast<float*>(a.d_logits)[t * a.ld_d + e] = y;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (mine >= 0) mysel[mine] = 0.f;
    }
}

// b_e += rate sign(mean of the counts - c_e), for one layer a workgroup; the sums
// are whole numbers.
__global__ __launch_bounds__(256) void route_bias_kernel(int32_t* counts, int E, const float* bias, float* out, float rate,
                                                         int reset) {
    __shared__ long long part[4];
    const int e = threadIdx.x;
    const int64_t at = int64_t(blockIdx.x) * E + e;
    const long long c = e < E ? counts[at] : 0;
    long long all = c;
    for (int d = 32; d; d >>= 1) all += __shfl_xor(all, d, 64);
    if ((e & 63) == 0) part[e >> 6] = all;
    __syncthreads();
    all = part[0] + part[1] + part[2] + part[3];
    if (e >= E) return;
    const long long less = all - c * E;
    out[at] = less > 0 ? bias[at] + rate : less < 0 ? bias[at] - rate : bias[at];
    if (reset) counts[at] = 0;
}

// Calls f(bf16, logits per lane) for E experts.
template <class F>
void with_row(int dtype, int E, F f) {
    const auto lanes = [&](auto bf) {
        if (E <= 16) f(bf, std::integral_constant<int, 1>());
        else if (E <= 32) f(bf, std::integral_constant<int, 2>());
        else if (E <= 64) f(bf, std::integral_constant<int, 4>());
        else if (E <= 128) f(bf, std::integral_constant<int, 8>());
        else f(bf, std::integral_constant<int, 16>());
    };
    if (dtype == STMOE_BF16) lanes(std::true_type());
    else lanes(std::false_type());
}

const char* bad_router(int64_t T, int64_t ld, int E, int K, int dtype, int score, float scale) {
    if (T < 0 || T > (int64_t(1) << 26)) return "T must be in [0, 2^26]";
    if (E < 1 || E > kMaxE) return "E must be in [1, 256]";
    if (K < 1 || K > E || K > kMaxK) return "K must be in [1, min(E, 16)]";
    if (ld < E || ld > (int64_t(1) << 31)) return "the row stride must be in [E, 2^31]";
    if (dtype != STMOE_BF16 && dtype != STMOE_F32) return "dtype must be STMOE_BF16 or STMOE_F32";
    if (score != STMOE_SOFTMAX && score != STMOE_SIGMOID) return "score must be STMOE_SOFTMAX or STMOE_SIGMOID";
    if (!(scale > -INFINITY && scale < INFINITY)) return "scale must be finite";
    return nullptr;
}

}  // namespace

const char* bad_groups(int E, int K, int n_groups, int top_groups, int group_top) {
    if (n_groups < 1 || n_groups > E || E % n_groups) return "n_groups must divide E";
    if (top_groups < 1 || top_groups > n_groups) return "top_groups must be in [1, n_groups]";
    if (group_top != 1 && group_top != 2) return "group_top must be 1 or 2";
    if (K > E / n_groups * top_groups) return "K must not exceed the experts of top_groups groups";
    return nullptr;
}

}  // namespace stmoe

using namespace stmoe;

extern "C" int moe_route_scored(const void* logits, int64_t T, int64_t ld, int E, int K, int dtype, int score,
                                const float* bias, int n_groups, int top_groups, int group_top, int renorm, float scale,
                                const uint8_t* mask, int32_t* topk_idx, float* topk_w, int32_t* counts, void* stream) {
    clear_error();
    if (const char* bad = bad_router(T, ld, E, K, dtype, score, scale)) STMOE_CHECK(false, bad);
    if (const char* bad = bad_groups(E, K, n_groups, top_groups, group_top)) STMOE_CHECK(false, bad);
    if (T == 0) return STMOE_OK;
    STMOE_CHECK(logits && topk_idx && topk_w, "null pointer");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(logits) % (dtype == STMOE_BF16 ? 2 : 4) == 0,
                "logits must be aligned to their elements");
    ScoredArgs a{logits, T, ld, E, K, score == STMOE_SIGMOID, n_groups, top_groups, group_top, renorm ? 1 : 0, scale,
                 bias, mask, topk_idx, topk_w, counts};
    const int64_t per = kWaves * kRows, wg = (T + per - 1) / per;
    const dim3 grid(unsigned(wg < 1024 ? wg : 1024));
    with_row(dtype, E, [&](auto bf, auto v) {
        hipLaunchKernelGGL((route_scored_kernel<bf(), v()>), grid, dim3(kThreads), 0, as_stream(stream), a);
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

extern "C" int moe_route_scored_backward(const void* logits, int64_t T, int64_t ld, int E, int K, int dtype, int score,
                                         int renorm, float scale, const int32_t* topk_idx, const float* d_w,
                                         void* d_logits, int64_t ld_d, void* stream) {
    clear_error();
    if (const char* bad = bad_router(T, ld, E, K, dtype, score, scale)) STMOE_CHECK(false, bad);
    STMOE_CHECK(ld_d >= E && ld_d <= (int64_t(1) << 31), "the gradient's row stride must be in [E, 2^31]");
    if (T == 0) return STMOE_OK;
    STMOE_CHECK(logits && topk_idx && d_w && d_logits, "null pointer");
    const uintptr_t esz = dtype == STMOE_BF16 ? 2 : 4;
    STMOE_CHECK(reinterpret_cast<uintptr_t>(logits) % esz == 0 && reinterpret_cast<uintptr_t>(d_logits) % esz == 0,
                "logits and d_logits must be aligned to their elements");
    ScoredGradArgs a{logits, T, ld, ld_d, E, K, score == STMOE_SIGMOID, renorm ? 1 : 0, scale, topk_idx, d_w, d_logits};
    const int64_t per = kWaves * kRows, wg = (T + per - 1) / per;
    const dim3 grid(unsigned(wg < 1024 ? wg : 1024));
    with_row(dtype, E, [&](auto bf, auto v) {
        hipLaunchKernelGGL((route_scored_grad_kernel<bf(), v()>), grid, dim3(kThreads), 0, as_stream(stream), a);
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

extern "C" int moe_route_bias_step(int32_t* counts, int L, int E, const float* bias, float rate, float* bias_out,
                                   int reset, void* stream) {
    clear_error();
    STMOE_CHECK(L >= 0 && L <= 65535, "L must be in [0, 65535]");
    STMOE_CHECK(E >= 1 && E <= kMaxE, "E must be in [1, 256]");
    if (L == 0) return STMOE_OK;
    STMOE_CHECK(counts && bias && bias_out, "null pointer");
    hipLaunchKernelGGL(route_bias_kernel, dim3(unsigned(L)), dim3(256), 0, as_stream(stream), counts, E, bias, bias_out,
                       rate, reset ? 1 : 0);
    STMOE_LAUNCHED();
    return STMOE_OK;
}
