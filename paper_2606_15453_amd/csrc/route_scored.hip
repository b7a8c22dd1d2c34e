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
// experts whose choices are 1e-7 apart change places, one row in some hundred.  So a
// row is first selected from in 32 bits, with a bound on the choices' errors; where two
// of those it would compare are nearer than that (and not equal by equal logits and
// biases), or it holds a NaN or an infinity, the wave does its rows again in 64 bits.
//
// A row belongs to 16 lanes, four rows to a wave, expert e to lane e mod 16.  The K best
// are found without K rounds: no more than some ten of 256 choices reach the K-th of
// the 16 lanes' best ones; those go to LDS, one to a lane, and 15 rotations rank them
// (32768 x 256 fp32, half of eight groups, top 8: 35 us and 11 for the second launch,
// 104 with K rounds in 64 bits).  What bounds it are its instructions, some 1100 for four
// rows, twice that with groups; the logits' 34 MB alone take 8 us.  The gradient is bound
// by its bytes, 35 MB in 10.6 us, 3.2 TB/s.
#include <type_traits>
#include <utility>

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
    int fill;                      // a row with fewer than K candidates gets other experts, of weight 0
};

template <bool BF>
__device__ __forceinline__ float logit(const void* p, int64_t at) {
    return BF ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(p)[at]) << 16)
              : reinterpret_cast<const float*>(p)[at];
}

// A lane's logits, experts 16 v + l, of the row at element `at`; minus infinity beyond E.
template <bool BF, int V>
__device__ __forceinline__ void load_row(const void* logits, int64_t at, int E, int l, float (&z)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = kLanes * v + l;
        z[v] = e < E ? logit<BF>(logits, at + e) : -INFINITY;
    }
}

__device__ __forceinline__ void wave_lds() {
    // a wave's LDS accesses complete in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The selection of a row in 64 bits: lane k gets the k-th expert (-1: there is none).
// Its loops stay loops, its values in LDS (key, one for every expert) and memory: few
// rows come here, and the others keep their registers.  Batches that come here whole pay for
// it: 32768 rows of equal logits without biases 650 us with 256 experts and 126 with 64 (with
// biases that differ 38 and 22, as any batch), over 16 groups 930 and 290.
template <bool BF, int V>
__device__ __forceinline__ int select64(const ScoredArgs& a, int64_t row, bool live, int l, uint64_t* key) {
    const auto at = [&](int v) {
        const int e = kLanes * v + l;
        return live && e < a.E ? logit<BF>(a.logits, row + e) : -INFINITY;
    };
    double top = 0.0, sum = 1.0;
    if (!a.sigmoid) {
        top = -INFINITY;
#pragma unroll 1
        for (int v = 0; v < V; ++v) top = fmax(top, double(at(v)));
        top = largest(top);
        sum = 0.0;
#pragma unroll 1
        for (int v = 0; v < V; ++v) {
            const double z = at(v);
            sum += z == -INFINITY ? 0.0 : exp(z - top);
        }
        sum = row16::sum(sum);
    }
    // a choice's key; 0 where there is no candidate
    const auto key_at = [&](int v, bool scores) {
        const int e = kLanes * v + l;
        const double z = at(v);
        const float b = a.bias && e < a.E ? a.bias[e] : 0.f;
        if (z == -INFINITY || b == -INFINITY) return uint64_t(0);
        return key64((!scores ? z : a.sigmoid ? 1.0 / (1.0 + exp(-z)) : exp(z - top) / sum) + double(b));
    };
    uint32_t kept = ~0u;
    if (a.top_groups < a.groups) {
        const int size = a.E / a.groups;
#pragma unroll 1
        for (int v = 0; v < V; ++v) key[kLanes * v + l] = key_at(v, a.bias || a.group_top == 2);
        wave_lds();
        for (int g = l; g < a.groups; g += kLanes) {
            uint64_t first = 0, second = 0;
            for (int i = 0; i < size; ++i) {
                const uint64_t k = key[g * size + i];
                second = max(second, min(first, k));
                first = max(first, k);
            }
            // in the place of the group's first choice
            key[g * size] = a.group_top == 2 && second ? key64(value64(first) + value64(second)) : first;
        }
        wave_lds();
        kept = 0u;
#pragma unroll 1
        for (int v = 0; v < V; ++v) {
            const int e = kLanes * v + l, g = e < a.E ? e / size : 0;
            const uint64_t mine = key[g * size];
            int before = 0;
            for (int i = 0; i < a.groups; ++i) {
                const uint64_t other = key[i * size];
                before += other > mine || (other == mine && i < g);
            }
            kept |= uint32_t(before < a.top_groups) << v;
        }
        wave_lds();
    }
#pragma unroll 1
    for (int v = 0; v < V; ++v) key[kLanes * v + l] = (kept >> v) & 1 ? key_at(v, a.bias != nullptr) : 0ull;
    int mine = -1;
#pragma unroll 1
    for (int k = 0; k < a.K; ++k) {
        uint64_t own = 0;
        uint32_t e = ~0u;
#pragma unroll 1
        for (int v = V - 1; v >= 0; --v) {
            const uint64_t o = key[kLanes * v + l];
            e = o >= own ? uint32_t(kLanes * v + l) : e;
            own = max(own, o);
        }
        const uint64_t best = largest(own);
        const uint32_t first = least(own == best && best ? e : ~0u);
        if (l == k) mine = int(first);
        if (first == e && best) key[e] = 0ull;
    }
    return mine;
}

// Scores whose quotients are the selected sigmoids', which may be below the smallest number:
// with a largest logit m below 0, of which they may be any fraction, e^-m times those.
__device__ __forceinline__ float sigmoid_of_row(float z, bool renorm) {
    const float m = renorm ? fminf(largest(z), 0.f) : 0.f;
    const float e = expf(-fabsf(z));
    return (z >= 0.f ? 1.f : m == 0.f ? e : expf(z - m)) / (1.f + e);
}

// A row's room: its choices in 64 bits, the group stage's values, or the candidates of
// the selection (choice in 32 bits, logit, bias, expert; choice in 64), a place of its own
// for what a lane holds beside them; the winners.
template <int V>
struct RowRoom {
    union {
        uint64_t key[V * kLanes];
        double by[V * kLanes + 16];
        struct {
            u32x4 found[3 * kLanes];
            double c[3 * kLanes];
        };
    };
    uint2 sel[kLanes];
};

// f(n) for the rotations n = 1 to N of a row.
template <class F, int... N>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, N...>) {
    (f(std::integral_constant<int, N + 1>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void rotations(F f) { each(f, std::make_integer_sequence<int, N>()); }

// What a choice may be off by in 32 bits.  A sigmoid's exponential has an argument off by
// 2^-23.4 of itself and a last bit, the quotient two: 2.4e-7 at most, as |z| s (1 - s) is
// below 1/4; the sum with the bias 2^-24 of itself.  A softmax's probability p is off by
// its share of an argument of up to 83 (below, p is 0 and equal ones are done again): 1.5e-5 p.
__device__ __forceinline__ float slack(bool sigmoid, float s, float c) {
    return sigmoid ? 3.4e-7f * (1.f + fabsf(c)) : 0x1p-16f * s + 0x1p-22f * fabsf(c);
}

__device__ __forceinline__ float exp_of(float x) { return __expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }
__device__ __forceinline__ float inverse(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ double inverse(double x) { return 1.0 / x; }

// Ranks a row's n candidates, N a lane, and leaves the first K in room.sel.  Equal ones
// are in order of their experts.  In 32 bits, true where two are nearer than their
// choices' slack without equal logits and biases, and a softmax's sum is not known in 64.
template <class F, int V, int N>
__device__ __forceinline__ bool rank(const ScoredArgs& a, RowRoom<V>& room, int n, int l, bool exact) {
    constexpr bool F32 = sizeof(F) == 4;
    F c[N];
    float z[N], b[N], off[N];
    int e[N], before[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const u32x4 q = room.found[kLanes * i + l];
        const bool is = kLanes * i + l < n;
        if constexpr (F32) c[i] = is ? __uint_as_float(q[0]) : -INFINITY;
        else c[i] = is ? room.c[kLanes * i + l] : -INFINITY;
        z[i] = __uint_as_float(q[1]);
        b[i] = __uint_as_float(q[2]);
        e[i] = int(q[3]);
        off[i] = !is ? -1.f : exact || !F32 ? 0.f : 2.0625f * slack(a.sigmoid, fabsf(float(c[i]) - b[i]), float(c[i]));
        before[i] = 0;
    }
    // in 64 bits near ones are equal ones
    bool near = false;
    const auto against = [&](int i, F o) {
        before[i] += o > c[i];
        if constexpr (F32) near |= fabsf(o - c[i]) <= off[i];
        else near |= o == c[i] && o != -INFINITY;
    };
    rotations<15>([&](auto m) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const F o = rotate<m()>(c[j]);
#pragma unroll
            for (int i = 0; i < N; ++i) against(i, o);
        }
    });
    if constexpr (N == 2) {
        against(0, c[1]);
        against(1, c[0]);
    }
    bool other = false;
    if (__any(near)) {
        const auto tied = [&](int i, F oc, float oz, float ob, int oe) {
            before[i] += oc == c[i] && oe < e[i];
            if constexpr (F32) other |= fabsf(oc - c[i]) <= off[i] && !(oz == z[i] && ob == b[i]);
        };
        rotations<15>([&](auto m) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                // every lane takes part in a rotation: none behind a condition of its own
                const F oc = rotate<m()>(c[j]);
                const float oz = rotate<m()>(z[j]), ob = rotate<m()>(b[j]);
                const int oe = rotate<m()>(e[j]);
#pragma unroll
                for (int i = 0; i < N; ++i) tied(i, oc, oz, ob, oe);
            }
        });
        if constexpr (N == 2) {
            tied(0, c[1], z[1], b[1], e[1]);
            tied(1, c[0], z[0], b[0], e[0]);
        }
    }
    other = other && !exact;
    if constexpr (F32)
        if (a.sigmoid && __any(other)) {
            // a candidate's choice in 64 bits takes its own logit and bias alone
            double d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                d[i] = kLanes * i + l < n ? 1.0 / (1.0 + exp(-double(z[i]))) + double(b[i]) : -INFINITY;
                before[i] = 0;
            }
            const auto less = [&](int i, double o, int oe) { before[i] += o > d[i] || (o == d[i] && oe < e[i]); };
            rotations<15>([&](auto m) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const double o = rotate<m()>(d[j]);
                    const int oe = rotate<m()>(e[j]);
#pragma unroll
                    for (int i = 0; i < N; ++i) less(i, o, oe);
                }
            });
            if constexpr (N == 2) {
                less(0, d[1], e[1]);
                less(1, d[0], e[0]);
            }
            other = false;
        }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (kLanes * i + l < n && before[i] < a.K) room.sel[before[i]] = make_uint2(uint32_t(e[i]), __float_as_uint(z[i]));
    return other;
}

// What a lane keeps for all rows.
template <int V>
struct Mine {
    float bias[V];
    uint32_t group[(V + 7) / 8];   // four bits a value
    __device__ __forceinline__ uint32_t of(int v) const { return group[v / 8] >> (4 * (v % 8)) & 15u; }
};

// Selects from a row of logits z: lane k gets the k-th expert and its logit (-1, minus
// infinity: there is none); top and total: the softmax's.  True where it takes 64 bits,
// or, in those, the plain selection (NaN and infinities, over 16 groups, over 32
// candidates that are not below the K-th of the lanes' best ones).
template <class F, int V>
__device__ __forceinline__ bool select(const ScoredArgs& a, RowRoom<V>& room, const Mine<V>& own, int l, int r,
                                       const float (&z)[V], float& top, float& total, int& mine, float& zk) {
    constexpr bool F32 = sizeof(F) == 4;
    const bool grouped = a.top_groups < a.groups, exact = a.bias == nullptr;
    const bool by_scores = !exact || (grouped && a.group_top == 2), in32 = !grouped || a.groups <= kLanes;
    // scores, and what chooses: of experts (c), and of groups
    F s[V], c[V];
    top = 0.f;
    total = 1.f;
    if (!a.sigmoid) {
        top = z[0];
#pragma unroll
        for (int v = 1; v < V; ++v) top = fmaxf(top, z[v]);
        top = largest(top);
        const F from = top == -INFINITY ? 0.f : top;
        F sum = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[v] = exp_of(F(z[v]) - from);
            sum += s[v];
        }
        sum = row16::sum(sum);
        total = float(sum);
        if (by_scores) {
            const F inv = sum > 0 ? 1 / sum : sum;         // NaN stays
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] = F32 ? s[v] * inv : sum > 0 ? s[v] / sum : inv;
        }
    } else if (by_scores) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = inverse(1 + exp_of(-F(z[v])));
    }
    if (by_scores)
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = z[v] == -INFINITY ? F(-INFINITY) : s[v] + F(own.bias[v]);
    bool again = !in32;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = exact ? F(z[v]) : s[v];
        again |= !(c[v] < F(INFINITY));
    }
    if (grouped && in32) {
        const int size = a.E / a.groups;
        // up to eight groups have two lanes each
        const bool pairs = a.groups <= 8;
        const int g = pairs ? l & 7 : l;
        F* const by = reinterpret_cast<F*>(room.by);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = kLanes * v + l;
            by[e < a.E ? e + int(own.of(v)) : V * kLanes + 15] = by_scores ? s[v] : c[v];
        }
        wave_lds();
        F first = -INFINITY, second = -INFINITY;
        if (g < a.groups) {
#pragma unroll 8
            for (int i = pairs ? l >> 3 : 0; i < size; i += pairs ? 2 : 1) {
                const F k = by[g * (size + 1) + i];
                second = fmax(second, fmin(first, k));
                first = fmax(first, k);
            }
        }
        if (pairs) {
            const F o1 = rotate<8>(first), o2 = rotate<8>(second);
            second = fmax(fmax(second, o2), fmin(first, o1));
            first = fmax(first, o1);
        }
        const bool both = a.group_top == 2 && second != F(-INFINITY);
        const F sum = both ? first + second : first;
        // two numbers whose sum is none in 32 bits
        if constexpr (F32) again |= both && !(fabsf(sum) < INFINITY);
        // the terms' slack, each by its own size: terms of opposite sign leave a small sum of two
        // large errors.  What slack has of |c| holds the sum's rounding too
        float off = 0.f;
        if constexpr (F32) {
            const float p = a.sigmoid ? 0.f : 1.f / total;
            if (first != F(-INFINITY)) off = 1.03125f * slack(a.sigmoid, p, first);
            if (both) off += 1.03125f * slack(a.sigmoid, p, second);
        }
        int before = 0;
        bool near = false;
        const auto against = [&](auto n) {
            const F other = rotate<n()>(sum);
            const int at = rotate<n()>(g);
            before += other > sum || (other == sum && at < g);
            if constexpr (F32) near |= fabsf(other - sum) <= off + rotate<n()>(off);
        };
        if (pairs) rotations<7>(against);
        else rotations<15>(against);
        if (F32 && by_scores && __any(near)) {
            // it matters between a group that is kept and one that is not
            rotations<15>([&](auto n) {
                const F other = rotate<n()>(sum);
                const int there = rotate<n()>(before);
                const float offs = off + rotate<n()>(off);
                again |= fabsf(float(other - sum)) <= offs && (there < a.top_groups) != (before < a.top_groups);
            });
        }
        const uint32_t kept = uint32_t(__ballot(before < a.top_groups) >> (kLanes * r));
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (F32) {
                const uint32_t keep = uint32_t(__builtin_amdgcn_sbfe(int(kept), own.of(v), 1));
                c[v] = __uint_as_float((__float_as_uint(c[v]) & keep) | (0xff800000u & ~keep));
            } else {
                c[v] = (kept >> own.of(v)) & 1u ? c[v] : F(-INFINITY);
            }
        }
        wave_lds();
    }
    // candidates: all that are not below the K-th of the lanes' best ones
    F best = c[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = fmax(best, c[v]);
    int above = 0;
    rotations<15>([&](auto n) { above += rotate<n()>(best) > best; });
    const F limit = -largest(above < a.K ? -best : F(-INFINITY));
    F edge = limit;
    if (F32 && !exact) {
        best = largest(best);
        edge -= 2.f * slack(a.sigmoid, a.sigmoid ? 0.f : 1.f / total, fmaxf(fabsf(float(best)), fabsf(float(limit))));
    }
    edge = fmax(edge, F(-3.402823466e38f));        // minus infinity is none (NaN: all rows again)
    int own_n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) own_n += c[v] >= edge;
    int place = own_n;
    place += __builtin_amdgcn_update_dpp(0, place, 0x111, 0xf, 0xf, false);
    place += __builtin_amdgcn_update_dpp(0, place, 0x112, 0xf, 0xf, false);
    place += __builtin_amdgcn_update_dpp(0, place, 0x114, 0xf, 0xf, false);
    place += __builtin_amdgcn_update_dpp(0, place, 0x118, 0xf, 0xf, false);
    const int n = __shfl(place, r * kLanes + kLanes - 1, 64);
    again |= n > 2 * kLanes;
    place -= own_n;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool is = c[v] >= edge;
        const int to = is && place < 2 * kLanes ? place : 2 * kLanes + l;
        room.found[to] = u32x4{__float_as_uint(float(c[v])), __float_as_uint(z[v]), __float_as_uint(own.bias[v]),
                               uint32_t(kLanes * v + l)};
        if constexpr (!F32) room.c[to] = c[v];
        place += is;
    }
    room.sel[l] = make_uint2(~0u, 0xff800000u);
    wave_lds();
    if (__any(n > kLanes)) again |= rank<F, V, 2>(a, room, n, l, exact);
    else again |= rank<F, V, 1>(a, room, n, l, exact);
    wave_lds();
    const uint2 won = room.sel[l];
    mine = l < a.K ? int(won.x) : -1;
    zk = mine >= 0 ? __uint_as_float(won.y) : -INFINITY;
    wave_lds();
    return __any(again);
}

// Small batches select in 32 bits and at once again in 64 where that takes it (kBoth).
// In large ones rows done again would hold up the others of their waves, and that code's
// registers halve the waves a CU holds: kFirst marks such rows' first expert, kAgain
// looks for the marks and selects there.  us in one launch, in two (256 experts, eight
// groups): 4096 tokens 14.4, 20.2; 8192 22.6, 20.7; 32768 67.6, 41.0.
enum { kBoth, kFirst, kAgain };
constexpr int kMark = -2;
constexpr int64_t kSmall = 6144;   // tokens

template <bool BF, int V, int MODE>
__global__ __launch_bounds__(kThreads) void route_scored_kernel(ScoredArgs a) {
    __shared__ RowRoom<V> rooms[kWaves][kRows];
    __shared__ int32_t lc[V * kLanes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (kLanes - 1), r = lane / kLanes;
    RowRoom<V>& room = rooms[wave][r];
    if (a.counts) {
        for (int e = threadIdx.x; e < V * kLanes; e += kThreads) lc[e] = 0;
        __syncthreads();
    }
    const int size = a.E / a.groups;
    Mine<V> own;
#pragma unroll
    for (int v = 0; v < V; v += 8) own.group[v / 8] = 0u;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = kLanes * v + l;
        own.bias[v] = a.bias && e < a.E ? a.bias[e] : 0.f;
        if (a.top_groups < a.groups && a.groups <= kLanes && e < a.E) own.group[v / 8] |= uint32_t(e / size) << (4 * (v % 8));
    }
    // four rows from t0 on, in 32 or in 64 bits
    const auto rows = [&](int64_t t0, bool first, bool again) __attribute__((always_inline)) {
        const int64_t t = t0 + r;
        const bool in = t < a.T;
        // rows beyond the batch and masked ones have no candidates
        const uint8_t live = in && a.mask ? a.mask[t] : uint8_t(in);
        const int64_t row = (in ? t : a.T - 1) * a.ld;
        float z[V], top, total, zk;
        load_row<BF, V>(a.logits, row, a.E, l, z);
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = live ? z[v] : -INFINITY;
        int mine;
        bool more = true;
        if (first) more = select<float, V>(a, room, own, l, r, z, top, total, mine, zk);
        if (more) {
            if (!again) {
                if (in && l == 0) a.idx[t * a.K] = kMark;
                return;
            }
            if (select<double, V>(a, room, own, l, r, z, top, total, mine, zk)) {
                mine = select64<BF, V>(a, row, live, l, room.key);
                if (l >= a.K) mine = -1;
                zk = mine >= 0 ? logit<BF>(a.logits, row + mine) : -INFINITY;
                wave_lds();
            }
        }
        // lane k: the weight of selected expert k
        float w;
        if (a.sigmoid) {
            w = sigmoid_of_row(zk, a.renorm);
            if (mine < 0) w = 0.f;
        } else {
            // renormalised: from the selected ones' largest; the row's may be any distance above
            if (a.renorm) top = largest(zk);
            w = mine >= 0 ? expf(zk - top) : 0.f;
        }
        // a softmax's sum that is NaN makes its row NaN, also where what is selected has none
        if (a.renorm) total = total != total ? total : row16::sum(w);
        w = mine >= 0 ? a.scale * (w / total) : 0.f;
        if (a.fill && __any(in && l < a.K && mine < 0))
            for (int e = 0; e < a.E; ++e) {
                // the row's first free place takes the lowest expert it has not
                const uint32_t has = uint32_t(__ballot(mine == e) >> (kLanes * r)) & 0xffffu;
                const uint32_t free = uint32_t(__ballot(l < a.K && mine < 0) >> (kLanes * r)) & 0xffffu;
                if (!has && free && l == __ffs(int(free)) - 1) mine = e;
            }
        if (in && l < a.K) {
            a.idx[t * a.K + l] = mine;
            a.w[t * a.K + l] = w;
        }
        if (a.counts && mine >= 0) atomicAdd(&lc[mine], 1);
    };
    const int64_t step = int64_t(gridDim.x) * kWaves * (MODE == kAgain ? 64 : kRows);
    for (int64_t t0 = (int64_t(blockIdx.x) * kWaves + wave) * (MODE == kAgain ? 64 : kRows); t0 < a.T; t0 += step) {
        if constexpr (MODE == kAgain) {
            uint64_t marked = __ballot(t0 + lane < a.T && a.idx[(t0 + lane) * a.K] == kMark);
            while (marked) {
                const int at = (__ffsll((unsigned long long)marked) - 1) / kRows * kRows;
                rows(t0 + at, false, true);
                marked &= ~(15ull << at);
            }
        } else {
            rows(t0, true, MODE == kBoth);
        }
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
            const int e = kLanes * v + l;
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

int launch_scored(const ScoredArgs& a, int dtype, hipStream_t s) {
    const int64_t per = kWaves * kRows, wg = (a.T + per - 1) / per, marks = (a.T + 64 * kWaves - 1) / (64 * kWaves);
    const auto most = [](int64_t n, int64_t m) { return dim3(unsigned(n < m ? n : m)); };
    // 512 workgroups, as many as the CUs hold, in the large form (1024: 5 us more, of
    // their counts' atomics above all)
    with_row(dtype, a.E, [&](auto bf, auto v) {
        if (a.T <= kSmall) {
            hipLaunchKernelGGL((route_scored_kernel<bf(), v(), kBoth>), most(wg, 1024), dim3(kThreads), 0, s, a);
        } else {
            hipLaunchKernelGGL((route_scored_kernel<bf(), v(), kFirst>), most(wg, 512), dim3(kThreads), 0, s, a);
            hipLaunchKernelGGL((route_scored_kernel<bf(), v(), kAgain>), most(marks, 512), dim3(kThreads), 0, s, a);
        }
    });
    STMOE_LAUNCHED();
    return STMOE_OK;
}

}  // namespace

// Rows of fp32 logits [B][E] for the decode path: every row gets K experts.  Shapes are
// validated by the caller.
int route_scored_rows(const float* z, int B, int E, int K, int score, const float* bias, int n_groups, int top_groups,
                      int group_top, int renorm, float scale, int32_t* idx, float* w, hipStream_t s) {
    return launch_scored(ScoredArgs{z, B, E, E, K, score == STMOE_SIGMOID, n_groups, top_groups, group_top, renorm, scale,
                                    bias, nullptr, idx, w, nullptr, 1},
                         STMOE_F32, s);
}

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
    return launch_scored(ScoredArgs{logits, T, ld, E, K, score == STMOE_SIGMOID, n_groups, top_groups, group_top,
                                    renorm ? 1 : 0, scale, bias, mask, topk_idx, topk_w, counts, 0},
                         dtype, as_stream(stream));
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
