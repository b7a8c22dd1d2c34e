// The plan of a batch with low-rank adapters (lora_plan.h): a stable counting sort
// of the tokens by adapter.  Up to 1024 tokens one launch of one workgroup; beyond,
// a workgroup per 1024 tokens ranks its own, one adds their counts up and writes
// the tiles, and a third launch writes the order.  Made once for a batch, used by
// every projection of every layer: 8 us for 64 tokens, 17 for 8192.
#include "lora_plan.h"

namespace stmoe {
namespace {

using namespace lora;

struct PlanArgs {
    const int32_t* adapter;        // [T]
    int T, n;
    char* plan;
};

__device__ __forceinline__ int key_of(const PlanArgs& a, int t) {
    const int k = a.adapter[t];
    return k >= 0 && k < a.n ? k : a.n;
}

// Ranks the workgroup's token among those before it with the same key; hist [n + 1]
// (LDS) holds the counts afterwards.
__device__ __forceinline__ int rank_tokens(int key, bool in, int n, int* hist) {
    for (int k = threadIdx.x; k <= n; k += kPlanThreads) hist[k] = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the wave's lanes with this key
    uint64_t same = __ballot(in);
    for (int b = 0; (n >> b) != 0; ++b) {
        const uint64_t one = __ballot((key >> b) & 1);
        same &= ((key >> b) & 1) ? one : ~one;
    }
    const int within = __popcll(same & ((1ull << lane) - 1)), all = __popcll(same);
    int rank = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        __syncthreads();
        if (w == wave && in) {
            const int before = hist[key];
            rank = before + within;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (within == 0) hist[key] = before + all;
        }
    }
    __syncthreads();
    return rank;
}

// Exclusive sum over the workgroup's threads; *all: the sum of all.
__device__ __forceinline__ int exclusive(int v, int* part, int* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(s, d, 64);
        if (lane >= d) s += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = s;
    __syncthreads();
    int before = 0, sum = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        before += w < wave ? part[w] : 0;
        sum += part[w];
    }
    *all = sum;
    return before + s - v;
}

// From the counts of every key (LDS; overwritten by its first position) the segments
// and the tiles.
__device__ __forceinline__ void write_tables(const PlanArgs& a, int* count, int* part) {
    const PlanLayout y = plan_layout(a.T, a.n);
    int32_t* seg = reinterpret_cast<int32_t*>(a.plan + y.seg);
    PlanHead* head = reinterpret_cast<PlanHead*>(a.plan);
    const int per = (a.n + 1 + kPlanThreads - 1) / kPlanThreads, k0 = threadIdx.x * per;
    for (int s = 0; s < kTables; ++s) {
        int32_t* base = reinterpret_cast<int32_t*>(a.plan + y.base[s]);
        const int size = tile_tokens(s);
        int mine = 0, all;
        for (int k = k0; k < k0 + per && k <= a.n; ++k) mine += (count[k] + size - 1) / size;
        int at = exclusive(mine, part, &all);
        for (int k = k0; k < k0 + per && k <= a.n; ++k) {
            base[k] = at;
            at += (count[k] + size - 1) / size;
        }
        if (threadIdx.x == 0) {
            base[a.n + 1] = all;
            head->tiles[s] = all;
        }
    }
    int mine = 0, all;
    for (int k = k0; k < k0 + per && k <= a.n; ++k) mine += count[k];
    int at = exclusive(mine, part, &all);
    for (int k = k0; k < k0 + per && k <= a.n; ++k) {
        const int c = count[k];
        count[k] = at;
        seg[k] = at;
        at += c;
    }
    if (threadIdx.x == 0) {
        seg[a.n + 1] = a.T;
        count[a.n + 1] = a.T;
        head->T = a.T;
        head->n = a.n;
    }
    __threadfence_block();
    __syncthreads();
    for (int s = 0; s < kTables; ++s) {
        const int32_t* base = reinterpret_cast<const int32_t*>(a.plan + y.base[s]);
        Tile* tiles = reinterpret_cast<Tile*>(a.plan + y.tiles[s]);
        const int size = tile_tokens(s), all_s = base[a.n + 1];
        for (int i = threadIdx.x; i < all_s; i += kPlanThreads) {
            int lo = 0, hi = a.n;                  // the last key whose tiles start at or before i
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (base[mid] <= i) lo = mid;
                else hi = mid - 1;
            }
            Tile t;
            t.adapter = lo < a.n ? lo : -1;
            t.piece = i - base[lo];
            t.first = count[lo] + t.piece * size;
            const int left = count[lo + 1] - t.first;
            t.count = left < size ? left : size;
            tiles[i] = t;
        }
    }
}

__global__ __launch_bounds__(kPlanThreads) void lora_plan_one_kernel(PlanArgs a) {
    __shared__ int hist[kMaxAdapters + 2];
    __shared__ int part[kPlanThreads / 64];
    const PlanLayout y = plan_layout(a.T, a.n);
    const int t = threadIdx.x;
    const bool in = t < a.T;
    const int key = in ? key_of(a, t) : 0;
    const int rank = rank_tokens(key, in, a.n, hist);
    write_tables(a, hist, part);
    if (in) reinterpret_cast<int32_t*>(a.plan + y.order)[hist[key] + rank] = t;
}

__global__ __launch_bounds__(kPlanThreads) void lora_plan_rank_kernel(PlanArgs a) {
    __shared__ int hist[kMaxAdapters + 2];
    const PlanLayout y = plan_layout(a.T, a.n);
    const int t = blockIdx.x * kPlanThreads + threadIdx.x;
    const bool in = t < a.T;
    const int rank = rank_tokens(in ? key_of(a, t) : 0, in, a.n, hist);
    if (in) reinterpret_cast<int32_t*>(a.plan + y.rank)[t] = rank;
    int32_t* out = reinterpret_cast<int32_t*>(a.plan + y.hist) + size_t(blockIdx.x) * (a.n + 1);
    for (int k = threadIdx.x; k <= a.n; k += kPlanThreads) out[k] = hist[k];
}

__global__ __launch_bounds__(kPlanThreads) void lora_plan_sum_kernel(PlanArgs a) {
    __shared__ int count[kMaxAdapters + 2];
    __shared__ int part[kPlanThreads / 64];
    const PlanLayout y = plan_layout(a.T, a.n);
    int32_t* hist = reinterpret_cast<int32_t*>(a.plan + y.hist);
    for (int k = threadIdx.x; k <= a.n; k += kPlanThreads) {
        int sum = 0;
        for (int b = 0; b < y.blocks; ++b) {
            const size_t at = size_t(b) * (a.n + 1) + k;
            const int c = hist[at];
            hist[at] = sum;
            sum += c;
        }
        count[k] = sum;
    }
    __syncthreads();
    write_tables(a, count, part);
}

__global__ __launch_bounds__(kPlanThreads) void lora_plan_order_kernel(PlanArgs a) {
    const PlanLayout y = plan_layout(a.T, a.n);
    const int t = blockIdx.x * kPlanThreads + threadIdx.x;
    if (t >= a.T) return;
    const int key = key_of(a, t);
    const int at = reinterpret_cast<const int32_t*>(a.plan + y.seg)[key] +
                   reinterpret_cast<const int32_t*>(a.plan + y.hist)[size_t(blockIdx.x) * (a.n + 1) + key] +
                   reinterpret_cast<const int32_t*>(a.plan + y.rank)[t];
    reinterpret_cast<int32_t*>(a.plan + y.order)[at] = t;
}

}  // namespace
}  // namespace stmoe

using namespace stmoe;

extern "C" size_t moe_lora_plan_bytes(int T, int n_adapters) {
    if (T < 0 || T > lora::kMaxTokens || n_adapters < 1 || n_adapters > lora::kMaxAdapters) return 0;
    return lora::plan_layout(T, n_adapters).total;
}

extern "C" int moe_lora_plan(const int32_t* adapter, int T, int n_adapters, void* plan, size_t plan_bytes, void* stream) {
    clear_error();
    STMOE_CHECK(T >= 0 && T <= lora::kMaxTokens, "T must be in [0, 65536]");
    STMOE_CHECK(n_adapters >= 1 && n_adapters <= lora::kMaxAdapters, "n_adapters must be in [1, 4096]");
    if (T == 0) return STMOE_OK;
    STMOE_CHECK(adapter && plan, "null pointer");
    STMOE_CHECK(plan_bytes >= moe_lora_plan_bytes(T, n_adapters), "plan too small");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(plan) % 256 == 0, "plan must be 256-byte aligned");
    STMOE_CHECK(reinterpret_cast<uintptr_t>(adapter) % 4 == 0, "adapter must be aligned to its elements");
    const PlanArgs a{adapter, T, n_adapters, reinterpret_cast<char*>(plan)};
    hipStream_t s = as_stream(stream);
    const int blocks = lora::plan_layout(T, n_adapters).blocks;
    if (blocks == 1) {
        hipLaunchKernelGGL(lora_plan_one_kernel, dim3(1), dim3(lora::kPlanThreads), 0, s, a);
        STMOE_LAUNCHED();
        return STMOE_OK;
    }
    hipLaunchKernelGGL(lora_plan_rank_kernel, dim3(unsigned(blocks)), dim3(lora::kPlanThreads), 0, s, a);
    STMOE_LAUNCHED();
    hipLaunchKernelGGL(lora_plan_sum_kernel, dim3(1), dim3(lora::kPlanThreads), 0, s, a);
    STMOE_LAUNCHED();
    hipLaunchKernelGGL(lora_plan_order_kernel, dim3(unsigned(blocks)), dim3(lora::kPlanThreads), 0, s, a);
    STMOE_LAUNCHED();
    return STMOE_OK;
}
