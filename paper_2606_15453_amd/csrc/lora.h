// Low-rank adapters: what the general kernels (lora.hip) and those for bf16 rows in
// whole 16-byte chunks (lora_bf16.hip) share.
#pragma once

#include "lora_plan.h"

namespace stmoe {
namespace lora {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Args {
    Plan plan;
    const void* plan_at;           // the whole plan (host)
    int T, n, R;
    const int32_t* ranks;          // [n] or null: all R
    const float* scales;           // [n] or null: 1
};

__device__ __forceinline__ bool planned(const Args& g) { return g.plan.head->T == g.T && g.plan.head->n == g.n; }
// Tile i of the table; false where the plan has none.  The tile is loaded beside the
// plan's head: i is below the table's room.
__device__ __forceinline__ bool tile_of(const Args& g, int i, Tile& t) {
    const int T = g.plan.head->T, n = g.plan.head->n, tiles = *g.plan.tiles_n;
    t = g.plan.tiles[i];
    return T == g.T && n == g.n && i < tiles;
}
__device__ __forceinline__ int rank_of(const Args& g, int a) {
    const int r = g.ranks ? g.ranks[a] : g.R;
    return r < 0 ? 0 : r < g.R ? r : g.R;
}

struct ShrinkArgs {
    Args g;
    const void* x;                 // [T] rows of C values, row stride ld
    int64_t ld;
    int C;
    const void* const* m;          // [n] matrices [r][C]
    int scaled;                    // by the adapter's scale
    float* v;                      // [T][R]; columns beyond the rank get 0
    int parts;                     // of the columns: v is [parts][T][R] then
};

struct ExpandArgs {
    Args g;
    const float* v;                // [parts][T][R], to be summed
    int parts;
    float* v_out;                  // [T][R] the sum, or null
    const void* const* m;          // [n] matrices [r][C]
    int C, scaled;
    const void* base;              // [T] rows of C values, row stride ld_base, or null: 0
    int64_t ld_base;
    void* y;                       // out, row stride ld
    int64_t ld;
};

// The sum of v's parts (an even number) for a tile's tokens, shared among the `of`
// workgroups that hold the tile's columns: one for all was the launch's last by far
// (4096 x 4096, rank 64, two parts: 33.7 us, 23.7 so).
__device__ __forceinline__ void sum_parts(const ExpandArgs& a, const int32_t* order, int count, int nth, int of) {
    const int64_t part = int64_t(a.g.T) * a.g.R;
    for (int i = nth * int(blockDim.x) + threadIdx.x; i < count * a.g.R; i += of * int(blockDim.x)) {
        const int k = i / a.g.R;
        const int64_t at = int64_t(order[k]) * a.g.R + (i - k * a.g.R);
        float sum = 0.f;
        for (int p = 0; p < a.parts; p += 2) {
            const float v0 = a.v[p * part + at], v1 = a.v[(p + 1) * part + at];
            sum += v0;
            sum += v1;
        }
        a.v_out[at] = sum;
    }
}

struct OuterArgs {
    Args g;
    const void* x;                 // [T] rows of C values, row stride ld
    int64_t ld;
    int C;
    const float* u;                // [T][R]
    int scaled;
    float* const* d;               // [n] gradients [r][C], out
    float* part;                   // [outer_slots][R][C] sums of tiles of adapters with several
};

// A tile's place among the sums of adapters with several tiles: two of their tiles
// start within `size` tokens only if the first is an adapter's last.
__host__ __device__ inline int outer_slot(int first, int size, bool last) { return 2 * (first / size) + last; }
inline size_t outer_slots(int T, int size) { return 2 * (size_t(T) / size + 1); }

// One of two calls' arguments, field by field: a reference to either would put both into
// scratch memory (lora_outer_bf16_kernel 31 us for it, not 21, lora_join_kernel 13.4, not 4.9).
__device__ __forceinline__ OuterArgs one_of(bool second, const OuterArgs& p, const OuterArgs& o) {
    OuterArgs a = p;
    a.x = second ? o.x : p.x;
    a.ld = second ? o.ld : p.ld;
    a.C = second ? o.C : p.C;
    a.u = second ? o.u : p.u;
    a.scaled = second ? o.scaled : p.scaled;
    a.d = second ? o.d : p.d;
    a.part = second ? o.part : p.part;
    return a;
}

// lora_bf16.hip
int outer_bf16(const OuterArgs (&a)[2], int table, hipStream_t s);
int shrink_bf16(const ShrinkArgs& a, int table, hipStream_t s);
int expand_bf16(const ExpandArgs& a, int table, bool ybf, hipStream_t s);

inline Args with_table(Args g, int table) {
    g.plan = plan_of(g.plan_at, g.T, g.n, table);
    return g;
}

inline bool chunks16(const void* p, int64_t ld, int C, int esz) {
    return C % (16 / esz) == 0 && ld * esz % 16 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

}  // namespace lora
}  // namespace stmoe
