// The plan of a batch with low-rank adapters: the tokens in the order of their
// adapters (a stable sort), and tiles of tokens that have one adapter.
#pragma once

#include "common.h"

namespace stmoe {
namespace lora {

constexpr int kMaxTokens = 65536;
constexpr int kMaxAdapters = 4096;
constexpr int kMaxRank = 128;
constexpr int kMaxCols = 65536;
constexpr int kPlanThreads = 1024;         // tokens that one workgroup sorts

// tokens per tile of the tables: two for the products of single tokens, two for sums
// over tokens
constexpr int kTables = 4;
__host__ __device__ constexpr int tile_tokens(int s) { return 16 << (2 * s); }

struct Tile {
    int32_t adapter;               // -1: tokens without one
    int32_t first, count;          // in the sorted order
    int32_t piece;                 // the tile's number among its adapter's
};

// Offsets in bytes of the plan of T tokens and n adapters (n stands for tokens without one).
struct PlanLayout {
    int blocks, max_tiles[kTables];
    size_t seg, order, rank, hist, base[kTables], tiles[kTables], total;
};

// The first words of a plan.
struct PlanHead {
    int32_t T, n, tiles[kTables];
};

__host__ __device__ inline PlanLayout plan_layout(int T, int n) {
    PlanLayout y{};
    size_t off = 256;
    auto take = [&](size_t b) { const size_t at = off; off = (off + b + 255) / 256 * 256; return at; };
    y.blocks = (T + kPlanThreads - 1) / kPlanThreads;
    y.seg = take(size_t(n + 2) * 4);
    y.order = take(size_t(T) * 4);
    y.rank = take(size_t(T) * 4);
    y.hist = take(size_t(y.blocks) * (n + 1) * 4);
    for (int s = 0; s < kTables; ++s) {
        y.max_tiles[s] = T / tile_tokens(s) + (T < n + 1 ? T : n + 1);
        y.base[s] = take(size_t(n + 2) * 4);
        y.tiles[s] = take(size_t(y.max_tiles[s]) * sizeof(Tile));
    }
    y.total = off;
    return y;
}

// What the kernels read of a plan: one of its tables.
struct Plan {
    const PlanHead* head;
    const int32_t* tiles_n;        // [1] tiles of the table
    const int32_t* seg;            // [n + 2] first position of every adapter; T
    const int32_t* order;          // [T] token at every position
    const int32_t* base;           // [n + 2] first tile of every adapter
    const Tile* tiles;
    int size;                      // tokens per tile
};

inline Plan plan_of(const void* plan, int T, int n, int table) {
    const PlanLayout y = plan_layout(T, n);
    const char* p = reinterpret_cast<const char*>(plan);
    Plan o{};
    o.head = reinterpret_cast<const PlanHead*>(p);
    o.tiles_n = o.head->tiles + table;
    o.seg = reinterpret_cast<const int32_t*>(p + y.seg);
    o.order = reinterpret_cast<const int32_t*>(p + y.order);
    o.base = reinterpret_cast<const int32_t*>(p + y.base[table]);
    o.tiles = reinterpret_cast<const Tile*>(p + y.tiles[table]);
    o.size = tile_tokens(table);
    return o;
}

}  // namespace lora
}  // namespace stmoe
