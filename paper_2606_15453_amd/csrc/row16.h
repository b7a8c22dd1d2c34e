// A row of values held by 16 lanes, a row of the vector unit, four rows a wave:
// rotations, sums and maxima within the row, and the order of candidates as keys.
#pragma once

#include "common.h"

namespace stmoe {
namespace row16 {

constexpr int kLanes = 16;
constexpr int kRows = 64 / kLanes;         // rows a wave works on

template <int N>
__device__ __forceinline__ uint32_t rotate(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(int(v), int(v), 0x120 + N, 0xf, 0xf, false));
}
template <int N>
__device__ __forceinline__ int rotate(int v) { return int(rotate<N>(uint32_t(v))); }
template <int N>
__device__ __forceinline__ float rotate(float v) { return __uint_as_float(rotate<N>(__float_as_uint(v))); }
template <int N>
__device__ __forceinline__ uint64_t rotate(uint64_t v) {
    return uint64_t(rotate<N>(uint32_t(v >> 32))) << 32 | rotate<N>(uint32_t(v));
}
template <int N>
__device__ __forceinline__ double rotate(double v) {
    return __longlong_as_double((long long)rotate<N>(uint64_t(__double_as_longlong(v))));
}

template <class T>
__device__ __forceinline__ T sum(T v) {
    v += rotate<8>(v);
    v += rotate<4>(v);
    v += rotate<2>(v);
    return v + rotate<1>(v);
}
template <class T>
__device__ __forceinline__ T largest(T v) {
    v = max(v, rotate<8>(v));
    v = max(v, rotate<4>(v));
    v = max(v, rotate<2>(v));
    return max(v, rotate<1>(v));
}
template <class T>
__device__ __forceinline__ T least(T v) {
    v = min(v, rotate<8>(v));
    v = min(v, rotate<4>(v));
    v = min(v, rotate<2>(v));
    return min(v, rotate<1>(v));
}

// Candidates' order as unsigned keys: larger value, larger key; -0 and +0 are
// one value; NaN 1, below every number; what is no candidate has 0.
__device__ __forceinline__ uint64_t key64(double v) {
    const uint64_t u = v == 0.0 ? 0ull : uint64_t(__double_as_longlong(v));
    return v != v ? 1ull : (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double value64(uint64_t key) {
    return key == 1ull ? __builtin_nan("") : __longlong_as_double((long long)((key >> 63) ? key & 0x7fffffffffffffffull : ~key));
}

}  // namespace row16
}  // namespace stmoe
