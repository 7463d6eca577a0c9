// Sums and maxima over aligned groups of L lanes (L = 4, 8, 16, 32 or 64), and 16-byte pieces of rows.  Internal to the library.
//
// Steps of one, two, four and eight lanes are DPP forms of the operation itself (swaps inside a quad, then mirrored halves and rows: by then the
// lanes that mirroring exchanges hold the same value), steps of 16 and 32 the permlane swaps: no trip through LDS, where a step of a shuffle costs a
// ds_bpermute.  Every lane of a group gets the same bits, in a fixed order.  All 64 lanes have to take part.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rl {

// An output of this size or more is stored past the caches: with what is read beside it, it would not stay in the 256 MB in front of the memory
// until the next kernel reads it, and would be written back while that one runs.  Forward and backward, us, past them / through them: rows of 8192 x 4096
// to two experts (128 MB) 70 / 81, back from eight of 8192 x 2048 (256 MB) 162 / 173, norms of 16384 x 5120 (160 MB) 255 / 266; below, the backward finds
// what the forward wrote: 8192 x 4096 (64 MB) 102 / 97, 16384 x 2048 106 / 99.
constexpr int64_t kStreamBytes = 128LL << 20;

#if defined(__HIPCC__)
template <int CTRL>
__device__ __forceinline__ uint32_t dpp32(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
// one step: the group's other half as this lane sees it (1 to 8 lanes)
template <int STEP>
__device__ __forceinline__ uint32_t across32(uint32_t x) {
  if constexpr (STEP == 1) return dpp32<0xB1>(x);        // quad_perm [1, 0, 3, 2]
  else if constexpr (STEP == 2) return dpp32<0x4E>(x);   // quad_perm [2, 3, 0, 1]
  else if constexpr (STEP == 4) return dpp32<0x141>(x);  // row_half_mirror
  else return dpp32<0x140>(x);                           // row_mirror
}
template <int STEP, typename V>
__device__ __forceinline__ V across(V v) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, across32<STEP>(__builtin_bit_cast(uint32_t, v)));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = across32<STEP>((uint32_t)u), hi = across32<STEP>((uint32_t)(u >> 32));
    return __builtin_bit_cast(V, lo | hi << 32);
  }
}
// steps of 16 and 32 lanes: both halves' values on every lane, in the same order
template <int STEP, typename V, typename Op>
__device__ __forceinline__ V join_halves(V v, Op op) {
  auto swap = [](uint32_t x) {
    if constexpr (STEP == 16) return __builtin_amdgcn_permlane16_swap(x, x, false, false);
    else return __builtin_amdgcn_permlane32_swap(x, x, false, false);
  };
  if constexpr (sizeof(V) == 4) {
    const auto s = swap(__builtin_bit_cast(uint32_t, v));
    return op(__builtin_bit_cast(V, (uint32_t)s[0]), __builtin_bit_cast(V, (uint32_t)s[1]));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const auto lo = swap((uint32_t)u), hi = swap((uint32_t)(u >> 32));
    return op(__builtin_bit_cast(V, (uint64_t)lo[0] | (uint64_t)hi[0] << 32), __builtin_bit_cast(V, (uint64_t)lo[1] | (uint64_t)hi[1] << 32));
  }
}
struct OpAdd { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct OpMax { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; } };
template <int L, typename V, typename Op>
__device__ __forceinline__ V lanes_reduce(V v, Op op) {
  if constexpr (L > 1) v = op(v, across<1>(v));
  if constexpr (L > 2) v = op(v, across<2>(v));
  if constexpr (L > 4) v = op(v, across<4>(v));
  if constexpr (L > 8) v = op(v, across<8>(v));
  if constexpr (L > 16) v = join_halves<16>(v, op);
  if constexpr (L > 32) v = join_halves<32>(v, op);
  return v;
}
template <int L, typename V> __device__ __forceinline__ V lanes_sum(V v) { return lanes_reduce<L>(v, OpAdd()); }
template <int L, typename V> __device__ __forceinline__ V lanes_max(V v) { return lanes_reduce<L>(v, OpMax()); }

// 16 bytes of a row
template <typename T>
struct Piece {
  static constexpr int N = 16 / (int)sizeof(T);
  using V4 = __attribute__((__vector_size__(4 * sizeof(int)))) int;
  V4 v;
  __device__ __forceinline__ static Piece zero() { return Piece{V4{0, 0, 0, 0}}; }
  __device__ __forceinline__ static Piece load(const T* p) { return Piece{*reinterpret_cast<const V4*>(p)}; }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<V4*>(p) = v; }
  // past the caches, where `stream` (kStreamBytes).  The empty statements keep the compiler from making one ordinary store of the two.
  __device__ __forceinline__ void store(T* p, bool stream) const {
    if (stream) {
      asm volatile("");
      __builtin_nontemporal_store(v, reinterpret_cast<V4*>(p));
      asm volatile("");
    } else {
      store(p);
    }
  }
  __device__ __forceinline__ void get(float (&f)[N]) const {
    T t[N];
    *reinterpret_cast<V4*>(t) = v;
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = (float)t[k];
  }
  __device__ __forceinline__ static Piece of(const float (&f)[N]) {
    T t[N];
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = (T)f[k];
    return Piece{*reinterpret_cast<const V4*>(t)};
  }
};
#endif

}  // namespace rl
