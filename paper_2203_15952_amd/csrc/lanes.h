// Sums and maxima over aligned groups of 4, 8 or 16 lanes that leave every lane with the result.  The values move inside the vector
// instructions themselves (data-parallel primitives) and not through LDS: neighbours, neighbouring pairs, then the mirror
// image in 8 and in 16 lanes, which is the other half's value, as the lanes of a half hold the same by then.  All lanes take part.
#pragma once
#include "aqt_internal.h"

namespace aqt {
namespace {

template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, true));
}
// Lane K's of the four.
template <int K>
__device__ __forceinline__ float of_four(float v) {
  return __uint_as_float(moved<K * 0x55>(__float_as_uint(v)));
}

// The other lane's of an aligned pair.
__device__ __forceinline__ float of_neighbour(float v) { return __uint_as_float(moved<0xB1>(__float_as_uint(v))); }

template <int L>
__device__ __forceinline__ float group_sum(float v) {
  v += __uint_as_float(moved<0xB1>(__float_as_uint(v)));                   // lanes 1 0 3 2
  v += __uint_as_float(moved<0x4E>(__float_as_uint(v)));                   // lanes 2 3 0 1
  if constexpr (L > 4) v += __uint_as_float(moved<0x141>(__float_as_uint(v)));   // mirrored in 8
  if constexpr (L > 8) v += __uint_as_float(moved<0x140>(__float_as_uint(v)));   // mirrored in 16
  return v;
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = max(v, moved<0xB1>(v));
  v = max(v, moved<0x4E>(v));
  if constexpr (L > 4) v = max(v, moved<0x141>(v));
  if constexpr (L > 8) v = max(v, moved<0x140>(v));
  return v;
}

}  // namespace
}  // namespace aqt
