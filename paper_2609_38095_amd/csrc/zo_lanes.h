// What the decode-step kernels share: reductions over neighbouring lanes, element-wise access at
// any dimension, launch status.
#ifndef ZO_LANES_H_
#define ZO_LANES_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "zo_decode.h"
#include "zo_stream.h"

namespace zo {

template <int kCtrl>
__device__ __forceinline__ float lanes_moved(float v) {  // data-parallel move within rows of 16 lanes
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), kCtrl, 0xF, 0xF, true));
}

// The sum over aligned groups of L lanes (a power of two), in every lane of the group. Each step
// adds a pair in both of its lanes, so all lanes hold the same bits.
template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
  if constexpr (L >= 2) v += lanes_moved<0xB1>(v);   // neighbours
  if constexpr (L >= 4) v += lanes_moved<0x4E>(v);   // pairs of a quad
  if constexpr (L >= 8) v += lanes_moved<0x141>(v);  // quads of a half row
  if constexpr (L >= 16) v += lanes_moved<0x140>(v); // halves of a row
  if constexpr (L >= 32) v += __shfl_xor(v, 16, 64);
  if constexpr (L >= 64) v += __shfl_xor(v, 32, 64);
  return v;
}

inline int launched() { return hipGetLastError() == hipSuccess ? ZO_OK : ZO_ERR_HIP; }

}  // namespace zo

#endif  // ZO_LANES_H_
