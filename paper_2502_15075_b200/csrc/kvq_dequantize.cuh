// What the kernels that turn codes back into 16 bits share.
#pragma once

#include "kvq_internal.h"

namespace kvq {

// Bytes i and j of `bytes` as exact floats.
__device__ __forceinline__ f32x2 code_pair(uint32_t bytes, int i, int j) {
  const float a = __uint_as_float(__byte_perm(bytes, 0x4B000000u, 0x7540u + (uint32_t)i));
  const float b = __uint_as_float(__byte_perm(bytes, 0x4B000000u, 0x7540u + (uint32_t)j));
  return add2(pack2(a, b), pack2(-8388608.0f, -8388608.0f));
}
template <int DTYPE>
__device__ __forceinline__ uint32_t pack16(f32x2 v) {
  const float2 f = unpack2(v);
  if constexpr (DTYPE == KVQ_FP16) {
    const __half2 h = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

}  // namespace kvq
