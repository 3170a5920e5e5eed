// Device helpers of the decoding kernels (gfx950, wave64).
#pragma once

#include "sx_device.h"
#include "sx_kv4.h"

namespace sx {

// Eight consecutive elements as float32, and back with one rounding (16- and 32-bit types).
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 v = *(const uint4*)p;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  } else {
    const float4 v0 = ((const float4*)p)[0], v1 = ((const float4*)p)[1];
    x[0] = v0.x; x[1] = v0.y; x[2] = v0.z; x[3] = v0.w;
    x[4] = v1.x; x[5] = v1.y; x[6] = v1.z; x[7] = v1.w;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    *(uint4*)p = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                            pack_bf16x2(x[6], x[7]));
  } else {
    ((float4*)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    ((float4*)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// Eight elements as they lie in memory: 4 or 8 dwords.
template <typename T>
struct Raw8 {
  uint32_t w[sizeof(T) * 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint4 v = ((const uint4*)p)[i];
      w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
    }
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 2) return e % 2 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
    else return __uint_as_float(w[e]);
  }
};

// Four dwords of codes have eight elements each; a byte's two elements as bfloat16 times 2^e (s: float32 2^e,
// NaN groups +inf: the instruction reads the exponent, 255 as NaN).  Exact for every byte and scale.
template <int BYTE>
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, BYTE));
}
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace sx
