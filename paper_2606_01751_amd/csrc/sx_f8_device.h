// Device helpers of the 8-bit layer body (include/sx_f8.h).
#pragma once

#include "sx_device.h"
#include "sx_f8k.h"

namespace sx {

// Rows that a call takes of request r, and where its n-th one lies.
__device__ __forceinline__ int f8_count(const F8Rows& a, int r) {
  const int most = a.reqs ? min(a.max_rows, a.reqs[r].T) : a.max_rows;
  return a.n_rows ? min(max(a.n_rows[r], 0), most) : most;
}
__device__ __forceinline__ int64_t f8_slot(const F8Rows& a, int r, int n) { return a.reqs ? (int64_t)a.reqs[r].tok_off + n : n; }
// by token: -1 where the listed row is none of the request's
__device__ __forceinline__ int64_t f8_row(const F8Rows& a, int r, int n, bool by_token) {
  if (!a.reqs || !by_token) return f8_slot(a, r, n);
  const int t = a.rows[a.reqs[r].tok_off + n];
  return t >= 0 && t < a.reqs[r].T ? (int64_t)a.reqs[r].tok_off + t : -1;
}

// Maximum over 16 consecutive lanes (a DPP row), in all of them: rotations by 8, 4, 2 and 1.  Unsigned, so that the bits
// of magnitudes compare as the magnitudes do and a NaN above infinity.
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
}

// Scale byte of a group whose largest magnitude has these bits: 448 = 1.75 * 2^8, so amax = m * 2^E needs e = E - 8, or
// E - 7 where m > 1.75.
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return 255;
  const int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(b, 1);
}

// Eight elements in units of their group's scale as e4m3 codes, ties to even (no magnitude is above 448).  The division by
// a power of two is exact where the quotient is not far below e4m3's smallest number.
__device__ __forceinline__ uint2 f8_codes8(const float v[8], uint32_t byte) {
  const float inv = byte == 255 ? 0.0f : __uint_as_float((254u - byte) << 23);
  uint2 o;
  int w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, w[i], true);
  }
  o.x = byte == 255 ? 0u : (uint32_t)w[0];
  o.y = byte == 255 ? 0u : (uint32_t)w[1];
  return o;
}

// Eight elements a lane, lane 0 of the wave at a multiple of 512 elements of its row of k elements at column c (the lane's
// own first element): codes to y8, the scale bytes of the wave's four groups as one word to ys, 0 for groups behind the
// row's end.  Every lane of the wave is here; lanes with c >= k hold zeros.
__device__ __forceinline__ void f8_put8(const float v[8], int c, int k, uint8_t* y8, uint8_t* ys, int lane) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  const uint32_t byte = f8_scale_byte(row16_max(m));
  const uint2 o = f8_codes8(v, byte);
  if (c < k) *(uint2*)(y8 + c) = o;
  const uint32_t b = c < k ? byte : 0;
  const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)b, 0) | (uint32_t)__builtin_amdgcn_readlane((int)b, 16) << 8 |
                        (uint32_t)__builtin_amdgcn_readlane((int)b, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)b, 48) << 24;
  if (lane == 0 && c < k) *(uint32_t*)(ys + c / kF8Group) = word;
}

__device__ __forceinline__ void unpack8(const uint4& v, float o[8]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = bf16_lo(u[i]);
    o[2 * i + 1] = bf16_hi(u[i]);
  }
}
__device__ __forceinline__ uint4 pack8(const float v[8]) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

}  // namespace sx
