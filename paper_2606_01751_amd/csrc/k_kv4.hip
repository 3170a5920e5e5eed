// Moves between rows or blocks of 16- or 32-bit K/V and the 4-bit pool (include/sx_decode.h).
//
//   kv4_write_kernel   rows by slot, or whole blocks, rounded to 4 bits
//   kv4_read_kernel    the same way back, exactly
//
// A wave takes 16 tokens of one KV head: lane l has token l / 4 and, in step `it`, the 8 elements from
// d = 32 it + 8 (l % 4), so four neighbouring lanes hold the 32 elements that share a scale.  The scale
// comes from the largest absolute value's bits: 2^E with 1.m >= 1.75 (m > 0x600000) needs e = E - 1, else
// E - 2 (7 * 2^e = 1.75 * 2^(e + 2)).  The conversion instruction rounds to nearest with ties to even and
// saturates, which is the definition; every 4-bit value is a bfloat16 value, so reading is exact.
#include "sx_kv4_device.h"

namespace sx {
namespace {

// Byte offsets inside a record of the dword (D = 128) or the two bytes (D = 64: 4 elements of a column
// group) that hold elements d .. of token t.
template <int D>
__device__ __forceinline__ int k_code_off(int t, int d) {
  return d / (D / 4) * (2 * D) + t * (D / 8) + d % (D / 4) / 2;
}
template <int D>
__device__ __forceinline__ int v_code_off(int t, int d) {
  return kv4_v_codes(D) + ((t / 4 * 16 + d / (D / 16)) * 4 + t % 4) * (D / 32);
}

// Eight elements -> codes and their group's scale byte.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t* byte) {
  // as integers: the absolute values order like their bits, and NaN and infinity come out on top
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
  if (top >= 0x7f800000u) {
    *byte = 255;
    return 0;
  }
  const int b = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u);
  *byte = (uint32_t)min(max(b, 1), 252);
  const float s = kv4_scale(*byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return w;
}

// Where token t of tile `tile`, head h lives: element offset of its row on the 16- or 32-bit side (K and
// V), its record, its token in the block; false: not moved.
template <int D, bool BLOCKS>
__device__ __forceinline__ bool locate(const Kv4MoveK& a, int tile, int t, int h, int64_t* ko, int64_t* vo,
                                       uint8_t** rec, int* tt) {
  if constexpr (BLOCKS) {
    const int cb = a.cache_blocks[tile], pb = a.idx[tile];
    if (cb < 0 || cb >= a.n_cache_blocks || pb < 0 || pb >= a.n_blocks) return false;
    *ko = *vo = (((int64_t)cb * a.Hkv + h) * kBlock + t) * D;
    *rec = a.pool + ((int64_t)pb * a.Hkv + h) * kv4_record(D);
    *tt = t;
  } else {
    const int i = tile * kBlock + t;
    if (i >= a.n) return false;
    const int slot = a.idx[i];
    if (slot < 0 || slot / kBlock >= a.n_blocks) return false;
    *ko = (int64_t)i * a.k_ld + h * D;
    *vo = (int64_t)i * a.v_ld + h * D;
    *rec = a.pool + ((int64_t)(slot / kBlock) * a.Hkv + h) * kv4_record(D);
    *tt = slot % kBlock;
  }
  return true;
}

template <typename T, int D, bool BLOCKS>
__global__ __launch_bounds__(256) void kv4_write_kernel(Kv4MoveK a, int tiles) {
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= (int64_t)tiles * a.Hkv) return;
  const int tile = (int)(item / a.Hkv), h = (int)(item % a.Hkv);
  const int lane = threadIdx.x & 63, t = lane >> 2, m = lane & 3;
  int64_t ko = 0, vo = 0;
  uint8_t* rec = nullptr;
  int tt = 0;
  const bool live = locate<D, BLOCKS>(a, tile, t, h, &ko, &vo, &rec, &tt);
  if (!live) return;   // (a token's four lanes leave together)
#pragma unroll
  for (int it = 0; it < D / 32; ++it) {
    const int d = it * 32 + m * 8;
    float x[8];
    uint32_t byte;
    load8((const T*)a.k + ko + d, x);
    *(uint32_t*)(rec + k_code_off<D>(tt, d)) = quantise8(x, &byte);
    if (m == 0) rec[kv4_k_scales(D) + it * 16 + tt] = (uint8_t)byte;
    load8((const T*)a.v + vo + d, x);
    const uint32_t w = quantise8(x, &byte);
    if constexpr (D == 128) {
      *(uint32_t*)(rec + v_code_off<D>(tt, d)) = w;
    } else {
      *(uint16_t*)(rec + v_code_off<D>(tt, d)) = (uint16_t)w;
      *(uint16_t*)(rec + v_code_off<D>(tt, d + 4)) = (uint16_t)(w >> 16);
    }
    if (m == 0) rec[kv4_v_scales(D) + it * 16 + tt] = (uint8_t)byte;
  }
}

template <typename T>
__device__ __forceinline__ void put8(T* p, uint32_t w, float s) {
  const uint32_t u[4] = {kv4_pair<0>(w, s), kv4_pair<1>(w, s), kv4_pair<2>(w, s), kv4_pair<3>(w, s)};
  if constexpr (sizeof(T) == 2) {
    *(uint4*)p = make_uint4(u[0], u[1], u[2], u[3]);
  } else {
    const float x[8] = {bf16_lo(u[0]), bf16_hi(u[0]), bf16_lo(u[1]), bf16_hi(u[1]),
                        bf16_lo(u[2]), bf16_hi(u[2]), bf16_lo(u[3]), bf16_hi(u[3])};
    store8(p, x);
  }
}

template <typename T, int D, bool BLOCKS>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4MoveK a, int tiles) {
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= (int64_t)tiles * a.Hkv) return;
  const int tile = (int)(item / a.Hkv), h = (int)(item % a.Hkv);
  const int lane = threadIdx.x & 63, t = lane >> 2, m = lane & 3;
  int64_t ko = 0, vo = 0;
  uint8_t* rec = nullptr;
  int tt = 0;
  if (!locate<D, BLOCKS>(a, tile, t, h, &ko, &vo, &rec, &tt)) return;
#pragma unroll
  for (int it = 0; it < D / 32; ++it) {
    const int d = it * 32 + m * 8;
    put8((T*)a.k + ko + d, *(const uint32_t*)(rec + k_code_off<D>(tt, d)),
         kv4_scale(rec[kv4_k_scales(D) + it * 16 + tt]));
    uint32_t w;
    if constexpr (D == 128)
      w = *(const uint32_t*)(rec + v_code_off<D>(tt, d));
    else
      w = *(const uint16_t*)(rec + v_code_off<D>(tt, d)) | (uint32_t)*(const uint16_t*)(rec + v_code_off<D>(tt, d + 4)) << 16;
    put8((T*)a.v + vo + d, w, kv4_scale(rec[kv4_v_scales(D) + it * 16 + tt]));
  }
}

}  // namespace

#define SX_MOVE(KERNEL, T_, D_)                                                                                \
  do {                                                                                                         \
    if (blocks) hipLaunchKernelGGL((KERNEL<T_, D_, true>), grid, dim3(256), 0, s, a, tiles);                   \
    else hipLaunchKernelGGL((KERNEL<T_, D_, false>), grid, dim3(256), 0, s, a, tiles);                         \
  } while (0)
#define SX_MOVE_ALL(KERNEL)                                                                                    \
  const int tiles = blocks ? a.n : (a.n + kBlock - 1) / kBlock;                                                \
  const dim3 grid((unsigned)(((int64_t)tiles * a.Hkv + 3) / 4));                                               \
  if (f32) { if (D == 128) SX_MOVE(KERNEL, float, 128); else SX_MOVE(KERNEL, float, 64); }                     \
  else { if (D == 128) SX_MOVE(KERNEL, uint16_t, 128); else SX_MOVE(KERNEL, uint16_t, 64); }                   \
  return hipGetLastError();

hipError_t launch_kv4_write(const Kv4MoveK& a, int D, bool f32, bool blocks, hipStream_t s) { SX_MOVE_ALL(kv4_write_kernel) }
hipError_t launch_kv4_read(const Kv4MoveK& a, int D, bool f32, bool blocks, hipStream_t s) { SX_MOVE_ALL(kv4_read_kernel) }

}  // namespace sx
