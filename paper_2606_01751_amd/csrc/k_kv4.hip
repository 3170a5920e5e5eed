// Moves between rows or blocks of 16- or 32-bit K/V and the 4-bit pool (include/sx_decode.h).
//
//   kv4_write_kernel   rows by slot, or whole blocks, rounded to 4 bits
//   kv4_read_kernel    the same way back, exactly
//
// A wave takes 16 tokens of one KV head, 512 elements an instruction: lane l has 8 elements, d = 8 (l % (D / 8)), of
// token NI (l / (D / 8)) + i in step i of NI, so an instruction moves whole rows, four neighbouring lanes hold the 32
// elements that share a scale, and a lane's steps are neighbours in V's byte order (with D = 128 its four tokens' codes
// are 16 consecutive bytes of a block; K's become so by a transposition over the four lanes of a group).  The
// scale comes from the largest absolute value's bits: 2^E with 1.m >= 1.75 (m > 0x600000) needs e = E - 1, else
// E - 2 (7 * 2^e = 1.75 * 2^(e + 2)).  The conversion instruction rounds to nearest with ties to even and
// saturates, which is the definition; every 4-bit value is a bfloat16 value, so reading is exact.  Both are bound by HBM:
// 2048 blocks of 8 heads of 128 (bfloat16) take 34 us, 5.0 TB/s read and written, and back, the pool still in the cache,
// 27.6 us, 6.2 TB/s.
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

// Value of lane l ^ X of the same four lanes.
template <int X>
__device__ __forceinline__ uint32_t quad_xor(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, X == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true);   // quad_perm 1032, 2301
}

// Transposes x[4] over four lanes: lane m's x[j] becomes lane j's x[m].
__device__ __forceinline__ void quad_transpose(uint32_t (&x)[4], int m) {
#pragma unroll
  for (int j = 0; j < 4; j += 2) {
    const uint32_t y = quad_xor<1>(m & 1 ? x[j] : x[j + 1]);
    if (m & 1) x[j] = y;
    else x[j + 1] = y;
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t y = quad_xor<2>(m & 2 ? x[j] : x[j + 2]);
    if (m & 2) x[j] = y;
    else x[j + 2] = y;
  }
}

// Eight elements -> codes and their group's scale byte.
template <typename T>
__device__ __forceinline__ uint32_t quantise8(const Raw8<T>& raw, uint32_t* byte) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = raw.at(e);
  // as integers: the absolute values order like their bits, and NaN and infinity come out on top
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, quad_xor<1>(top));
  top = max(top, quad_xor<2>(top));
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
  // (rows become float32 a group at a time: 52 registers, eight waves a SIMD; all of them at once took 92, and 2048
  // blocks of 8 heads of 128 41 us instead of 34)
  constexpr int LPR = D / 8, NI = LPR / 4;   // lanes a row, steps
  const uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (item >= (uint32_t)tiles * a.Hkv) return;
  const int tile = item / (uint32_t)a.Hkv, h = item % (uint32_t)a.Hkv;
  const int lane = threadIdx.x & 63, d = lane % LPR * 8, m = lane & 3;
  Raw8<T> k[NI], v[NI];
  uint8_t* rec[NI];
  int tt[NI];
  bool live[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    int64_t ko = 0, vo = 0;
    rec[i] = nullptr;
    tt[i] = 0;
    if constexpr (!BLOCKS) {                 // (the rows are on their way beside the slots)
      const int64_t row = min(tile * kBlock + lane / LPR * NI + i, a.n - 1);
      k[i].load((const T*)a.k + row * a.k_ld + h * D + d);
      v[i].load((const T*)a.v + row * a.v_ld + h * D + d);
    }
    live[i] = locate<D, BLOCKS>(a, tile, lane / LPR * NI + i, h, &ko, &vo, &rec[i], &tt[i]);
    if constexpr (BLOCKS) {
      if (!live[0]) return;                  // (one block: all or none)
      k[i].load((const T*)a.k + ko + d);
      v[i].load((const T*)a.v + vo + d);
    }
  }
  uint32_t kw[NI] = {}, vw[NI] = {}, kb[NI] = {}, vb[NI] = {};
#pragma unroll
  for (int i = 0; i < NI; ++i)
    if (live[i]) {                           // (a token's lanes stay together)
      kw[i] = quantise8(k[i], &kb[i]);
      vw[i] = quantise8(v[i], &vb[i]);
    }
  const int g = d / kKv4Group;
  if constexpr (D == 128) {
    // lane m of a group takes token 4 (l / 16) + m: the 16 bytes of its K, and its scales
    uint32_t mk[4] = {kb[0], kb[1], kb[2], kb[3]}, mv[4] = {vb[0], vb[1], vb[2], vb[3]};
    quad_transpose(kw, m);
    const uint32_t ks = m & 2 ? (m & 1 ? mk[3] : mk[2]) : (m & 1 ? mk[1] : mk[0]);
    const uint32_t vs = m & 2 ? (m & 1 ? mv[3] : mv[2]) : (m & 1 ? mv[1] : mv[0]);
    uint8_t* r = rec[0];
    int t = tt[0];
    bool on = live[0];
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (m == i) {
        r = rec[i];
        t = tt[i];
        on = live[i];
      }
    if (on) {
      *(uint4*)(r + k_code_off<D>(t, g * kKv4Group)) = make_uint4(kw[0], kw[1], kw[2], kw[3]);
      r[kv4_k_scales(D) + g * 16 + t] = (uint8_t)ks;
      r[kv4_v_scales(D) + g * 16 + t] = (uint8_t)vs;
    }
    if constexpr (BLOCKS) {
      *(uint4*)(rec[0] + v_code_off<D>(tt[0], d)) = make_uint4(vw[0], vw[1], vw[2], vw[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (live[i]) *(uint32_t*)(rec[i] + v_code_off<D>(tt[i], d)) = vw[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (live[i]) {
        *(uint32_t*)(rec[i] + k_code_off<D>(tt[i], d)) = kw[i];
        if (m == 0) {
          rec[i][kv4_k_scales(D) + g * 16 + tt[i]] = (uint8_t)kb[i];
          rec[i][kv4_v_scales(D) + g * 16 + tt[i]] = (uint8_t)vb[i];
        }
        if constexpr (!BLOCKS) {
          *(uint16_t*)(rec[i] + v_code_off<D>(tt[i], d)) = (uint16_t)vw[i];
          *(uint16_t*)(rec[i] + v_code_off<D>(tt[i], d + 4)) = (uint16_t)(vw[i] >> 16);
        }
      }
    if constexpr (BLOCKS) {                  // tokens t, t + 1 of both column groups
      *(uint32_t*)(rec[0] + v_code_off<D>(tt[0], d)) = __builtin_amdgcn_perm(vw[1], vw[0], 0x05040100u);
      *(uint32_t*)(rec[0] + v_code_off<D>(tt[0], d + 4)) = __builtin_amdgcn_perm(vw[1], vw[0], 0x07060302u);
    }
  }
}

// Streaming stores: what leaves is read by a later launch at the earliest.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <typename T>
__device__ __forceinline__ void put8(T* p, uint32_t w, float s) {
  const u32x4_t u = {kv4_pair<0>(w, s), kv4_pair<1>(w, s), kv4_pair<2>(w, s), kv4_pair<3>(w, s)};
  if constexpr (sizeof(T) == 2) {
    __builtin_nontemporal_store(u, (u32x4_t*)p);
  } else {
    const u32x4_t a = {u[0] << 16, u[0] & 0xffff0000u, u[1] << 16, u[1] & 0xffff0000u};
    const u32x4_t b = {u[2] << 16, u[2] & 0xffff0000u, u[3] << 16, u[3] & 0xffff0000u};
    __builtin_nontemporal_store(a, (u32x4_t*)p);
    __builtin_nontemporal_store(b, (u32x4_t*)p + 1);
  }
}

template <typename T, int D, bool BLOCKS>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4MoveK a, int tiles) {
  constexpr int LPR = D / 8, NI = LPR / 4;
  const uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (item >= (uint32_t)tiles * a.Hkv) return;
  const int tile = item / (uint32_t)a.Hkv, h = item % (uint32_t)a.Hkv;
  const int lane = threadIdx.x & 63, d = lane % LPR * 8;
  int64_t ko[NI], vo[NI];
  uint32_t kw[NI], vw[NI], ks[NI], vs[NI];
  bool live[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    uint8_t* rec;
    int tt;
    live[i] = locate<D, BLOCKS>(a, tile, lane / LPR * NI + i, h, &ko[i], &vo[i], &rec, &tt);
    if (live[i]) {
      kw[i] = *(const uint32_t*)(rec + k_code_off<D>(tt, d));
      if constexpr (D == 128)
        vw[i] = *(const uint32_t*)(rec + v_code_off<D>(tt, d));
      else
        vw[i] = *(const uint16_t*)(rec + v_code_off<D>(tt, d)) | (uint32_t)*(const uint16_t*)(rec + v_code_off<D>(tt, d + 4)) << 16;
      ks[i] = rec[kv4_k_scales(D) + d / kKv4Group * 16 + tt];
      vs[i] = rec[kv4_v_scales(D) + d / kKv4Group * 16 + tt];
    }
  }
#pragma unroll
  for (int i = 0; i < NI; ++i)
    if (live[i]) {
      put8((T*)a.k + ko[i] + d, kw[i], kv4_scale(ks[i]));
      put8((T*)a.v + vo[i] + d, vw[i], kv4_scale(vs[i]));
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
