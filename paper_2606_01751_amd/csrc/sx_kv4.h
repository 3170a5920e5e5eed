// Internal declarations of the decoding calls (include/sx_decode.h), shared by their host side and kernels.
#pragma once

#include <algorithm>

#include "sx_decode.h"
#include "sx_internal.h"

namespace sx {

// ---- the 4-bit record of one KV head of one block (include/sx_decode.h) ----
constexpr int kKv4Group = 32;   // elements that share a scale
__host__ __device__ constexpr int kv4_record(int d) { return 17 * d; }
__host__ __device__ constexpr int kv4_v_codes(int d) { return 8 * d; }
__host__ __device__ constexpr int kv4_k_scales(int d) { return 16 * d; }
__host__ __device__ constexpr int kv4_v_scales(int d) { return 16 * d + d / 2; }

// ---- split of a request's keys over workgroups ----
// A request of `rows` query rows per KV head (tokens x group) and `len` keys is cut into chunks of equal
// length, by its own sizes and the head count alone, so that its result does not depend on the rest of the
// batch: at least kKv4Chunk keys each, at most kKv4Splits of them, and at most kKv4Parts parts (rows x heads x
// chunks), which is a workgroup of 256 rows for each of 256 compute units: more rows fill the chip unsplit.  17 to
// 255 rows count as 256 (128 rows over 65536 keys, 8 heads: 68 us in 32 chunks, 78 in 64); up to 16 as 16.
// kKv4Chunk, at 1024, 512 and 2048: 64 requests of up to 8192 keys (28 / 4 heads, d = 128) 45.5, 50.4 and 47.3 us; 256
// requests of 1024 keys (32 / 8) 58, 75 and 59; 24 of up to 5 tokens and 6000 keys (16 / 4, d = 64) 19.5, 20.0 and 25.2;
// 128 of 5 tokens over 4608 keys (32 / 8, d = 128), which alone gain by the longest, 207, 237 and 181.
constexpr int kKv4Chunk = 1024;
constexpr int kKv4Splits = 64;
constexpr int kKv4Parts = 65536;
constexpr int kKv4Step = 128;    // a chunk's length is a multiple of this
struct Kv4Split {
  int n, keys;   // chunks, and keys of each but the last
};
inline uint32_t kv4_most_chunks(uint32_t rows, uint32_t heads) {
  const uint32_t counted = rows <= 16 ? 16 : rows <= 256 ? 256 : rows;
  const uint32_t n = kKv4Parts / counted / heads;
  return n < 1 ? 1 : n > kKv4Splits ? kKv4Splits : n;
}
// (most16, most256: kv4_most_chunks of up to 16 and 256 rows)
__device__ inline Kv4Split kv4_split(int rows, int len, int heads, int most16, int most256) {
  uint32_t most = rows <= 16 ? most16 : most256;
  if (rows > 256) most = min(max(kKv4Parts / (uint32_t)rows / (uint32_t)heads, 1u), (uint32_t)kKv4Splits);
  const uint32_t n = min(max(((uint32_t)len + kKv4Chunk - 1) / kKv4Chunk, 1u), most);
  const uint32_t units = ((uint32_t)len + kKv4Step - 1) / kKv4Step & 0xffffff;   // (len <= 2^30: 24-bit divisions)
  const uint32_t per = (units + n - 1) / n;
  return {(int)(per > 0 ? (units + per - 1) / per : 1), (int)(per * kKv4Step)};
}
// Division by the heads of a group: n / G = n * magic >> (31 + shift) for 0 <= n < 2^31, with 2^shift the next power of
// two and magic = 2^(31 + shift) / G + 1, which is too large by at most 1, so the product by less than 2^(31 + shift) / G.
struct Kv4Heads {
  uint32_t magic;
  int shift;
  __host__ __device__ int of(int n) const { return (int)((uint64_t)(uint32_t)n * magic >> (31 + shift)); }
};
inline Kv4Heads kv4_heads(uint32_t g) {
  int s = 0;
  while ((1u << s) < g) ++s;
  return {(uint32_t)(((uint64_t)1 << (31 + s)) / g + 1), s};
}
// most chunks, and most partial rows per head (rows x chunks, where there is more than one chunk), of a request of
// at most `rows` rows and `len` keys
inline int kv4_max_chunks(int len) {
  const int64_t n = ((int64_t)len + kKv4Chunk - 1) / kKv4Chunk;
  return (int)(n < 1 ? 1 : n > kKv4Splits ? kKv4Splits : n);
}
inline int64_t kv4_part_rows(int64_t rows, int len, int heads) {
  const int64_t c = kv4_max_chunks(len), cap = std::max(kKv4Parts / heads, 16);
  return c <= 1 ? 0 : std::min(rows * c, cap);   // (more than one chunk: rows x heads x chunks <= kKv4Parts)
}

struct AppendSlotsK {
  const int32_t* ctx;
  const int32_t* add;        // may be null: one token each
  const int32_t* free_blocks;
  const int32_t* free_head;  // may be null
  int32_t* table;
  int32_t* seq;
  int32_t* cu;
  int32_t* pos;
  int32_t* slots;
  int32_t* state;
  int n_req, block, n_free, max_blocks, max_tokens;
};
hipError_t launch_append_slots(const AppendSlotsK& a, hipStream_t s);

struct QkNormRopeK {
  const void* q;
  const void* k;
  void* qo;
  void* ko;
  int64_t q_ld, k_ld, qo_ld, ko_ld;   // elements between token rows
  const void* gq;                     // may be null
  const void* gk;
  float eps;
  int n, Hq, Hkv;
  const int32_t* pos;                 // [n] by token row
  double theta[64];                   // frequencies (plan calls: the plan's array instead)
  // plan's row list
  const ReqDev* reqs;
  const int32_t* rows;
  const int32_t* n_rows;
  const int32_t* tok_pos;
  const double* d_theta;
  int max_rows, n_req;
};
hipError_t launch_qk_norm_rope(const QkNormRopeK& a, int D, bool f32, bool neox, hipStream_t s);

struct Kv4MoveK {
  void* k;              // 16- or 32-bit side
  void* v;
  int64_t k_ld, v_ld;   // rows: elements between token rows
  const int32_t* idx;   // slots, or pool blocks
  const int32_t* cache_blocks;   // blocks only
  uint8_t* pool;
  int64_t n_blocks, n_cache_blocks;
  int n, Hkv;
};
hipError_t launch_kv4_write(const Kv4MoveK& a, int D, bool f32, bool blocks, hipStream_t s);
hipError_t launch_kv4_read(const Kv4MoveK& a, int D, bool f32, bool blocks, hipStream_t s);

struct Kv4AttnK {
  const void* q;
  int64_t q_ld;
  const int32_t* cu;
  const int32_t* lens;
  const int32_t* table;
  const uint8_t* pool;
  void* out;
  float* lse;
  float* part;          // [n_req][Hkv][part_rows][D] unnormalised partial outputs
  float2* part_ml;      // [n_req][Hkv][part_rows] (max, sum), base-2 scores
  int64_t n_blocks, part_rows;
  int max_blocks, n_req, total_q, max_q, max_keys, Hq, Hkv, G;   // max_keys: min(max_seqlen, max_blocks * 16)
  int most16, most256;  // kv4_split
  Kv4Heads group;       // division by G
  float scale;          // softmax scale * log2(e)
};
hipError_t launch_kv4_attn(const Kv4AttnK& a, int D, bool f32, hipStream_t s);

// Checked library: device-side validation (synchronises the stream); verdict as in sx_internal.h.
hipError_t device_check_lengths(const int32_t* ctx, const int32_t* add, int32_t n_req, hipStream_t s, int verdict[4]);
hipError_t device_check_index(const int32_t* idx, int32_t n, int32_t low, int64_t limit, hipStream_t s, int verdict[4]);
hipError_t device_check_kv4(const Kv4AttnK& a, hipStream_t s, int verdict[4]);

}  // namespace sx
