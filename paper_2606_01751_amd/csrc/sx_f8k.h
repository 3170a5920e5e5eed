// Internal declarations of the 8-bit layer body (include/sx_f8.h), shared by its host side and kernels.
#pragma once

#include "sx_f8.h"
#include "sx_internal.h"

namespace sx {

constexpr int kF8Group = 128;       // elements that share a scale
constexpr int kF8MaxK = 65536;
constexpr int kF8MaxParts = 4;
constexpr int kMoeMaxExperts = 1024;
constexpr int kMoeMaxTop = 16;

__host__ __device__ constexpr int f8_ld(int k) { return (k / kF8Group + 3) / 4 * 4; }

// The rows of a call: a plan's listed rows, or (reqs NULL) rows 0 .. count - 1 of every array.
struct F8Rows {
  const ReqDev* reqs;
  const int32_t* rows;     // plan only, NULL: no operand is addressed by token
  const int32_t* n_rows;   // [n_req]; without a plan [1], or NULL: max_rows rows
  int max_rows, n_req;
};

struct F8NormK {
  F8Rows r;
  const uint16_t* x;
  const uint16_t* delta;
  const uint16_t* gamma;
  uint16_t* x_out;
  uint16_t* y16;
  uint8_t* y8;
  uint8_t* ys;
  float eps;
  int h, ld, x_tok, y_tok;
};

struct F8SiluK {
  F8Rows r;
  const uint16_t* gu;
  uint8_t* y8;
  uint8_t* ys;
  int f, ld;
};

struct F8GemmK {
  F8Rows r;                 // listed rows, or:
  const int32_t* offsets;   // [n_experts + 1] (grouped by expert where not NULL)
  const int32_t* order;     // [n_places] or NULL
  const uint8_t* x;
  const uint8_t* xs;
  const uint8_t* w;
  const uint8_t* ws;
  const uint16_t* res;
  uint16_t* y[kF8MaxParts];   // part p: columns pn[p] .. pn[p + 1] - 1, row stride pn[p + 1] - pn[p]
  int pn[kF8MaxParts + 1];
  int n_parts, K, N, ld, x_tok, y_tok;
  int n_experts, n_places, x_rows, gather, scatter;
  int m_tiles;                // rows: tiles of every request; experts: tiles of the whole launch
  int run;                    // tiles of features that a workgroup takes one after the other
};

struct MoeRouteK {
  F8Rows r;
  const void* logits;
  int32_t* ids;
  float* weights;
  int32_t* offsets;
  int32_t* order;
  int32_t* counts;   // [blocks][n_experts]
  int n_experts, top_k, renormalise;
  int blocks, per_req, rows_per_block, reqs_per_block;   // see moe_blocks
};

struct MoeCombineK {
  F8Rows r;
  const uint16_t* y;
  const float* weights;
  const uint16_t* res;
  uint16_t* out;
  int top_k, h, out_tok;
};

// Workgroups of the routing: per_req of them share a request's rows, rows_per_block (a multiple of 64) each; or, of
// more than kMoeBlocks requests, one takes reqs_per_block whole ones.  Every one reads all the others' counts, so there
// are about kMoeBlocks at most.
constexpr int kMoeBlocks = 256;
constexpr int kMoeRows = 64;   // rows of a workgroup, where kMoeBlocks of them are enough
inline void moe_blocks(int n_req, int max_rows, MoeRouteK* a) {
  a->reqs_per_block = n_req > kMoeBlocks ? (n_req + kMoeBlocks - 1) / kMoeBlocks : 1;
  int64_t per = n_req > kMoeBlocks ? 1 : kMoeBlocks / n_req;
  const int64_t want = ((int64_t)max_rows + kMoeRows - 1) / kMoeRows;
  if (per > want) per = want;
  if (per < 1) per = 1;
  a->rows_per_block = (int)((((int64_t)max_rows + per - 1) / per + 63) / 64 * 64);
  if (a->rows_per_block < 64) a->rows_per_block = 64;
  a->per_req = (int)(((int64_t)max_rows + a->rows_per_block - 1) / a->rows_per_block);
  if (a->per_req < 1) a->per_req = 1;
  a->blocks = a->per_req > 1 ? n_req * a->per_req : (n_req + a->reqs_per_block - 1) / a->reqs_per_block;
}

// (checked library) offsets of n_experts groups within n_places; the order's entries of the places in use, from 0 up to
// n_places, and what they stand for (entry / gather) below x_rows
hipError_t device_check_index(const int32_t* idx, int32_t n, int32_t low, int64_t limit, hipStream_t s, int verdict[4]);
hipError_t device_check_offsets(const int32_t* offsets, int32_t n_experts, int32_t n_places, hipStream_t s, int verdict[4]);
hipError_t device_check_order(const int32_t* offsets, int32_t n_experts, const int32_t* order, int32_t n_places, int32_t gather,
                              int32_t x_rows, hipStream_t s, int verdict[4]);

hipError_t launch_f8_pack_weight(const uint16_t* w, int64_t n, int k, uint8_t* codes, uint8_t* scales, hipStream_t s);
hipError_t launch_add_rmsnorm_f8(const F8NormK& a, hipStream_t s);
hipError_t launch_silu_mul_f8(const F8SiluK& a, hipStream_t s);
hipError_t launch_gemm_f8(F8GemmK& a, int n_cu, hipStream_t s);   // hipErrorInvalidConfiguration: too many tiles
hipError_t launch_moe_route(const MoeRouteK& a, bool f32, hipStream_t s);
hipError_t launch_moe_combine(const MoeCombineK& a, hipStream_t s);

}  // namespace sx
