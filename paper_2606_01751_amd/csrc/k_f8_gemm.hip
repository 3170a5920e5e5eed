// Products of the 8-bit layer body (include/sx_f8.h): y[row] = x[row] w^T of listed rows, and of rows grouped by expert.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 e4m3 numbers, times a power of two for each of its
// rows and columns: one block of the format a step, so the scales cost no instruction of their own and the sums stay in
// the accumulator.  Computed transposed, y^T = w x^T: the A operand is a slice of w (16 output features), the B operand
// a slice of x^T (16 rows), so a lane owns one row of the result and four consecutive features.  Operands hold 32
// elements a lane; here they are the 16 from 16 g on and the 16 from 64 + 16 g on of the block's 128 (g = lane / 16), on
// both sides alike, so that 16-byte loads of four lanes cover 64 bytes.
//
// The instruction aligns the products of eight consecutive elements to the largest one's exponent and cuts them off 13 bits
// below it (measured: beside a product of 1 in its eight, 2^-13 is added and 2^-14 is not); sums of eights are float32.
// Over normal data that is 2^-14.5 of a result, next to 2^-9 of its rounding to bfloat16.
//
// Every kernel adds the blocks of k one by one in ascending order into one accumulator, so a row's result does not depend
// on the kernel or tile that the launch's size chose.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "sx_f8_device.h"

namespace sx {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8_t operand(i32x4_t a, i32x4_t b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// One block of k: scale bytes S of the words sw and sx.
template <int S>
__device__ __forceinline__ f32x4_t mfma_block(const i32x8_t& w, const i32x8_t& x, const f32x4_t& c, int sw, int sx) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, S, sw, S, sx);
}

// The rows of a workgroup: rows m0 .. m0 + BM - 1 of nr of request (or expert) r.
struct RowTile {
  int r, m0, nr;
  int64_t a;   // experts: the first place of expert r
};

// Row tile number `idx` of the launch; false where there is none.
template <int BM, bool EXPERTS>
__device__ __forceinline__ bool row_tile(const F8GemmK& a, int idx, int lane, RowTile* t) {
  if constexpr (EXPERTS) {
    auto first = [&](int e) { return min(max(a.offsets[e], 0), a.n_places); };
    auto len = [&](int e) { return max(first(e + 1) - first(e), 0); };
    int r, q;
    locate_request(idx, a.n_experts, [&](int e) { return (len(e) + BM - 1) / BM; }, &r, &q, lane);
    if (r < 0) return false;
    r = __builtin_amdgcn_readfirstlane(r);
    *t = {r, __builtin_amdgcn_readfirstlane(q) * BM, len(r), first(r)};
  } else {
    const int r = idx / a.m_tiles;
    *t = {r, (idx - r * a.m_tiles) * BM, f8_count(a.r, r), 0};
  }
  return t->m0 < t->nr;
}

// Where row m of the tile's list lies in x (always a row of x: what is out of range is not stored) and in y (-1: nowhere).
template <bool EXPERTS>
__device__ __forceinline__ int64_t x_row(const F8GemmK& a, const RowTile& t, int m) {
  if constexpr (EXPERTS) {
    int64_t p = t.a + m;
    if (a.gather) p = min(max(a.order[p], 0), a.n_places - 1) / a.gather;
    return min(p, (int64_t)a.x_rows - 1);
  } else {
    const int64_t p = f8_row(a.r, t.r, m, a.x_tok);
    return p < 0 ? f8_slot(a.r, t.r, m) : p;
  }
}
template <bool EXPERTS>
__device__ __forceinline__ int64_t y_row(const F8GemmK& a, const RowTile& t, int m) {
  if constexpr (EXPERTS) {
    const int64_t p = t.a + m;
    if (!a.gather && !a.scatter) return p < a.x_rows ? p : -1;
    const int o = a.order[p];
    if (o < 0 || o >= a.n_places || (a.gather ? o / a.gather : p) >= a.x_rows) return -1;
    return a.scatter ? o : p;
  } else {
    if (f8_row(a.r, t.r, m, a.x_tok) < 0) return -1;
    return f8_row(a.r, t.r, m, a.y_tok);
  }
}

// Four consecutive features n of a row of y.
__device__ __forceinline__ void put4(const F8GemmK& a, int64_t row, int part, int n, f32x4_t v) {
  if (row < 0) return;
  const int64_t at = row * (a.pn[part + 1] - a.pn[part]) + (n - a.pn[part]);
  if (a.res) {
    const uint2 rv = *(const uint2*)(a.res + at);
    v[0] += bf16_lo(rv.x);
    v[1] += bf16_hi(rv.x);
    v[2] += bf16_lo(rv.y);
    v[3] += bf16_hi(rv.y);
  }
  uint2 o;
  o.x = pack_bf16x2(v[0], v[1]);
  o.y = pack_bf16x2(v[2], v[3]);
  *(uint2*)(a.y[part] + at) = o;
}

__device__ __forceinline__ int part_of(const F8GemmK& a, int n) {
  int p = 0;
  while (p + 1 < a.n_parts && n >= a.pn[p + 1]) ++p;
  return p;
}

// A wave's results, FI x RJ fragments, through its own part of LDS (epilogue_lds bytes), so that rows go out in whole runs
// of 32 FI bytes: a store of the fragments themselves (4 features a lane) touches 16 rows at 32 bytes each.  Rows m0 .. of
// the tile's list, features nw .. of one part.  A residual is fetched into the same places first.
template <int FI, int RJ>
constexpr int epilogue_lds() { return 16 * RJ * (32 * FI + 16) + 16 * RJ * 8; }   // (16 bytes a row against bank conflicts)
template <int FI, int RJ, bool EXPERTS>
__device__ __forceinline__ void put_tile(const F8GemmK& a, const RowTile& t, int m0, int nw, const f32x4_t (&acc)[FI][RJ], char* lds, int lane) {
  constexpr int LD = 32 * FI + 16, ROWS = 16 * RJ, CH = 2 * FI, RPI = 64 / CH;   // 16-byte chunks of a row, rows an instruction
  static_assert(64 % CH == 0, "whole rows an instruction");
  const int lr = lane % 16, g = lane / 16;
  const int part = part_of(a, nw);
  const int64_t ld = a.pn[part + 1] - a.pn[part];
  const int col = nw - a.pn[part] + lane % CH * 8;
  int64_t* const yrow = (int64_t*)(lds + ROWS * LD);
#pragma unroll
  for (int i = 0; i < ROWS; i += 64)
    if (i + lane < ROWS) yrow[i + lane] = m0 + i + lane < t.nr ? y_row<EXPERTS>(a, t, m0 + i + lane) : -1;
  if (a.res) {
#pragma unroll 4
    for (int i = 0; i < ROWS; i += RPI) {
      const int row = i + lane / CH;
      if ((ROWS % RPI == 0 || row < ROWS) && yrow[row] >= 0) *(uint4*)(lds + row * LD + lane % CH * 16) = *(const uint4*)(a.res + yrow[row] * ld + col);
    }
  }
#pragma unroll
  for (int j = 0; j < RJ; ++j)
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      uint2* const at = (uint2*)(lds + (16 * j + lr) * LD + 32 * i + 8 * g);
      f32x4_t v = acc[i][j];
      if (a.res) {
        const uint2 rv = *at;
        v[0] += bf16_lo(rv.x);
        v[1] += bf16_hi(rv.x);
        v[2] += bf16_lo(rv.y);
        v[3] += bf16_hi(rv.y);
      }
      *at = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
#pragma unroll 4
  for (int i = 0; i < ROWS; i += RPI) {
    const int row = i + lane / CH;
    if (ROWS % RPI != 0 && row >= ROWS) continue;
    const int64_t y = yrow[row];
    const uint4 v = *(const uint4*)(lds + row * LD + lane % CH * 16);
    if (y >= 0) *(uint4*)(a.y[part] + y * ld + col) = v;
  }
}

// ---------------------------------------------------------------------------------------------
// Few rows: a wave of its own takes 16 FI features and 16 RJ rows and reads both operands from memory into registers, D
// blocks of k ahead, so no wave waits for another and nothing passes through LDS.
// ---------------------------------------------------------------------------------------------
template <int FI, int RJ, int D, bool EXPERTS>
__global__ __launch_bounds__(64, 1) void f8_stream_kernel(F8GemmK a) {
  constexpr int BM = 16 * RJ, BN = 16 * FI;
  static_assert(D % 4 == 0, "scale bytes come four blocks at once");
  const int lane = threadIdx.x, lr = lane % 16, g = lane / 16;
  const int n_nt = a.N / BN;
  const int idx = blockIdx.x / n_nt, n0 = (int)(blockIdx.x - (unsigned)idx * n_nt) * BN;
  RowTile t;
  if (!row_tile<BM, EXPERTS>(a, idx, lane, &t)) return;
  const int64_t e = EXPERTS ? t.r : 0;
  const uint8_t* w = a.w + (e * a.N + n0 + lr) * a.K + 16 * g;
  const uint8_t* ws = a.ws + (e * (a.N / kF8Group) + n0 / kF8Group) * a.ld;
  const uint8_t* x[RJ];
  const uint8_t* xs[RJ];
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    const int64_t row = x_row<EXPERTS>(a, t, min(t.m0 + 16 * j + lr, t.nr - 1));
    x[j] = a.x + row * a.K + 16 * g;
    xs[j] = a.xs + row * a.ld;
  }
  f32x4_t acc[FI][RJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4_t{};
  const int nb = a.K / kF8Group;
  i32x8_t wo[D][FI], xo[D][RJ];
  int sw[D / 4], sx[D / 4][RJ];
  auto load = [&](int s, int b) {   // block b into place s
    const int at = b * kF8Group;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const uint8_t* p = w + (int64_t)i * 16 * a.K + at;
      wo[s][i] = operand(*(const i32x4_t*)p, *(const i32x4_t*)(p + 64));
    }
#pragma unroll
    for (int j = 0; j < RJ; ++j) xo[s][j] = operand(*(const i32x4_t*)(x[j] + at), *(const i32x4_t*)(x[j] + at + 64));
  };
  auto load_scales = [&](int s, int b) {   // of blocks b .. b + 3
    sw[s] = *(const int*)(ws + b);
#pragma unroll
    for (int j = 0; j < RJ; ++j) sx[s][j] = *(const int*)(xs[j] + b);
  };
#pragma unroll
  for (int s = 0; s < D; ++s) {
    if (s < nb) {
      if (s % 4 == 0) load_scales(s / 4, s);
      load(s, s);
    }
  }
  auto step = [&](auto c, int b) {
    constexpr int S = decltype(c)::value;
    if (b + S < nb) {
#pragma unroll
      for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < RJ; ++j) acc[i][j] = mfma_block<S % 4>(wo[S][i], xo[S][j], acc[i][j], sw[S / 4], sx[S / 4][j]);
    }
    if (b + D + S < nb) load(S, b + D + S);
    if constexpr (S % 4 == 3)
      if (b + D + S - 3 < nb) load_scales(S / 4, b + D + S - 3);
  };
  for (int b = 0; b < nb; b += D)
    [&]<int... S>(std::integer_sequence<int, S...>) { (step(std::integral_constant<int, S>{}, b), ...); }(std::make_integer_sequence<int, D>{});
  const int part = part_of(a, n0);
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    const int m = t.m0 + 16 * j + lr;
    if (m < t.nr) {
      const int64_t row = y_row<EXPERTS>(a, t, m);
#pragma unroll
      for (int i = 0; i < FI; ++i) put4(a, row, part, n0 + 16 * i + 4 * g, acc[i][j]);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Tiles of BN features x BM rows, WN x WM waves.  Blocks of k move through NST stages of LDS, global -> LDS directly; a tile
// row (one block, 128 bytes) holds 8 chunks of 16 bytes, XOR-swizzled per row so that the 16 rows of a read hit distinct
// banks.  While the matrix instructions of a block run, the operands of the next one are read (those of x into the
// registers that are free after their last use, those of w into a second set), and a stage is refilled as soon as all
// waves have read it.  The scale bytes go ahead of the first stage the same way, for all of k.
// ---------------------------------------------------------------------------------------------
constexpr int kLdsBytes = 163840;   // LDS of a compute unit
constexpr unsigned kXcds = 8;   // XCDs of the chip, which deals workgroups round-robin
constexpr int kRowGroup = 8;    // row tiles per group of the tile order

// s_waitcnt with vmcnt <= n (n < 64), expcnt and lgkmcnt left unconstrained (gfx9 encoding)
#define SX_WAIT_VM(n) __builtin_amdgcn_s_waitcnt(((n) & 0xF) | ((((n) >> 4) & 3) << 14) | (0x7 << 4) | (0xF << 8))

__device__ __forceinline__ int chunk_swz(int c, int row) { return c ^ ((row >> 1) & 7); }   // (two rows per 256-byte line)

// Bytes of LDS: the stages, then the scale bytes of x as [word][BM] words, and those of the tile's blocks of w, each of them
// padded to whole transfers of 64 words.
__host__ __device__ constexpr int tile_x_scales(int bm, int ld) { return (bm * ld + 255) / 256 * 256; }
__host__ __device__ constexpr int tile_w_scales(int ld) { return (ld + 255) / 256 * 256; }
template <int BN, int BM, int NST>
constexpr int tile_lds(int ld) {
  return NST * (BN + BM) * kF8Group + tile_x_scales(BM, ld) + (BN + kF8Group - 1) / kF8Group * tile_w_scales(ld);
}

template <int BN, int BM, int WN, int WM, int NST, bool EXPERTS>
__global__ __launch_bounds__(WN * WM * 64, 1) void f8_tile_kernel(F8GemmK a) {
  constexpr int NW = WN * WM;
  constexpr int FI = BN / WN / 16, RJ = BM / WM / 16;       // fragments of a wave
  constexpr int STAGE = (BN + BM) * kF8Group;
  constexpr int PW = BN / 8 / NW, PX = BM / 8 / NW, ND = PW + PX;   // transfers of 1 KB (8 rows) a wave and stage
  constexpr int NM = FI * RJ;
  // transfers that refill a stage are issued from the entry of the next block on: D0 of them beside a block's second half,
  // the others beside the next one's first
  constexpr int D0 = (ND * 3 + 3) / 4;
  static_assert(PW * NW * 8 == BN && PX * NW * 8 == BM, "transfers spread evenly over the waves");
  static_assert(FI % 2 == 0, "two halves");
  static_assert(BN / WN <= kF8Group, "a wave's features lie in one block of the weight");
  static_assert((NST - 1) * ND < 64, "transfers in flight");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wu = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Tile order: groups of kRowGroup row tiles, the feature tile slowest within a group; block b runs on XCD b mod 8, and
  // each XCD takes a contiguous run of tiles, so its workgroups read the same slices of w and x through one L2.
  const int n_nt = (a.N + BN - 1) / BN;
  const unsigned per_xcd = gridDim.x / kXcds;   // the grid is a multiple of kXcds
  const unsigned L = blockIdx.x % kXcds * per_xcd + blockIdx.x / kXcds;
  const int n_mt = EXPERTS ? a.m_tiles : a.m_tiles * a.r.n_req;
  const unsigned grp = L / (unsigned)(kRowGroup * n_nt);
  if (grp * kRowGroup >= (unsigned)n_mt) return;
  const int in_g = (int)(L - grp * (kRowGroup * n_nt));
  const int gm = min(kRowGroup, n_mt - (int)grp * kRowGroup);
  const int nt = in_g / gm;
  if (nt >= n_nt) return;
  RowTile t;
  if (!row_tile<BM, EXPERTS>(a, (int)grp * kRowGroup + in_g % gm, lane, &t)) return;
  const int n0 = nt * BN, K = a.K, nb = K / kF8Group;
  const int64_t e = EXPERTS ? t.r : 0;

  // ---- transfers: 1 KB holds rows 8 q .. 8 q + 7 of a tile; lane l fills row 8 q + l / 8, physical chunk l % 8 with the
  // logical chunk that chunk_swz maps there.  A wave moves transfers wu + NW i of both operands. ----
  const uint8_t* const w0 = a.w + (e * a.N + n0) * K;
  const int wrow = 8 * wu + lane / 8;
  // (chunk_swz is an involution; of an odd number of waves every other transfer has the other half's chunk)
  const uint32_t woff[2] = {(uint32_t)(wrow * K + chunk_swz(lane % 8, wrow) * 16),
                            (uint32_t)(wrow * K + chunk_swz(lane % 8, wrow + 8 * (NW % 2)) * 16)};
  const uint8_t* src[PX];
#pragma unroll
  for (int i = 0; i < PX; ++i) {
    const int row = 8 * (wu + NW * i) + lane / 8;
    src[i] = a.x + x_row<EXPERTS>(a, t, min(t.m0 + row, t.nr - 1)) * K + chunk_swz(lane % 8, row) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // transfer d of this wave for block b, into stage b mod NST; no lane takes part behind the last block (a branch would let the
  // compiler move matrix instructions over it)
  auto dma = [&](int b, int d) {
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)(b % NST * STAGE) +
                                                       (uint32_t)(d < PW ? (wu + NW * d) * 1024 : BN * kF8Group + (wu + NW * (d - PW)) * 1024));
    const int lanes = __builtin_amdgcn_readfirstlane(b < nb ? -1 : 0);
    if (d < PW) {
      // (rows behind the weight's last one are read from the tile's first rows and not stored)
      const int row = n0 + 8 * (wu + NW * d) < a.N ? 8 * NW * d : -8 * wu;
      const uint8_t* base = w0 + (int64_t)row * K + b * kF8Group;
      asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\ts_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" ::"v"(woff[d % 2]), "s"(base),
                   "s"(at), "s"(lanes)
                   : "m0", "memory");
    } else {
      asm volatile("s_mov_b32 exec_lo, %2\n\ts_mov_b32 exec_hi, %2\n\ts_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off\n\ts_mov_b64 exec, -1" ::"v"(
                       src[d - PW] + b * kF8Group),
                   "s"(at), "s"(lanes)
                   : "m0", "memory");
    }
  };
  // Before a block is read: this wave's transfers of it have landed (of the NST - 2 blocks behind it they may be in flight) and its
  // reads of the block before are done (the barrier alone does not wait for them), and so are the other waves'; past it
  // the stage of the block before is free.
  auto enter = [&] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    SX_WAIT_VM((NST - 2) * ND & 63);
    __syncthreads();
  };

  const int wn = wu % WN, wm = wu / WN;
  const int lr = lane % 16, g = lane / 16;
  const int nw = n0 + wn * (BN / WN);          // the wave's first feature
  uint32_t lane_off[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) lane_off[h] = (uint32_t)(lr * kF8Group + (chunk_swz(4 * h + g, lr) << 4));
  f32x4_t acc[FI][RJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4_t{};

  SX_WAIT_VM(0);   // the row indices above are the compiler's loads
  // ---- scale bytes, then the first stages ----
  const int words = a.ld / 4;
  const uint32_t xs0 = lds0 + NST * STAGE, ws0 = xs0 + tile_x_scales(BM, a.ld);
  auto dma_word = [&](const uint8_t* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(__builtin_amdgcn_readfirstlane(to)) : "m0", "memory");
  };
  for (int q = wu; q < tile_x_scales(BM, a.ld) / 256; q += NW) {
    const int i = min(q * 64 + lane, BM * words - 1);
    dma_word(a.xs + x_row<EXPERTS>(a, t, min(t.m0 + i % BM, t.nr - 1)) * a.ld + 4 * (i / BM), xs0 + q * 256);
  }
  for (int q = wu; q < (BN + kF8Group - 1) / kF8Group * (tile_w_scales(a.ld) / 256); q += NW) {
    const int per = tile_w_scales(a.ld) / 256, blk = q / per;
    const int64_t at = e * (a.N / kF8Group) + min(n0 / kF8Group + blk, a.N / kF8Group - 1);
    dma_word(a.ws + at * a.ld + 4 * min((q - blk * per) * 64 + lane, words - 1), ws0 + q * 256);
  }
#pragma unroll
  for (int b = 0; b < NST; ++b)
#pragma unroll
    for (int d = 0; d < (b == NST - 1 ? D0 : ND); ++d) dma(b, d);
  SX_WAIT_VM(((NST - 2) * ND + D0) & 63);   // the scale bytes and the first stage
  __syncthreads();

  auto lds16 = [](uint32_t at) { return *(const __attribute__((address_space(3))) i32x4_t*)(uintptr_t)at; };
  auto lds1 = [](uint32_t at) { return (int)*(const __attribute__((address_space(3))) uint8_t*)(uintptr_t)at; };
  const uint32_t ws_at = ws0 + (n0 % kF8Group + wn * (BN / WN)) / kF8Group * tile_w_scales(a.ld);
  const uint32_t xs_at = xs0 + 4 * (wm * (BM / WM) + lr);
  auto w_scale = [&](int b) { return lds1(ws_at + b); };
  auto x_scale = [&](int b, int j) { return lds1(xs_at + (b >> 2) * (4 * BM) + (b & 3) + j * 64); };
  // A block in two halves, the wave's lower features and its upper ones, against all its rows.  Beside the first half the
  // upper features' operands are read; beside the second, once the next block is entered, its lower features' and its
  // rows' into the registers that are free after their last use.  The order is pinned: matrix instruction m, then the reads
  // and transfers due.
  constexpr int FH = FI / 2, HM = FH * RJ, P0 = FH;   // P0: matrix instructions of the second half before the next block is entered
  i32x8_t fw[FI], fx[RJ];
  int sx[RJ], sw;
  const uint32_t wb = lds0 + (uint32_t)(wn * FI * 16 * kF8Group), xb = lds0 + (uint32_t)((BN + wm * RJ * 16) * kF8Group);
  auto read = [&](const uint32_t (&base)[2], int f) {
    return operand(lds16(base[0] + (uint32_t)(f * 16 * kF8Group)), lds16(base[1] + (uint32_t)(f * 16 * kF8Group)));
  };
  auto mfma = [&](int i, int j) { acc[i][j] = mfma_block<0>(fw[i], fx[j], acc[i][j], sw, sx[j]); };
  {
    const uint32_t w0[2] = {wb + lane_off[0], wb + lane_off[1]}, x0[2] = {xb + lane_off[0], xb + lane_off[1]};
#pragma unroll
    for (int j = 0; j < RJ; ++j) {
      fx[j] = read(x0, j);
      sx[j] = x_scale(0, j);
    }
#pragma unroll
    for (int i = 0; i < FH; ++i) fw[i] = read(w0, i);
  }
  sw = w_scale(0);
  __builtin_amdgcn_s_waitcnt(0xF | (3 << 14) | (0x7 << 4));   // lgkmcnt 0: else the loop waits for its last reads at its start
  for (int b = 0; b < nb; ++b) {
    const int next = min(b + 1, nb - 1);   // (what is read behind the last block is never used)
    const uint32_t cur = (uint32_t)(b % NST * STAGE), nxt = (uint32_t)((b + 1) % NST * STAGE);
    // one base register per operand and half of a block (the empty asm keeps the sums from being re-associated into one
    // register per read)
    uint32_t wc[2], wx[2], xx[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      wc[h] = wb + cur + lane_off[h];
      wx[h] = wb + nxt + lane_off[h];
      xx[h] = xb + nxt + lane_off[h];
      asm volatile("" : "+v"(wc[h]), "+v"(wx[h]), "+v"(xx[h]));
    }
#pragma unroll
    for (int m = 0; m < HM; ++m) {
      mfma(m % FH, m / FH);
#pragma unroll
      for (int f = 0; f < FH; ++f)
        if (m == f * (HM > 2 ? HM - 2 : 0) / FH) fw[FH + f] = read(wc, FH + f);
#pragma unroll
      for (int d = D0; d < ND; ++d)
        if (m == min(1 + (d - D0) * 2, HM - 1)) dma(b - 1 + NST, d);
      __builtin_amdgcn_sched_barrier(0);
    }
    int swn = 0;
#pragma unroll
    for (int m = 0; m < HM; ++m) {
      mfma(FH + m % FH, m / FH);
      if (m == P0 - 1) {
        __builtin_amdgcn_sched_barrier(0);
        enter();
        swn = w_scale(next);
      }
#pragma unroll
      for (int f = 0; f < FH; ++f)
        if (m == min(P0 + f * (HM - P0) / FH, HM - 1)) fw[f] = read(wx, f);
#pragma unroll
      for (int f = 0; f < RJ; ++f) {
        if (m == min(max((f + 1) * FH - 1, P0), HM - 1)) {
          fx[f] = read(xx, f);
          sx[f] = x_scale(next, f);
        }
      }
#pragma unroll
      for (int d = 0; d < D0; ++d)
        if (m == min(P0 + d * (HM - P0) / D0, HM - 1)) dma(b + NST, d);
      __builtin_amdgcn_sched_barrier(0);
    }
    sw = swn;
  }

  __syncthreads();   // (all waves have read the stages)
  if (nw < a.N)
    put_tile<FI, RJ, EXPERTS>(a, t, t.m0 + wm * RJ * 16, nw, acc, smem + wu * epilogue_lds<FI, RJ>(), lane);
}

// ---------------------------------------------------------------------------------------------
// Small tiles: a wave's few matrix instructions a block do not cover the way of its operands from LDS, so KB blocks are
// taken at once, with one barrier.  Layout and transfers as above; NST is the number of blocks that LDS holds.
// ---------------------------------------------------------------------------------------------
template <int BN, int BM, int WN, int WM, int KB, int NST, bool EXPERTS>
__global__ __launch_bounds__(WN * WM * 64, 1) void f8_narrow_kernel(F8GemmK a) {
  constexpr int NW = WN * WM;
  constexpr int FI = BN / WN / 16, RJ = BM / WM / 16;       // fragments of a wave
  constexpr int STAGE = (BN + BM) * kF8Group;
  constexpr int PW = BN / 8 / NW, PX = BM / 8 / NW, ND = PW + PX;   // transfers of 1 KB (8 rows) a wave and stage
  static_assert(PW * NW * 8 == BN && PX * NW * 8 == BM, "transfers spread evenly over the waves");
  static_assert(BN / WN <= kF8Group, "a wave's features lie in one block of the weight");
  static_assert(NST % KB == 0 && NST > KB && NST * ND < 64, "transfers in flight");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wu = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Tile order: groups of kRowGroup row tiles, the feature tile slowest within a group; block b runs on XCD b mod 8, and
  // each XCD takes a contiguous run of tiles, so its workgroups read the same slices of w and x through one L2.
  const int n_nt = (a.N + BN - 1) / BN;
  const unsigned per_xcd = gridDim.x / kXcds;   // the grid is a multiple of kXcds
  const unsigned L = blockIdx.x % kXcds * per_xcd + blockIdx.x / kXcds;
  const int n_mt = EXPERTS ? a.m_tiles : a.m_tiles * a.r.n_req;
  const unsigned grp = L / (unsigned)(kRowGroup * n_nt);
  if (grp * kRowGroup >= (unsigned)n_mt) return;
  const int in_g = (int)(L - grp * (kRowGroup * n_nt));
  const int gm = min(kRowGroup, n_mt - (int)grp * kRowGroup);
  const int nt = in_g / gm;
  if (nt >= n_nt) return;
  RowTile t;
  if (!row_tile<BM, EXPERTS>(a, (int)grp * kRowGroup + in_g % gm, lane, &t)) return;
  const int n0 = nt * BN, K = a.K, nb = K / kF8Group;
  const int64_t e = EXPERTS ? t.r : 0;

  // ---- transfers: 1 KB holds rows 8 q .. 8 q + 7 of a tile; lane l fills row 8 q + l / 8, physical chunk l % 8 with the
  // logical chunk that chunk_swz maps there.  A wave moves transfers wu + NW i of both operands. ----
  const uint8_t* const w0 = a.w + (e * a.N + n0) * K;
  const int wrow = 8 * wu + lane / 8;
  // (chunk_swz is an involution; of an odd number of waves every other transfer has the other half's chunk)
  const uint32_t woff[2] = {(uint32_t)(wrow * K + chunk_swz(lane % 8, wrow) * 16),
                            (uint32_t)(wrow * K + chunk_swz(lane % 8, wrow + 8 * (NW % 2)) * 16)};
  const uint8_t* src[PX];
#pragma unroll
  for (int i = 0; i < PX; ++i) {
    const int row = 8 * (wu + NW * i) + lane / 8;
    src[i] = a.x + x_row<EXPERTS>(a, t, min(t.m0 + row, t.nr - 1)) * K + chunk_swz(lane % 8, row) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // transfer d of this wave for block b, into stage b mod NST; no lane takes part behind the last block (a branch would let the
  // compiler move matrix instructions over it)
  auto dma = [&](int b, int d) {
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)(b % NST * STAGE) +
                                                       (uint32_t)(d < PW ? (wu + NW * d) * 1024 : BN * kF8Group + (wu + NW * (d - PW)) * 1024));
    const int lanes = __builtin_amdgcn_readfirstlane(b < nb ? -1 : 0);
    if (d < PW) {
      // (rows behind the weight's last one are read from the tile's first rows and not stored)
      const int row = n0 + 8 * (wu + NW * d) < a.N ? 8 * NW * d : -8 * wu;
      const uint8_t* base = w0 + (int64_t)row * K + b * kF8Group;
      asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\ts_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" ::"v"(woff[d % 2]), "s"(base),
                   "s"(at), "s"(lanes)
                   : "m0", "memory");
    } else {
      asm volatile("s_mov_b32 exec_lo, %2\n\ts_mov_b32 exec_hi, %2\n\ts_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off\n\ts_mov_b64 exec, -1" ::"v"(
                       src[d - PW] + b * kF8Group),
                   "s"(at), "s"(lanes)
                   : "m0", "memory");
    }
  };
  const int wn = wu % WN, wm = wu / WN;
  const int lr = lane % 16, g = lane / 16;
  const int nw = n0 + wn * (BN / WN);          // the wave's first feature
  uint32_t lane_off[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) lane_off[h] = (uint32_t)(lr * kF8Group + (chunk_swz(4 * h + g, lr) << 4));
  f32x4_t acc[FI][RJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4_t{};

  SX_WAIT_VM(0);   // the row indices above are the compiler's loads
  // ---- scale bytes, then the first stages ----
  const int words = a.ld / 4;
  const uint32_t xs0 = lds0 + NST * STAGE, ws0 = xs0 + tile_x_scales(BM, a.ld);
  auto dma_word = [&](const uint8_t* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(__builtin_amdgcn_readfirstlane(to)) : "m0", "memory");
  };
  for (int q = wu; q < tile_x_scales(BM, a.ld) / 256; q += NW) {
    const int i = min(q * 64 + lane, BM * words - 1);
    dma_word(a.xs + x_row<EXPERTS>(a, t, min(t.m0 + i % BM, t.nr - 1)) * a.ld + 4 * (i / BM), xs0 + q * 256);
  }
  for (int q = wu; q < (BN + kF8Group - 1) / kF8Group * (tile_w_scales(a.ld) / 256); q += NW) {
    const int per = tile_w_scales(a.ld) / 256, blk = q / per;
    const int64_t at = e * (a.N / kF8Group) + min(n0 / kF8Group + blk, a.N / kF8Group - 1);
    dma_word(a.ws + at * a.ld + 4 * min((q - blk * per) * 64 + lane, words - 1), ws0 + q * 256);
  }
#pragma unroll
  for (int b = 0; b < NST; ++b)
#pragma unroll
    for (int d = 0; d < ND; ++d) dma(b, d);
  auto lds16 = [](uint32_t at) { return *(const __attribute__((address_space(3))) i32x4_t*)(uintptr_t)at; };
  auto lds1 = [](uint32_t at) { return (int)*(const __attribute__((address_space(3))) uint8_t*)(uintptr_t)at; };
  const uint32_t ws_at = ws0 + (n0 % kF8Group + wn * (BN / WN)) / kF8Group * tile_w_scales(a.ld);
  const uint32_t xs_at = xs0 + 4 * (wm * (BM / WM) + lr);
  auto w_scale = [&](int b) { return lds1(ws_at + b); };
  auto x_scale = [&](int b, int j) { return lds1(xs_at + (b >> 2) * (4 * BM) + (b & 3) + j * 64); };
  i32x8_t fw[KB][FI], fx[KB][RJ];
  int sw[KB], sx[KB][RJ];
  auto read = [&](uint32_t base) { return operand(lds16(base + lane_off[0]), lds16(base + lane_off[1])); };
  const uint32_t wb = lds0 + (uint32_t)(wn * FI * 16 * kF8Group), xb = lds0 + (uint32_t)((BN + wm * RJ * 16) * kF8Group);
  for (int b = 0; b < nb; b += KB) {
    // the KB blocks have landed: all transfers but those of the NST - 2 KB (at first NST - KB) blocks behind them, and all
    // waves have read the KB before, whose stages are refilled
    if (b == 0) SX_WAIT_VM((NST - KB) * ND & 63);
    else SX_WAIT_VM((NST - 2 * KB) * ND & 63);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int s = 0; s < KB; ++s) {
      const uint32_t at = (uint32_t)((b + s) % NST * STAGE);
      const int c = min(b + s, nb - 1);   // (what is read behind the last block is never used)
#pragma unroll
      for (int i = 0; i < FI; ++i) fw[s][i] = read(wb + at + (uint32_t)(i * 16 * kF8Group));
#pragma unroll
      for (int j = 0; j < RJ; ++j) {
        fx[s][j] = read(xb + at + (uint32_t)(j * 16 * kF8Group));
        sx[s][j] = x_scale(c, j);
      }
      sw[s] = w_scale(c);
    }
    if (b > 0)
#pragma unroll
      for (int s = 0; s < KB; ++s)
#pragma unroll
        for (int d = 0; d < ND; ++d) dma(b - KB + NST + s, d);
#pragma unroll
    for (int s = 0; s < KB; ++s)
      if (b + s < nb)
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
          for (int j = 0; j < RJ; ++j) acc[i][j] = mfma_block<0>(fw[s][i], fx[s][j], acc[i][j], sw[s], sx[s][j]);
  }

  __syncthreads();   // (all waves have read the stages)
  if (nw < a.N)
    put_tile<FI, RJ, EXPERTS>(a, t, t.m0 + wm * RJ * 16, nw, acc, smem + wu * epilogue_lds<FI, RJ>(), lane);
}

// Row tiles of BM rows that the launch may have to take.
int64_t count_tiles(const F8GemmK& a, int bm) {
  if (!a.offsets) return (int64_t)a.r.n_req * ((a.r.max_rows + bm - 1) / bm);
  return a.n_places / bm + (int64_t)(a.n_experts < a.n_places ? a.n_experts : a.n_places);
}

template <int FI, int RJ, int D>
hipError_t launch_stream(F8GemmK& a, hipStream_t s) {
  a.m_tiles = (a.r.max_rows + 16 * RJ - 1) / (16 * RJ);
  const int64_t blocks = count_tiles(a, 16 * RJ) * (a.N / (16 * FI));
  if (blocks >= ((int64_t)1 << 31)) return hipErrorInvalidConfiguration;
  if (a.offsets)
    hipLaunchKernelGGL((f8_stream_kernel<FI, RJ, D, true>), dim3((unsigned)blocks), dim3(64), 0, s, a);
  else
    hipLaunchKernelGGL((f8_stream_kernel<FI, RJ, D, false>), dim3((unsigned)blocks), dim3(64), 0, s, a);
  return hipGetLastError();
}

// Grid and LDS of a tiled launch; kernel(experts) is the kernel.
template <int BN, int BM, int WN, int WM, int NST, typename K>
hipError_t launch_tiled(F8GemmK& a, hipStream_t s, K plain, K experts) {
  const int64_t m_tiles = count_tiles(a, BM);
  a.m_tiles = a.offsets ? (int)m_tiles : (a.r.max_rows + BM - 1) / BM;
  const int64_t blocks = (m_tiles * ((a.N + BN - 1) / BN) + kXcds - 1) / kXcds * kXcds;
  const int lds = std::max(tile_lds<BN, BM, NST>(a.ld), WN * WM * epilogue_lds<BN / WN / 16, BM / WM / 16>());
  if (blocks >= ((int64_t)1 << 31) || lds > kLdsBytes) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(a.offsets ? experts : plain, dim3((unsigned)blocks), dim3(WN * WM * 64), lds, s, a);
  return hipGetLastError();
}
template <int BN, int BM, int WN, int WM, int NST>
hipError_t launch_tile(F8GemmK& a, hipStream_t s) {
  return launch_tiled<BN, BM, WN, WM, NST>(a, s, f8_tile_kernel<BN, BM, WN, WM, NST, false>, f8_tile_kernel<BN, BM, WN, WM, NST, true>);
}
template <int BN, int BM, int WN, int WM, int KB, int NST>
hipError_t launch_narrow(F8GemmK& a, hipStream_t s) {
  return launch_tiled<BN, BM, WN, WM, NST>(a, s, f8_narrow_kernel<BN, BM, WN, WM, KB, NST, false>,
                                           f8_narrow_kernel<BN, BM, WN, WM, KB, NST, true>);
}

// A launch's shape: what a round of workgroups over the compute units (occ on each) takes, per block of k and besides.
struct Shape {
  int bn, bm, nst, occ;
  double block, round;   // us
};
enum { kStream, k16x16, k64x32, k64x64, k128x64, k128x128, k128x128x2, k256x256, kShapes };
constexpr Shape kShape[kShapes] = {{16, 16, 0, 1, 0.16, 0.5},    {16, 16, 12, 3, 0.19, 1.2},  {64, 32, 10, 1, 0.245, 1.5},
                                   {64, 64, 6, 1, 0.27, 1.5},    {128, 64, 3, 2, 0.47, 2},    {128, 128, 4, 1, 0.55, 1.5},
                                   {128, 128, 2, 2, 1.05, 3},    {256, 256, 2, 1, 1.14, 9}};

// The shape of least time for listed rows.  Measured (us, K = 4096, weights from memory; the shape taken first, then its
// neighbours): 16 rows x 4096 features 8.7, 9.5, 11.4; 32 x 6144 10.1, 11.7, 12.3; 64 x 6144 11.8, 12.4, 19.9; 128 x 6144
// 12.6, 13.8, 21.3; 394 x 4096 16.0, 20.0, 22.7; 1000 x 6144 35.9, 32.5, 38.4; 6712 x 28672 662, 862, 929.
int best_shape(const F8GemmK& a, int n_cu) {
  int best = k64x32;
  double least = 1e300;
  const double nb = a.K / kF8Group;
  for (int i = 0; i < kShapes; ++i) {
    const Shape& h = kShape[i];
    const int64_t tiles = count_tiles(a, h.bm) * ((a.N + h.bn - 1) / h.bn);
    if (h.nst * (h.bn + h.bm) * kF8Group + tile_x_scales(h.bm, a.ld) + (h.bn + kF8Group - 1) / kF8Group * tile_w_scales(a.ld) > kLdsBytes ||
        tiles >= ((int64_t)1 << 31) - 64)
      continue;
    const double t = (double)((tiles + n_cu * h.occ - 1) / (n_cu * h.occ)) * (nb * h.block + h.round);
    if (t < least) {
      least = t;
      best = i;
    }
  }
  return best;
}

// Grouped rows, by the rows an expert has on average: few, a wave of its own reads each expert's weights past LDS (64 tokens
// x 8 of 128 experts, 2048 -> 1536: 62 us; 128 x 64 tiles 73, 256 x 256 131); many, 128 x 64 tiles (512 tokens 100; 132, 142)
// or, from 192 on, the largest of which a block's prologue does not take longer than its products (8192 tokens, 2048 ->
// 1536: 256 x 256 332, 128 x 128 380; 768 -> 2048: 259 of 128 x 128, 261).
int expert_shape(const F8GemmK& a) {
  const double rows = (double)a.n_places / a.n_experts;
  if (rows <= 12) return kStream;
  const bool fits = a.ld <= 112;   // (of 256 x 256 tiles)
  return rows < 192 ? k128x64 : a.K <= 1024 || !fits ? k128x128x2 : k256x256;
}

}  // namespace

hipError_t launch_gemm_f8(F8GemmK& a, int n_cu, hipStream_t s) {
  switch (a.offsets ? expert_shape(a) : best_shape(a, n_cu)) {
    case kStream: return a.offsets ? launch_stream<2, 2, 4>(a, s) : launch_stream<1, 1, 8>(a, s);
    case k16x16: return launch_narrow<16, 16, 1, 1, 4, 12>(a, s);
    case k64x32: return launch_narrow<64, 32, 4, 1, 2, 10>(a, s);
    case k64x64: return launch_narrow<64, 64, 2, 2, 2, 6>(a, s);
    case k128x64: return launch_narrow<128, 64, 4, 2, 1, 3>(a, s);
    case k128x128: return launch_narrow<128, 128, 4, 2, 1, 4>(a, s);
    case k128x128x2: return launch_narrow<128, 128, 4, 2, 1, 2>(a, s);
    default: return launch_tile<256, 256, 2, 2, 2>(a, s);
  }
}

}  // namespace sx
