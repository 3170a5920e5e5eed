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
#include <cmath>
#include <type_traits>
#include <utility>

#include "sx_f8_device.h"

namespace sx {
namespace {

typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
// the same place in LDS written in one width and read in the other
typedef i32x2_t Alias2 __attribute__((may_alias));
typedef i32x4_t Alias4 __attribute__((may_alias));
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

// Inclusive prefix sums over the lanes of a wave.
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15, 31
  return x + __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
}

// Row tile number `idx` of the launch; false where there is none.  Experts: the tiles of 128 of them at a time, so that one
// round trip to memory finds most.
template <int BM, bool EXPERTS>
__device__ __forceinline__ bool row_tile(const F8GemmK& a, int idx, int lane, RowTile* t) {
  if constexpr (EXPERTS) {
    int base = 0;
    for (int e0 = 0; e0 < a.n_experts; e0 += 128) {
      int first[2], len[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int e = e0 + 64 * h + lane;
        first[h] = min(max(a.offsets[min(e, a.n_experts)], 0), a.n_places);
        len[h] = max(min(max(a.offsets[min(e + 1, a.n_experts)], 0), a.n_places) - first[h], 0);   // (0 behind the last expert)
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = (len[h] + BM - 1) / BM, upto = base + wave_prefix(c);
        const uint64_t m = __ballot(upto > idx);
        if (m != 0) {
          const int l = (int)__builtin_ctzll(m);
          const int before = __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(c, l);
          *t = {e0 + 64 * h + l, (idx - before) * BM, __builtin_amdgcn_readlane(len[h], l), __builtin_amdgcn_readlane(first[h], l)};
          return true;
        }
        base = __builtin_amdgcn_readlane(upto, 63);
      }
    }
    return false;
  } else {
    const int r = idx / a.m_tiles;
    *t = {r, (idx - r * a.m_tiles) * BM, f8_count(a.r, r), 0};
    return t->m0 < t->nr;
  }
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

__device__ __forceinline__ int part_of(const F8GemmK& a, int n) {
  int p = 0;
  while (p + 1 < a.n_parts && n >= a.pn[p + 1]) ++p;
  return p;
}

// Lanes of one wave exchange data through LDS, whose accesses the wave makes in order; what keeps the compiler from handing a
// lane's own earlier store to its later load.
__device__ __forceinline__ void wave_exchange() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// A wave's results, FI x RJ fragments, through its own part of LDS (epilogue_lds bytes), so that rows go out in whole runs
// of 32 FI bytes: a store of the fragments themselves (4 features a lane) touches 16 rows at 32 bytes each.  yrow (LDS):
// where the wave's rows lie in y, -1 for none; features nw .. of one part.  16 rows at a time; a residual is fetched ahead,
// and into the same places first; the stores follow a step behind (8192 tokens x 8 of 128 experts, 768 -> 2048: 201 us, 207
// with each behind its own exchange).
template <int FI>
constexpr int epilogue_lds() { return 16 * (32 * FI + 16); }   // (16 bytes a row against bank conflicts)
// AGPR: the sums are in accumulation registers; the empty asm keeps the compiler from fetching all of them at once.
// PRE: `pre` holds the residual already, of all rows.
template <int FI>
constexpr int put_loads() { return (16 + 32 / FI - 1) / (32 / FI); }   // instructions for 16 rows
template <bool AGPR, bool RES, bool PRE, int FI, int RJ>
__device__ __forceinline__ void put_rows(const F8GemmK& a, const int* yrow, int nw, const f32x4_t (&acc)[FI][RJ],
                                         const i32x4_t (&pre)[RJ][put_loads<FI>()], char* lds, int lane) {
  constexpr int LD = 32 * FI + 16, CH = 2 * FI, RPI = 64 / CH, IT = put_loads<FI>();   // 16-byte chunks of a row, rows an instruction
  static_assert(64 % CH == 0, "whole rows an instruction");
  const int lr = lane % 16, g = lane / 16;
  const int part = part_of(a, nw);
  const uint32_t ld = (uint32_t)(a.pn[part + 1] - a.pn[part]);
  const int col = nw - a.pn[part] + lane % CH * 8;
  uint16_t* const to = a.y[part] + col;
  const uint16_t* const from = a.res + col;
  auto row_of = [&](int j, int it) { return RPI > 16 && lane / CH >= 16 ? -1 : yrow[16 * j + it * RPI + lane / CH]; };
  int row[2][IT];           // of rows j and j + 1
  i32x4_t res[IT], q[IT];   // rows j's residual, rows j - 1's results
  auto rows = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < IT; ++it) row[j % 2][it] = row_of(j, it);
  };
  auto fetch = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      if constexpr (PRE) res[it] = pre[j][it];
      else res[it] = row[j % 2][it] >= 0 ? *(const i32x4_t*)(from + (uint64_t)(uint32_t)row[j % 2][it] * ld) : i32x4_t{};
    }
  };
  char* const mine = lds + lane / CH * LD + lane % CH * 16;
  auto store = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < IT; ++it)
      if (row[j % 2][it] >= 0) *(i32x4_t*)(to + (uint64_t)(uint32_t)row[j % 2][it] * ld) = q[it];
  };
  rows(0);
  if constexpr (RES) fetch(0);
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    if constexpr (RES) {
#pragma unroll
      for (int it = 0; it < IT; ++it)
        if (RPI <= 16 || lane / CH < 16) *(Alias4*)(mine + it * RPI * LD) = res[it];
      wave_exchange();
    }
    i32x2_t o[FI];
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      f32x4_t v = acc[i][j];
      if constexpr (AGPR) asm volatile("" : "+a"(v)::"memory");
      if constexpr (RES) {
        const i32x2_t rv = *(const Alias2*)(lds + lr * LD + 32 * i + 8 * g);
        v[0] += bf16_lo((uint32_t)rv[0]);
        v[1] += bf16_hi((uint32_t)rv[0]);
        v[2] += bf16_lo((uint32_t)rv[1]);
        v[3] += bf16_hi((uint32_t)rv[1]);
      }
      o[i] = i32x2_t{(int)pack_bf16x2(v[0], v[1]), (int)pack_bf16x2(v[2], v[3])};
    }
    if (j > 0) {
      store(j - 1);
      wave_exchange();
    }
#pragma unroll
    for (int i = 0; i < FI; ++i) *(Alias2*)(lds + lr * LD + 32 * i + 8 * g) = o[i];
    if (j + 1 < RJ) {
      rows(j + 1);
      if constexpr (RES) fetch(j + 1);
    }
    wave_exchange();
#pragma unroll
    for (int it = 0; it < IT; ++it) q[it] = *(const Alias4*)(mine + it * RPI * LD);
    wave_exchange();
  }
  store(RJ - 1);
}
// (One branch: a load that some path leaves in flight would have the compiler wait for all transfers in the next loop.)
template <bool AGPR, bool PRE, int FI, int RJ>
__device__ __forceinline__ void put_tile(const F8GemmK& a, const int* yrow, int nw, const f32x4_t (&acc)[FI][RJ],
                                         const i32x4_t (&pre)[RJ][put_loads<FI>()], char* lds, int lane) {
  if (a.res) put_rows<AGPR, true, PRE>(a, yrow, nw, acc, pre, lds, lane);
  else put_rows<AGPR, false, PRE>(a, yrow, nw, acc, pre, lds, lane);
}
template <bool AGPR, int FI, int RJ>
__device__ __forceinline__ void put_tile(const F8GemmK& a, const int* yrow, int nw, const f32x4_t (&acc)[FI][RJ], char* lds, int lane) {
  const i32x4_t none[RJ][put_loads<FI>()] = {};
  put_tile<AGPR, false>(a, yrow, nw, acc, none, lds, lane);
}

// ---------------------------------------------------------------------------------------------
// Few rows: a wave of its own takes 16 FI features and 16 RJ rows and reads both operands from memory into registers, D
// blocks of k ahead, so no wave waits for another and nothing passes through LDS.  Bound by memory where every weight serves
// one wave (64 tokens x 8 of 128 experts, 2048 -> 1536: 322 MB in 60 us, 5.4 TB/s; 1 row x 4096 x 14336, 59 MB in 17 us), and
// beyond by the loads, whose instructions touch 16 lines of memory for a kilobyte (64 rows x 6144 x 4096: 26 us, 12 by 64 x 32
// tiles through LDS).
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
  // four consecutive features of a row a lane and fragment: where they go, and the residual ahead of all else
  const int part = part_of(a, n0), ld = a.pn[part + 1] - a.pn[part], col = n0 - a.pn[part] + 4 * g;
  int64_t y[RJ];
  uint2 res[FI][RJ];
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    const int m = t.m0 + 16 * j + lr;
    y[j] = m < t.nr ? y_row<EXPERTS>(a, t, m) : -1;
    if (!EXPERTS && a.res)
#pragma unroll
      for (int i = 0; i < FI; ++i) res[i][j] = y[j] >= 0 ? *(const uint2*)(a.res + y[j] * ld + col + 16 * i) : make_uint2(0, 0);
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
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    if (y[j] >= 0) {
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        f32x4_t v = acc[i][j];
        if (!EXPERTS && a.res) {
          v[0] += bf16_lo(res[i][j].x);
          v[1] += bf16_hi(res[i][j].x);
          v[2] += bf16_lo(res[i][j].y);
          v[3] += bf16_hi(res[i][j].y);
        }
        *(uint2*)(a.y[part] + y[j] * ld + col + 16 * i) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Tiles of BN features x BM rows, WN x WM waves; a workgroup takes a.run of them, one beside the other, of the same rows.
// Blocks of k move through NST stages of LDS, global -> LDS directly, those of the next tile behind the last one's; a tile
// row (one block, 128 bytes) holds 8 chunks of 16 bytes, XOR-swizzled per row so that the 16 rows of a read hit distinct
// banks.  The scale bytes go ahead of the first stage the same way, for all of k and all tiles of the run.
//
// Bound: by the matrix cores and LDS alike in the largest tiles, 256 x 256 by four waves of 128 x 128 with their 256 sums in
// accumulation registers: of a block 2112 cycles of matrix instructions, 1344 of transfers and 1024 of reads.  6712 x
// 28672 x 4096 in 617 to 644 us by the card's clock, 2.45 to 2.55 PFLOP/s; without storing results 552 where it took 621: a
// tile's exchange through LDS is 2 us, its stores are 4.5.  By LDS and the length of the chain over k in the small ones: see
// there.
// ---------------------------------------------------------------------------------------------
constexpr int kLdsBytes = 163840;   // LDS of a compute unit
constexpr unsigned kXcds = 8;       // XCDs of the chip, which deals workgroups round-robin
constexpr int kRowGroup = 8;        // row tiles per group of the tile order (6712 x 28672 x 4096: of 4, 8, 16 625, 640, 647 us)

// s_waitcnt with vmcnt <= n (n < 64), expcnt and lgkmcnt left unconstrained (gfx9 encoding)
#define SX_WAIT_VM(n) __builtin_amdgcn_s_waitcnt(((n) & 0xF) | ((((n) >> 4) & 3) << 14) | (0x7 << 4) | (0xF << 8))

__device__ __forceinline__ int chunk_swz(int c, int row) { return c ^ ((row >> 1) & 7); }   // (two rows per 256-byte line)

// Bytes of LDS: the stages, the scale bytes of x as [word][BM] words, those of the run's blocks of w, each of them padded to
// whole transfers of 64 words, and where the rows lie in y.  The results of a run go through a place of their own behind
// that, those of a single tile through the stages.
__host__ __device__ constexpr int tile_x_scales(int bm, int ld) { return (bm * ld + 255) / 256 * 256; }
__host__ __device__ constexpr int tile_w_scales(int bn, int ld) { return (bn + kF8Group - 1) / kF8Group * ((ld + 255) / 256 * 256); }
__host__ __device__ constexpr int tile_fixed(int bn, int bm, int nst, int ld, int run) {
  return nst * (bn + bm) * kF8Group + tile_x_scales(bm, ld) + run * tile_w_scales(bn, ld) + 4 * bm;
}

// A block of k of a run: its tile, the block, its stage, and for its transfers: the stage's address in LDS with the wave's
// first kilobyte, the tile's weights at this block, how many transfers of w the wave has (fewer where the weight ends
// inside the tile), and all lanes, or none behind the last block.
struct Place {
  int tile, b, stage;
  uint32_t lds;
  const uint8_t* w;
  int dw, lanes;
};

template <int BN, int BM, int WN, int WM, int NST, bool EXPERTS>
struct Feed {
  static constexpr int NW = WN * WM, FI = BN / WN / 16, RJ = BM / WM / 16;
  static constexpr int STAGE = (BN + BM) * kF8Group;
  static constexpr int PW = BN / 8 / NW, PX = BM / 8 / NW, ND = PW + PX;   // transfers of 1 KB (8 rows) a wave and block
  static_assert(PW * NW * 8 == BN && PX * NW * 8 == BM, "transfers spread evenly over the waves");
  static_assert(BN / WN <= kF8Group, "a wave's features lie in one block of the weight");

  const F8GemmK& a;
  const int lane, wu, lr, g, wn, wm;
  int n0, nb, tiles;           // first feature, blocks of k, tiles of the run
  int dw_last;                 // the wave's transfers of w in the run's last tile
  int64_t to_next;             // from the last block of a tile's weights to the next tile's first
  uint32_t woff[PW];
  const uint8_t* src[PX];
  uint32_t lds0, xs_at, ws_at;
  int* yrow;                   // of the wave's rows
  char* out;                   // the wave's place for results

  __device__ __forceinline__ Feed(const F8GemmK& arg, int tid)
      : a(arg), lane(tid & 63), wu(__builtin_amdgcn_readfirstlane(tid >> 6)), lr(lane % 16), g(lane / 16), wn(wu % WN), wm(wu / WN) {}

  __device__ __forceinline__ Place begin(const uint8_t* w) const {
    return {0, 0, 0, lds0 + (uint32_t)wu * 1024, w, tiles > 1 ? PW : dw_last, -1};
  }
  // (without branches, over which the compiler would move matrix instructions)
  __device__ __forceinline__ void advance(Place& p) const {
    const bool wrap = p.stage + 1 == NST, last = p.b + 1 == nb;
    p.stage = wrap ? 0 : p.stage + 1;
    p.lds = wrap ? lds0 + (uint32_t)wu * 1024 : p.lds + STAGE;
    p.w += last ? to_next : kF8Group;
    p.b = last ? 0 : p.b + 1;
    p.tile += last ? 1 : 0;
    p.dw = p.tile + 1 < tiles ? PW : p.tile < tiles ? dw_last : 0;
    p.lanes = p.tile < tiles ? -1 : 0;
  }

  // Transfer d of this wave for the block at p; no lane takes part where there is none (a branch would let the compiler move
  // matrix instructions over it).  A memory instruction may read a scalar register five wait states after a vector
  // instruction, such as readfirstlane, wrote it, and a transfer to LDS m0 one wait
  // state after a scalar instruction wrote it; the compiler does not see into the statement, so they are kept there.
  __device__ __forceinline__ void dma(const Place& p, int d) const {
    const int dw = __builtin_amdgcn_readfirstlane(p.dw), lanes = __builtin_amdgcn_readfirstlane(p.lanes);
    const uint32_t lds = __builtin_amdgcn_readfirstlane(p.lds);
    const uint64_t wp = (uint64_t)p.w;
    const uint64_t w = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(wp >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)wp);
    if (d < PW)
      asm volatile("s_add_u32 m0, %4, %5\n\ts_cmp_gt_i32 %2, %3\n\ts_cselect_b32 exec_lo, -1, 0\n\ts_cselect_b32 exec_hi, -1, 0\n\t"
                   "s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" ::"v"(woff[d]), "s"(w), "s"(dw), "n"(d), "s"(lds),
                   "n"(NW * d * 1024)
                   : "m0", "scc", "memory");
    else
      asm volatile("s_add_u32 m0, %2, %3\n\ts_mov_b32 exec_lo, %1\n\ts_mov_b32 exec_hi, %1\n\t"
                   "global_load_lds_dwordx4 %0, off\n\ts_mov_b64 exec, -1" ::"v"(src[d - PW] + p.b * kF8Group), "s"(lanes), "s"(lds),
                   "n"(BN * kF8Group + NW * (d - PW) * 1024)
                   : "m0", "scc", "memory");
  }
  __device__ __forceinline__ void dma_word(const uint8_t* from, uint32_t to) const {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(__builtin_amdgcn_readfirstlane(to)) : "m0", "memory");
  }

  // The workgroup's run, its addresses and its scale bytes on their way; false where there is nothing to do.
  // Tile order: groups of kRowGroup row tiles, the run slowest within a group; block b runs on XCD b mod 8, and each XCD
  // takes a contiguous part of the order, so its workgroups read the same slices of w and x through one L2.
  __device__ __forceinline__ bool start(char* smem, Place* fill, i32x4_t (*pre)[put_loads<FI>()] = nullptr) {
    const int n_nt = (a.N + BN - 1) / BN, n_runs = (n_nt + a.run - 1) / a.run;
    const unsigned per_xcd = gridDim.x / kXcds;   // the grid is a multiple of kXcds
    const unsigned L = blockIdx.x % kXcds * per_xcd + blockIdx.x / kXcds;
    const int n_mt = EXPERTS ? a.m_tiles : a.m_tiles * a.r.n_req;
    const unsigned grp = L / (unsigned)(kRowGroup * n_runs);
    if (grp * kRowGroup >= (unsigned)n_mt) return false;
    const int in_g = (int)(L - grp * (kRowGroup * n_runs));
    const int gm = min(kRowGroup, n_mt - (int)grp * kRowGroup);
    const int run = in_g / gm;
    if (run >= n_runs) return false;
    RowTile t;
    if (!row_tile<BM, EXPERTS>(a, (int)grp * kRowGroup + in_g % gm, lane, &t)) return false;
    n0 = run * a.run * BN;
    tiles = min(a.run, n_nt - run * a.run);
    nb = a.K / kF8Group;
    const int K = a.K;
    const int64_t e = EXPERTS ? t.r : 0;
    to_next = (int64_t)BN * K - (int64_t)(nb - 1) * kF8Group;
    dw_last = min((max(a.N - n0 - (tiles - 1) * BN - 8 * wu, 0) + 8 * NW - 1) / (8 * NW), PW);
    // transfers: 1 KB holds rows 8 q .. 8 q + 7 of a tile; lane l fills row 8 q + l / 8, physical chunk l % 8 with the
    // logical chunk that chunk_swz maps there (an involution).  A wave moves transfers wu + NW i of both operands.
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int row = 8 * (wu + NW * i) + lane / 8;
      woff[i] = (uint32_t)(row * K + chunk_swz(lane % 8, row) * 16);
    }
#pragma unroll
    for (int i = 0; i < PX; ++i) {
      const int row = 8 * (wu + NW * i) + lane / 8;
      src[i] = a.x + x_row<EXPERTS>(a, t, min(t.m0 + row, t.nr - 1)) * K + chunk_swz(lane % 8, row) * 16;
    }
    lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    *fill = begin(a.w + (e * a.N + n0) * K);
    const int words = a.ld / 4;
    const uint32_t xs0 = lds0 + NST * STAGE, ws0 = xs0 + tile_x_scales(BM, a.ld);
    xs_at = xs0 + 4 * (wm * (BM / WM) + lr);
    ws_at = ws0 + (n0 % kF8Group + wn * (BN / WN)) / kF8Group * ((a.ld + 255) / 256 * 256);
    int* const rows = (int*)(smem + tile_fixed(BN, BM, NST, a.ld, a.run) - 4 * BM);
    yrow = rows + wm * (BM / WM);
    out = (a.run > 1 ? smem + tile_fixed(BN, BM, NST, a.ld, a.run) : smem) + wu * epilogue_lds<FI>();
    if (lane + 64 * wu < BM) rows[lane + 64 * wu] = t.m0 + lane + 64 * wu < t.nr ? (int)y_row<EXPERTS>(a, t, t.m0 + lane + 64 * wu) : -1;
    if constexpr (BM > 64 * NW) static_assert(BM <= 64 * NW, "a row a thread");
    if (!EXPERTS && pre && a.res) {   // the residual, ahead of all transfers (of one tile, whose sums it meets in put_rows)
      constexpr int CH = 2 * FI, RPI = 64 / CH;
      const int col = n0 + wn * (BN / WN) + lane % CH * 8;
#pragma unroll
      for (int j = 0; j < RJ; ++j)
#pragma unroll
        for (int it = 0; it < put_loads<FI>(); ++it) {
          const int m = t.m0 + wm * (BM / WM) + 16 * j + it * RPI + lane / CH;
          const int64_t y = (RPI > 16 && lane / CH >= 16) || m >= t.nr ? -1 : y_row<EXPERTS>(a, t, m);
          pre[j][it] = y >= 0 ? *(const i32x4_t*)(a.res + y * a.N + col) : i32x4_t{};
        }
    } else {
      SX_WAIT_VM(0);   // the indices above are the compiler's loads
    }
    for (int q = wu; q < tile_x_scales(BM, a.ld) / 256; q += NW) {
      const int i = min(q * 64 + lane, BM * words - 1);
      dma_word(a.xs + x_row<EXPERTS>(a, t, min(t.m0 + i % BM, t.nr - 1)) * a.ld + 4 * (i / BM), xs0 + q * 256);
    }
    // (a row of w's scale bytes after the other: those of a tile's blocks, tile after tile)
    const int per = (a.ld + 255) / 256, blocks = (BN + kF8Group - 1) / kF8Group;
    for (int q = wu; q < tiles * blocks * per; q += NW) {
      const int row = q / per;
      const int64_t at = e * (a.N / kF8Group) + min((n0 + row / blocks * BN) / kF8Group + row % blocks, a.N / kF8Group - 1);
      dma_word(a.ws + at * a.ld + 4 * min((q - row * per) * 64 + lane, words - 1), ws0 + q * 256);
    }
    return true;
  }
  __device__ __forceinline__ static i32x4_t lds16(uint32_t at) { return *(const __attribute__((address_space(3))) i32x4_t*)(uintptr_t)at; }
  __device__ __forceinline__ static int lds1(uint32_t at) { return (int)*(const __attribute__((address_space(3))) uint8_t*)(uintptr_t)at; }
  __device__ __forceinline__ static int lds4(uint32_t at) { return *(const __attribute__((address_space(3))) int*)(uintptr_t)at; }
  __device__ __forceinline__ int w_scale(int tile, int b) const { return lds1(ws_at + min(tile, tiles - 1) * tile_w_scales(BN, a.ld) + b); }
  __device__ __forceinline__ int x_scale(int b, int j) const { return lds1(xs_at + (b >> 2) * (4 * BM) + (b & 3) + j * 64); }
};

// Large tiles.  While the matrix instructions of a block run, the operands of the next one are read, and a stage is refilled
// as soon as all waves have read it.  One loop without branches: over a branch, or in a second copy of the loop, the
// compiler moves the accumulation registers about.
template <int BN, int BM, int WN, int WM, int NST, bool EXPERTS>
__global__ __launch_bounds__(WN * WM * 64, 1) void f8_tile_kernel(F8GemmK a) {
  typedef Feed<BN, BM, WN, WM, NST, EXPERTS> F;
  constexpr int FI = F::FI, RJ = F::RJ, ND = F::ND, STAGE = F::STAGE;
  // transfers that refill a stage are issued from the entry of the next block on: D0 of them beside a block's second half,
  // the others beside the next one's first
  constexpr int D0 = (ND * 3 + 3) / 4;
  static_assert(FI % 2 == 0, "two halves");
  static_assert((NST - 1) * ND < 64, "transfers in flight");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  F f(a, threadIdx.x);
  Place fill;
  if (!f.start(smem, &fill)) return;
  Place late = fill, cur = fill;
#pragma unroll
  for (int b = 0; b < NST; ++b) {
    late = fill;
#pragma unroll
    for (int d = 0; d < (b == NST - 1 ? D0 : ND); ++d) f.dma(fill, d);
    f.advance(fill);
  }
  SX_WAIT_VM(((NST - 2) * ND + D0) & 63);   // the scale bytes and the first stage
  __syncthreads();
  // Before a block is read: this wave's transfers of it have landed (of the NST - 2 blocks behind it they may be in flight) and its
  // reads of the block before are done (the barrier alone does not wait for them), and so are the other waves'; past it
  // the stage of the block before is free.
  auto enter = [&] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    SX_WAIT_VM((NST - 2) * ND & 63);
    __syncthreads();
  };
  uint32_t lane_off[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) lane_off[h] = (uint32_t)(f.lr * kF8Group + (chunk_swz(4 * h + f.g, f.lr) << 4));
  f32x4_t acc[FI][RJ];
  // A block in two halves, the wave's lower features and its upper ones, against all its rows.  Beside the first half the
  // upper features' operands are read; beside the second, once the next block is entered, its lower features' and its
  // rows' into the registers that are free after their last use.  The order is pinned: matrix instruction m, then the reads
  // and transfers due.
  constexpr int FH = FI / 2, HM = FH * RJ, P0 = FH;   // P0: matrix instructions of the second half before the next block is entered
  i32x8_t fw[FI], fx[RJ];
  int sx[RJ], sw;
  const uint32_t wb = f.lds0 + (uint32_t)(f.wn * FI * 16 * kF8Group), xb = f.lds0 + (uint32_t)((BN + f.wm * RJ * 16) * kF8Group);
  auto read = [&](const uint32_t (&base)[2], int i) {
    return operand(F::lds16(base[0] + (uint32_t)(i * 16 * kF8Group)), F::lds16(base[1] + (uint32_t)(i * 16 * kF8Group)));
  };
  auto mfma = [&](int i, int j) { acc[i][j] = mfma_block<0>(fw[i], fx[j], acc[i][j], sw, sx[j]); };
  {
    const uint32_t w0[2] = {wb + lane_off[0], wb + lane_off[1]}, x0[2] = {xb + lane_off[0], xb + lane_off[1]};
#pragma unroll
    for (int j = 0; j < RJ; ++j) {
      fx[j] = read(x0, j);
      sx[j] = f.x_scale(0, j);
    }
#pragma unroll
    for (int i = 0; i < FH; ++i) fw[i] = read(w0, i);
  }
  sw = f.w_scale(0, 0);
  __builtin_amdgcn_s_waitcnt(0xF | (3 << 14) | (0x7 << 4));   // lgkmcnt 0: else the loop waits for its last reads at its start
  for (int tile = 0; tile < f.tiles; ++tile) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4_t{};
    for (int b = 0; b < f.nb; ++b) {
      Place next = cur;
      f.advance(next);   // (what is read behind the last block is never used)
      // one base register per operand and half of a block (the empty asm keeps the sums from being re-associated into one
      // register per read)
      uint32_t wc[2], wx[2], xx[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        wc[h] = wb + cur.stage * STAGE + lane_off[h];
        wx[h] = wb + next.stage * STAGE + lane_off[h];
        xx[h] = xb + next.stage * STAGE + lane_off[h];
        asm volatile("" : "+v"(wc[h]), "+v"(wx[h]), "+v"(xx[h]));
      }
#pragma unroll
      for (int m = 0; m < HM; ++m) {
        mfma(m % FH, m / FH);
#pragma unroll
        for (int i = 0; i < FH; ++i)
          if (m == i * (HM > 2 ? HM - 2 : 0) / FH) fw[FH + i] = read(wc, FH + i);
#pragma unroll
        for (int d = D0; d < ND; ++d)
          if (m == min(1 + (d - D0) * 2, HM - 1)) f.dma(late, d);
        __builtin_amdgcn_sched_barrier(0);
      }
      int swn = 0;
#pragma unroll
      for (int m = 0; m < HM; ++m) {
        mfma(FH + m % FH, m / FH);
        if (m == P0 - 1) {
          __builtin_amdgcn_sched_barrier(0);
          enter();
          swn = f.w_scale(next.tile, next.b);
        }
#pragma unroll
        for (int i = 0; i < FH; ++i)
          if (m == min(P0 + i * (HM - P0) / FH, HM - 1)) fw[i] = read(wx, i);
#pragma unroll
        for (int j = 0; j < RJ; ++j)
          if (m == min(max((j + 1) * FH - 1, P0), HM - 1)) {
            fx[j] = read(xx, j);
            sx[j] = f.x_scale(next.b, j);
          }
#pragma unroll
        for (int d = 0; d < D0; ++d)
          if (m == min(P0 + d * (HM - P0) / D0, HM - 1)) f.dma(fill, d);
        __builtin_amdgcn_sched_barrier(0);
      }
      sw = swn;
      cur = next;
      late = fill;
      f.advance(fill);
    }
    const int nw = f.n0 + tile * BN + f.wn * (BN / WN);
    if (a.run == 1) __syncthreads();   // (all waves have read the stages)
    if (nw < a.N) put_tile<true>(a, f.yrow, nw, acc, f.out, f.lane);
  }
}

// Tiles of which two workgroups share a compute unit and fill each other's waits: a block is read, the next one's transfers
// go out, the block's matrix instructions run.  2048 x 4096 x 4096 43 us (1.6 PFLOP/s), 46 by 128 x 128 tiles read ahead, 59 by
// 256 x 256.
template <int BN, int BM, int WN, int WM, int NST, bool EXPERTS>
__global__ __launch_bounds__(WN * WM * 64, 1) void f8_pair_kernel(F8GemmK a) {
  typedef Feed<BN, BM, WN, WM, NST, EXPERTS> F;
  constexpr int FI = F::FI, RJ = F::RJ, ND = F::ND, STAGE = F::STAGE;
  static_assert(NST > 1 && NST * ND < 64, "transfers in flight");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  F f(a, threadIdx.x);
  Place fill;
  if (!f.start(smem, &fill)) return;
  int stage = 0;   // of the next block that is read
#pragma unroll
  for (int b = 0; b < NST; ++b) {
#pragma unroll
    for (int d = 0; d < ND; ++d) f.dma(fill, d);
    f.advance(fill);
  }
  uint32_t lane_off[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) lane_off[h] = (uint32_t)(f.lr * kF8Group + (chunk_swz(4 * h + f.g, f.lr) << 4));
  f32x4_t acc[FI][RJ];
  i32x8_t fw[FI], fx[RJ];
  int sw, sx[RJ];
  auto read = [&](uint32_t base) { return operand(F::lds16(base + lane_off[0]), F::lds16(base + lane_off[1])); };
  const uint32_t wb = f.lds0 + (uint32_t)(f.wn * FI * 16 * kF8Group), xb = f.lds0 + (uint32_t)((BN + f.wm * RJ * 16) * kF8Group);
  bool first = true;
  for (int tile = 0; tile < f.tiles; ++tile) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4_t{};
    for (int b = 0; b < f.nb; ++b) {
      // the block has landed: all transfers but those of the NST - 2 (at first NST - 1) blocks behind it, and all waves have
      // read the block before, whose stage is refilled
      if (first) SX_WAIT_VM((NST - 1) * ND & 63);
      else SX_WAIT_VM((NST - 2) * ND & 63);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __syncthreads();
      const uint32_t at = (uint32_t)(stage * STAGE);
      sw = f.w_scale(tile, b);
#pragma unroll
      for (int j = 0; j < RJ; ++j) sx[j] = f.x_scale(b, j);
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        fw[i] = read(wb + at + (uint32_t)(i * 16 * kF8Group));
        if (i == 0)
#pragma unroll
          for (int j = 0; j < RJ; ++j) fx[j] = read(xb + at + (uint32_t)(j * 16 * kF8Group));
      }
      stage = stage + 1 == NST ? 0 : stage + 1;
      if (!first) {
#pragma unroll
        for (int d = 0; d < ND; ++d) f.dma(fill, d);
        f.advance(fill);
      }
      first = false;
#pragma unroll
      for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < RJ; ++j) acc[i][j] = mfma_block<0>(fw[i], fx[j], acc[i][j], sw, sx[j]);
    }
    const int nw = f.n0 + tile * BN + f.wn * (BN / WN);
    if (a.run == 1) __syncthreads();   // (all waves have read the stages)
    if (nw < a.N) put_tile<false>(a, f.yrow, nw, acc, f.out, f.lane);
  }
}

// Small tiles: a wave's few matrix instructions a block do not cover the way of its operands from LDS, so those of the next
// block are read, into a second set of registers, before the block's matrix instructions and transfers.  One tile a
// workgroup.  The bound is LDS, which takes a transfer's kilobyte in 21 cycles and reads at 128 bytes a cycle: of a block's
// 420 cycles in 64 x 32 tiles 252 and 192 (96 rows x 4096 x 14336: 26 us; without the reads 21, without the transfers 15).
// More stages hide more of memory's latency, fewer leave room for a second workgroup (that product of weights from memory,
// with 4, 6 and 10 stages: 32.7, 29.4, 30.1 us; in 64 x 64 tiles 35 with 4 or 8).
template <int BN, int BM, int WN, int WM, int NST, bool EXPERTS>
__global__ __launch_bounds__(WN * WM * 64, 1) void f8_narrow_kernel(F8GemmK a) {
  typedef Feed<BN, BM, WN, WM, NST, EXPERTS> F;
  constexpr int FI = F::FI, RJ = F::RJ, ND = F::ND, STAGE = F::STAGE;
  static_assert(NST > 2 && NST * ND < 64, "transfers in flight");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  F f(a, threadIdx.x);
  Place fill;
  i32x4_t pre[RJ][put_loads<FI>()] = {};
  if (!f.start(smem, &fill, pre)) return;
#pragma unroll
  for (int b = 0; b < NST; ++b) {
#pragma unroll
    for (int d = 0; d < ND; ++d) f.dma(fill, d);
    f.advance(fill);
  }
  uint32_t lane_off[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) lane_off[h] = (uint32_t)(f.lr * kF8Group + (chunk_swz(4 * h + f.g, f.lr) << 4));
  f32x4_t acc[FI][RJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < RJ; ++j) acc[i][j] = f32x4_t{};
  i32x8_t fw[2][FI], fx[2][RJ];
  int sw, sx[RJ], swn = 0, sxn[RJ] = {};
  const uint32_t wb = f.lds0 + (uint32_t)(f.wn * FI * 16 * kF8Group), xb = f.lds0 + (uint32_t)((BN + f.wm * RJ * 16) * kF8Group);
  uint32_t at = 0;   // the stage of the next block that is read
  auto read_at = [&](uint32_t base) { return operand(F::lds16(base + lane_off[0]), F::lds16(base + lane_off[1])); };
  auto read = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FI; ++i) fw[s][i] = read_at(wb + at + (uint32_t)(i * 16 * kF8Group));
#pragma unroll
    for (int j = 0; j < RJ; ++j) fx[s][j] = read_at(xb + at + (uint32_t)(j * 16 * kF8Group));
    at = at + STAGE == NST * STAGE ? 0 : at + STAGE;
  };
  SX_WAIT_VM((NST - 1) * ND & 63);
  __syncthreads();
  read(0);
  sw = F::lds4(f.ws_at);
#pragma unroll
  for (int j = 0; j < RJ; ++j) sx[j] = F::lds4(f.xs_at + j * 64);
  auto step = [&](auto c, int b) __attribute__((always_inline)) {
    constexpr int S = decltype(c)::value;
    if (b + S >= f.nb) return;
    __builtin_amdgcn_s_waitcnt(0xF | (3 << 14) | (0x7 << 4));   // lgkmcnt 0: this block's operands
    SX_WAIT_VM((NST - 2) * ND & 63);                            // the next block has landed
    __syncthreads();
    read((S + 1) % 2);
    if (S == 3) {
      const int q = min(b + 4, f.nb - 1) & ~3;
      swn = F::lds4(f.ws_at + q);
#pragma unroll
      for (int j = 0; j < RJ; ++j) sxn[j] = F::lds4(f.xs_at + q * BM + j * 64);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = 0; m < max(FI * RJ, ND); ++m) {
      if (m < ND) f.dma(fill, m);
      if (m < FI * RJ) acc[m % FI][m / FI] = mfma_block<S>(fw[S % 2][m % FI], fx[S % 2][m / FI], acc[m % FI][m / FI], sw, sx[m / FI]);
    }
    f.advance(fill);
    if (S == 3) {
      sw = swn;
#pragma unroll
      for (int j = 0; j < RJ; ++j) sx[j] = sxn[j];
    }
  };
  for (int b = 0; b < f.nb; b += 4)
    [&]<int... S>(std::integer_sequence<int, S...>) { (step(std::integral_constant<int, S>{}, b), ...); }(std::make_integer_sequence<int, 4>{});
  const int nw = f.n0 + f.wn * (BN / WN);
  __builtin_amdgcn_s_waitcnt(0xF | (3 << 14) | (0x7 << 4));
  __syncthreads();   // (all waves have read the stages)
  if (nw < a.N) put_tile<false, true>(a, f.yrow, nw, acc, pre, f.out, f.lane);
}

// Row tiles of BM rows that the launch may have to take.
int64_t count_tiles(const F8GemmK& a, int bm) {
  if (!a.offsets) return (int64_t)a.r.n_req * (((int64_t)a.r.max_rows + bm - 1) / bm);
  return a.n_places / bm + (int64_t)(a.n_experts < a.n_places ? a.n_experts : a.n_places);
}

template <int FI, int RJ, int D, bool EXPERTS>
hipError_t launch_stream(F8GemmK& a, hipStream_t s) {
  a.m_tiles = (int)(((int64_t)a.r.max_rows + 16 * RJ - 1) / (16 * RJ));
  const int64_t blocks = count_tiles(a, 16 * RJ) * (a.N / (16 * FI));
  hipLaunchKernelGGL((f8_stream_kernel<FI, RJ, D, EXPERTS>), dim3((unsigned)blocks), dim3(64), 0, s, a);
  return hipGetLastError();
}

// Grid and LDS of a tiled launch, in runs of up to `most` tiles: as long as the workgroups of whole rounds then take no
// more tiles each than in shorter ones.  A run fetches its next tile while it computes and stores the last: 6712 x 28672 x
// 4096 in 256 x 256 tiles 635 us by runs of 4, 642 of 2, 660 singly; 8192 tokens x 8 of 128 experts, 768 -> 2048 202, 207 and
// 231, 2048 -> 2 x 768, with 16 blocks a tile, 304 to 323 whatever the run; of 8 no faster than of 4.
constexpr int kRun = 4;
template <int BN, int BM, int WN, int WM, int NST, typename K>
hipError_t launch_tiled(F8GemmK& a, int n_cu, int most, hipStream_t s, K plain, K experts) {
  const int64_t m_tiles = count_tiles(a, BM), n_tiles = (a.N + BN - 1) / BN;
  a.m_tiles = a.offsets ? (int)m_tiles : (int)(((int64_t)a.r.max_rows + BM - 1) / BM);
  constexpr int kOut = WN * WM * epilogue_lds<BN / WN / 16>();
  int lds = 0;
  int64_t least = INT64_MAX;
  for (int run = 1; run <= most; run *= 2) {
    const int need = tile_fixed(BN, BM, NST, a.ld, run) + (run > 1 ? kOut : 0);
    if (need > kLdsBytes) break;
    const int64_t slots = (int64_t)n_cu * (kLdsBytes / need), runs = m_tiles * ((n_tiles + run - 1) / run);
    const int64_t time = (runs + slots - 1) / slots * run;
    if (time <= least) {
      least = time;
      a.run = run;
      lds = need;
    }
  }
  if (lds == 0) return hipErrorInvalidConfiguration;
  const int64_t blocks = (m_tiles * ((n_tiles + a.run - 1) / a.run) + kXcds - 1) / kXcds * kXcds;
  hipLaunchKernelGGL(a.offsets ? experts : plain, dim3((unsigned)blocks), dim3(WN * WM * 64), lds, s, a);
  return hipGetLastError();
}
template <int BN, int BM, int WN, int WM, int NST>
hipError_t launch_tile(F8GemmK& a, int n_cu, hipStream_t s) {
  return launch_tiled<BN, BM, WN, WM, NST>(a, n_cu, kRun, s, f8_tile_kernel<BN, BM, WN, WM, NST, false>,
                                           f8_tile_kernel<BN, BM, WN, WM, NST, true>);
}
template <int BN, int BM, int WN, int WM, int NST>
hipError_t launch_pair(F8GemmK& a, int n_cu, hipStream_t s) {
  return launch_tiled<BN, BM, WN, WM, NST>(a, n_cu, kRun, s, f8_pair_kernel<BN, BM, WN, WM, NST, false>,
                                           f8_pair_kernel<BN, BM, WN, WM, NST, true>);
}
// GROUPED: for rows grouped by expert too.
template <int BN, int BM, int WN, int WM, int NST, bool GROUPED>
hipError_t launch_narrow(F8GemmK& a, int n_cu, hipStream_t s) {
  if (!GROUPED && a.offsets) return hipErrorInvalidConfiguration;
  return launch_tiled<BN, BM, WN, WM, NST>(a, n_cu, 1, s, f8_narrow_kernel<BN, BM, WN, WM, NST, false>,
                                           f8_narrow_kernel<BN, BM, WN, WM, NST, GROUPED>);
}

// What a launch of a shape takes, fitted to 105 products of 1 to 6712 rows by seven weights of 768 to 14336 x 1024 to 28672,
// weights from memory: `first` us and `block` us a block of k for a first round of workgroups, occ on each compute unit,
// `more` and `more_block` for each further one.
struct Shape {
  int bn, bm, nst, threads, occ;
  double first, block, more, more_block;
};
enum { kStream, k32x32, k64x32, k64x64, k128x64, k128x128, k128x128x2, k256x256, kShapes };
constexpr Shape kShape[kShapes] = {
    {16, 16, 0, 64, 1, 2.99, 0.134, 0.01, 0.115},    {32, 32, 6, 256, 1, 3.68, 0.193, 0.84, 0.093},
    {64, 32, 6, 256, 1, 3.71, 0.220, 1.26, 0.148},   {64, 64, 4, 256, 1, 3.62, 0.294, 1.45, 0.200},
    {128, 64, 3, 512, 1, 3.19, 0.474, 2.09, 0.310},  {128, 128, 4, 512, 1, 4.42, 0.554, 4.38, 0.591},
    {128, 128, 2, 512, 2, 3.00, 1.040, 9.23, 0.973}, {256, 256, 2, 256, 1, 7.90, 1.414, 10.69, 1.437}};
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 4096;   // of a launch (and room for the grid's rounding)
constexpr int kStreamExperts = 32;   // tile side of the streaming kernel for grouped rows (of listed ones: 16)

// The shape of least time; for those 105 products within 4% of the fastest (0.1% in the mean).  Some of them in us, weights
// from memory, the shape taken and its neighbours in the table: K = 4096, 1 row x 4096 features 8.0 (10.0), 1 x 6144 9.6 (10.1),
// 17 x 6144 10.4 (13.9, 11.1), 64 x 6144 12.0 (14.0, 14.1), 200 x 4096 13.2 (16.5, 18.1), 394 x 4096 18.4 (19.9, 22.2), 1000 x 4096
// 24.4 (28.7, 37.0), 2048 x 4096 42 (46, 59), 6712 x 28672 635 (845).  The costs hold no bound by the weights' bytes: of few rows
// by many features they give less than memory takes (1 x 28672 x 4096, 117 MB: 16.8 us, where four shapes take 27.4 to 28.5), but
// memory makes the shapes alike there.
// Grouped rows: few for each expert, by the streaming kernel, since the weights' way from memory is the bound (64 tokens x 8
// of 128 experts, 2048 -> 2 x 768: 68 us, 71 of 128 x 64 tiles; 256 x 8: 98, 87); else by the same costs and as many tiles as
// rows spread over the experts make, each expert's last one half full (2048 -> 2 x 768: 512 x 8 of 128 98 us of 128 x 64, 116 of
// 128 x 128; 2048 x 2 of 8 24 of 128 x 128 by twos, 30 of 128 x 64, 35 of 256 x 256; 8192 x 8 of 128 304 to 320 of 256 x 256, 356
// of 128 x 128; of 26 products within 7% of the fastest but for five, which are 9 to 20% off).
int best_shape(const F8GemmK& a, int n_cu) {
  const bool ex = a.offsets;
  if (ex && a.n_places <= 12 * (int64_t)a.n_experts && count_tiles(a, kStreamExperts) * (a.N / kStreamExperts) * 64 < kMaxThreads)
    return kStream;
  int best = -1;
  double least = 1e300;
  const double nb = a.K / kF8Group;
  for (int i = ex ? k128x64 : kStream; i < kShapes; ++i) {
    const Shape& h = kShape[i];
    const int64_t n_tiles = (a.N + h.bn - 1) / h.bn, most = count_tiles(a, h.bm) * n_tiles;
    if ((h.nst && (a.ld > kLdsBytes / h.bm || tile_fixed(h.bn, h.bm, h.nst, a.ld, 1) > kLdsBytes)) || most * h.threads >= kMaxThreads)
      continue;
    double tiles = (double)most;
    if (ex) {
      const double full = (double)a.n_places / a.n_experts / h.bm;
      tiles = a.n_experts * (full > 0.5 ? full + 0.5 : 1) * (double)n_tiles + n_cu / 8;
    }
    const double rounds = ceil(tiles / ((double)n_cu * h.occ));
    // (a streaming wave's loads touch 16 lines of w and one of x for each of up to 16 rows)
    const double lines = i == kStream && a.r.max_rows < 16 ? (16 + a.r.max_rows) / 32.0 : 1.0;
    const double t = h.first + nb * h.block + (rounds - 1) * (h.more + nb * h.more_block * lines);
    if (t < least) {
      least = t;
      best = i;
    }
  }
  return best;
}

}  // namespace

hipError_t launch_gemm_f8(F8GemmK& a, int n_cu, hipStream_t s) {
  switch (best_shape(a, n_cu)) {
    case kStream:
      if (a.offsets) return launch_stream<kStreamExperts / 16, kStreamExperts / 16, 4, true>(a, s);
      // Blocks ahead: 16 of them leave room for one wave a SIMD, which then has more on its way (1 row x 4096 x 14336 17.1 us,
      // 18.3 with 12, 20.3 with 8); where there are more waves, or few blocks, 12 (1 x 19200 x 4096 21.4, 24.8 with 16).
      if (a.K >= 16 * kF8Group && count_tiles(a, 16) * (a.N / 16) <= 4 * (int64_t)n_cu) return launch_stream<1, 1, 16, false>(a, s);
      return launch_stream<1, 1, 12, false>(a, s);
    case k32x32: return launch_narrow<32, 32, 2, 2, 6, false>(a, n_cu, s);
    case k64x32: return launch_narrow<64, 32, 2, 2, 6, false>(a, n_cu, s);
    case k64x64: return launch_narrow<64, 64, 2, 2, 4, false>(a, n_cu, s);
    case k128x64: return launch_narrow<128, 64, 4, 2, 3, true>(a, n_cu, s);
    case k128x128: return launch_narrow<128, 128, 4, 2, 4, true>(a, n_cu, s);
    case k128x128x2: return launch_pair<128, 128, 4, 2, 2>(a, n_cu, s);
    case k256x256: return launch_tile<256, 256, 2, 2, 2>(a, n_cu, s);
    default: return hipErrorInvalidConfiguration;   // (more workgroups than a launch has)
  }
}

}  // namespace sx
