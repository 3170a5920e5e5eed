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
#include <type_traits>

#include "sx_f8_device.h"

namespace sx {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8_t operand(const uint4& a, const uint4& b) {
  return i32x8_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

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

// Four consecutive features n of row m.
template <bool EXPERTS>
__device__ __forceinline__ void put4(const F8GemmK& a, const RowTile& t, int m, int part, int n, f32x4_t v) {
  const int64_t row = y_row<EXPERTS>(a, t, m);
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

// ---------------------------------------------------------------------------------------------
// A wave takes 16 features and 16 RJ rows and reads both operands from memory into registers.
// ---------------------------------------------------------------------------------------------
template <int RJ, bool EXPERTS>
__global__ __launch_bounds__(64) void f8_stream_kernel(F8GemmK a) {
  constexpr int BM = 16 * RJ;
  const int lane = threadIdx.x, lr = lane % 16, g = lane / 16;
  const int n_nt = a.N / 16;
  const int idx = blockIdx.x / n_nt, n0 = (int)(blockIdx.x - (unsigned)idx * n_nt) * 16;
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
  f32x4_t acc[RJ];
#pragma unroll
  for (int j = 0; j < RJ; ++j) acc[j] = f32x4_t{};
  const int nb = a.K / kF8Group;
  auto step = [&](auto s, int b, int sw, const int (&sx)[RJ]) {
    const uint8_t* wb = w + b * kF8Group;
    const i32x8_t wo = operand(*(const uint4*)wb, *(const uint4*)(wb + 64));
#pragma unroll
    for (int j = 0; j < RJ; ++j) {
      const uint8_t* xb = x[j] + b * kF8Group;
      acc[j] = mfma_block<decltype(s)::value>(wo, operand(*(const uint4*)xb, *(const uint4*)(xb + 64)), acc[j], sw, sx[j]);
    }
  };
  for (int b = 0; b < nb; b += 4) {
    const int sw = *(const int*)(ws + b);
    int sx[RJ];
#pragma unroll
    for (int j = 0; j < RJ; ++j) sx[j] = *(const int*)(xs[j] + b);
    step(std::integral_constant<int, 0>{}, b, sw, sx);
    if (b + 1 < nb) step(std::integral_constant<int, 1>{}, b + 1, sw, sx);
    if (b + 2 < nb) step(std::integral_constant<int, 2>{}, b + 2, sw, sx);
    if (b + 3 < nb) step(std::integral_constant<int, 3>{}, b + 3, sw, sx);
  }
  const int part = part_of(a, n0);
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
    const int m = t.m0 + 16 * j + lr;
    if (m < t.nr) put4<EXPERTS>(a, t, m, part, n0 + 4 * g, acc[j]);
  }
}

// Row tiles of BM rows that the launch may have to take.
int64_t count_tiles(const F8GemmK& a, int bm) {
  if (!a.offsets) return (int64_t)a.r.n_req * ((a.r.max_rows + bm - 1) / bm);
  return a.n_places / bm + (int64_t)(a.n_experts < a.n_places ? a.n_experts : a.n_places);
}

template <int RJ>
hipError_t launch_stream(F8GemmK& a, hipStream_t s) {
  a.m_tiles = (a.r.max_rows + 16 * RJ - 1) / (16 * RJ);
  const int64_t blocks = count_tiles(a, 16 * RJ) * (a.N / 16);
  if (blocks >= ((int64_t)1 << 31)) return hipErrorInvalidConfiguration;
  if (a.offsets)
    hipLaunchKernelGGL((f8_stream_kernel<RJ, true>), dim3((unsigned)blocks), dim3(64), 0, s, a);
  else
    hipLaunchKernelGGL((f8_stream_kernel<RJ, false>), dim3((unsigned)blocks), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_f8(F8GemmK& a, hipStream_t s) { return launch_stream<1>(a, s); }

}  // namespace sx
