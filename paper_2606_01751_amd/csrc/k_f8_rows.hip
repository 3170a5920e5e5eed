// Row kernels of the 8-bit layer body (include/sx_f8.h):
//
//   add_rmsnorm_f8_kernel  s = x + delta, y = s / sqrt(mean(s^2) + eps) * gamma, y in 8 bits (and in bfloat16)
//   silu_mul_f8_kernel     y = silu(gate) * up in 8 bits
//   f8_pack_weight_kernel  a weight's 128 x 128 blocks to 8 bits
//   moe_combine_kernel     weighted sum of a row's experts, added to the residual stream
#include "sx_f8_device.h"

namespace sx {
namespace {

// ---------------------------------------------------------------------------------------------
// TPR threads a row, the row's first NC pieces of 8 elements a thread held as they came; further pieces are read again in
// the second pass, which alone writes x_out, so that x_out may be x.  Sum of squares and products in float64, as in the
// bfloat16 layer body's norm: the float32 result is the nearest one, so a row's scales and codes do not hang on the order
// of a sum.  Bound by memory where rows are many (19997 x 3584 with addition and both outputs, 646 MB: 116 us, 5.6 TB/s), else
// by a wave's chain (48 x 4096: 4.5 us); rows of up to 1024 elements are a wave's own, without a barrier.
// ---------------------------------------------------------------------------------------------
template <int TPR, int NC>
__global__ __launch_bounds__(256) void add_rmsnorm_f8_kernel(F8NormK a) {
  constexpr int RPB = 256 / TPR, STEP = TPR * 8;
  __shared__ double part[4];
  const int lane = threadIdx.x & 63, t = threadIdx.x % TPR;
  const int n = blockIdx.x * RPB + threadIdx.x / TPR;
  const bool live = n < f8_count(a.r, blockIdx.y);
  const int64_t xr = live ? f8_row(a.r, blockIdx.y, n, a.x_tok) : -1;
  const int64_t yr = live ? f8_row(a.r, blockIdx.y, n, a.y_tok) : -1;
  if (xr < 0 || yr < 0) return;   // (whole rows: all threads that share a barrier)
  const int H = a.h;
  const uint16_t* x = a.x + xr * H;
  const uint16_t* delta = a.delta ? a.delta + f8_slot(a.r, blockIdx.y, n) * H : nullptr;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  // elements c .. c + 7 of s, as bfloat16
  auto load = [&](int c) {
    if (c >= H) return zero;
    uint4 v = *(const uint4*)(x + c);
    if (delta) {
      float f[8], d[8];
      unpack8(v, f);
      unpack8(*(const uint4*)(delta + c), d);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] += d[i];
      v = pack8(f);
    }
    return v;
  };
  uint4 s[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) s[i] = load(t * 8 + i * STEP);
  double inv = 1.0;
  if (a.gamma) {
    double ss = 0.0;
    auto add = [&](const uint4& v) {
      float f[8];
      unpack8(v, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)f[i], (double)f[i], ss);
    };
#pragma unroll
    for (int i = 0; i < NC; ++i) add(s[i]);
    for (int c = t * 8 + NC * STEP; c < H; c += STEP) add(load(c));
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
    if constexpr (TPR == 256) {
      if (lane == 0) part[threadIdx.x >> 6] = ss;
      __syncthreads();
      ss = part[0] + part[1] + part[2] + part[3];
    }
    inv = 1.0 / sqrt(ss / (double)H + (double)a.eps);
  }
  uint16_t* xo = a.x_out ? a.x_out + xr * H : nullptr;
  uint16_t* y16 = a.y16 ? a.y16 + yr * H : nullptr;
  auto put = [&](int c, const uint4& v) {
    float f[8];
    unpack8(v, f);
    if (a.gamma) {
      float g[8];
      unpack8(c < H ? *(const uint4*)(a.gamma + c) : zero, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (float)((double)f[i] * inv * (double)g[i]);
    }
    if (c < H) {
      if (xo) *(uint4*)(xo + c) = v;
      if (y16) *(uint4*)(y16 + c) = pack8(f);
    }
    if (a.y8) f8_put8(f, c, H, a.y8 + yr * H, a.ys + yr * a.ld, lane);
  };
  const int w0 = (t & ~63) * 8;   // the wave's first element of a piece
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (w0 + i * STEP < H) put(t * 8 + i * STEP, s[i]);
  for (int c0 = w0 + NC * STEP; c0 < H; c0 += STEP) put(c0 + lane * 8, load(c0 + lane * 8));
}

// ---------------------------------------------------------------------------------------------
// A wave takes NC pieces of 512 elements, 8 a lane, one after the other in the order of the rows.  Bound by memory where rows
// are many: 6712 x 14336 elements in 89 us (5.4 TB/s) with two pieces, 94 with one, 91 with four, 65536 x 768 in 53, 57 and
// 55; few rows by the chain of a wave, which two pieces lengthen: 300 x 14336 7.4 us, 6.7 with one, 17 x 14336 3.5, 3.1.
// What a piece computes counts too: with expf and a division 105 us in place of 89.
// ---------------------------------------------------------------------------------------------
constexpr int64_t kSiluTwo = 65536;   // pieces from which a wave takes two

// x / (1 + e^-x) * u.  e^-x = 2^p (1 + r ln 2) with p + r = -x / ln 2, r what the rounding of p lost; outside of +-100 e^-x
// is 0 or infinite anyway.  A quarter of the sum keeps its reciprocal, to one unit, above float32's smallest normal number.
__device__ __forceinline__ float silu_mul(float x, float u) {
  constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147182f;
  const float t = __builtin_amdgcn_fmed3f(x, -100.0f, 100.0f);
  const float p = t * -kLog2e;
  const float r = __builtin_fmaf(t, -kLog2eLow, __builtin_fmaf(t, -kLog2e, -p));
  const float e = __builtin_amdgcn_exp2f(p) * __builtin_fmaf(r, kLn2, 1.0f);
  return x * 0.25f * __builtin_amdgcn_rcpf(__builtin_fmaf(e, 0.25f, 0.25f)) * u;
}
template <int NC>
__global__ __launch_bounds__(256) void silu_mul_f8_kernel(F8SiluK a) {
  const int lane = threadIdx.x & 63;
  const unsigned per_row = (unsigned)(a.f + 511) / 512;
  const unsigned first = (blockIdx.x * 4 + (unsigned)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * NC;   // (below 2^32 / 64)
  const int count = f8_count(a.r, blockIdx.y);
  uint4 g[NC], u[NC];
  int64_t row[NC];
  int c[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const unsigned n = (first + i) / per_row;
    row[i] = (int)n < count ? f8_slot(a.r, blockIdx.y, (int)n) : -1;
    c[i] = (int)(first + i - n * per_row) * 512 + lane * 8;
    g[i] = u[i] = make_uint4(0, 0, 0, 0);
    if (row[i] >= 0 && c[i] < a.f) {
      g[i] = *(const uint4*)(a.gu + row[i] * 2 * a.f + c[i]);
      u[i] = *(const uint4*)(a.gu + row[i] * 2 * a.f + a.f + c[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    if (row[i] < 0) return;
    float x[8], y[8];
    unpack8(g[i], x);
    unpack8(u[i], y);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = silu_mul(x[e], y[e]);
    f8_put8(y, c[i], a.f, a.y8 + row[i] * a.f, a.ys + row[i] * a.ld, lane);
  }
}

// ---------------------------------------------------------------------------------------------
// One workgroup a block of 128 x 128; thread t takes pieces of 8 elements, 16 rows apart.  Run once for a weight.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void f8_pack_weight_kernel(const uint16_t* __restrict__ w, int k, uint8_t* __restrict__ codes,
                                                             uint8_t* __restrict__ scales, int ld) {
  __shared__ uint32_t part[4];
  const int kb = blockIdx.x;
  const int64_t nb = blockIdx.y;
  const int64_t at = (nb * 128 + threadIdx.x / 16) * k + (int64_t)kb * 128 + threadIdx.x % 16 * 8;
  uint4 v[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = *(const uint4*)(w + at + (int64_t)i * 16 * k);
    float f[8];
    unpack8(v[i], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7fffffffu);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  const uint32_t byte = f8_scale_byte(max(max(part[0], part[1]), max(part[2], part[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float f[8];
    unpack8(v[i], f);
    *(uint2*)(codes + at + (int64_t)i * 16 * k) = f8_codes8(f, byte);
  }
  if (threadIdx.x == 0) scales[nb * ld + kb] = (uint8_t)byte;
  const int groups = k / kF8Group;
  if (kb == groups - 1 && threadIdx.x < ld - groups) scales[nb * ld + groups + threadIdx.x] = 0;
}

// ---------------------------------------------------------------------------------------------
// Eight columns of a row a thread, the row's experts in ascending j in float32.  Bound by memory: 8192 x 2048, 8 experts, 337
// MB in 59 to 66 us (5.1 TB/s and more); 64 rows 4.5 us.  What it adds up are the products' results rounded to bfloat16, each
// off by up to 2^-8 of itself: against float64 the sums are 0.0018 (8 experts) to 0.0021 (fewer) off, 0.0017 with y in
// float32.  That would be twice the bytes on the way out of the product, which bounds it, and in here, 121 us in place of 66 for
// that many.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void moe_combine_kernel(MoeCombineK a) {
  const unsigned upr = (unsigned)a.h / 8;
  const unsigned g = blockIdx.x * 256 + threadIdx.x;   // (below 2^32)
  const unsigned n = g / upr;
  if (n >= (unsigned)f8_count(a.r, blockIdx.y)) return;
  const int c = (int)(g - n * upr) * 8;
  const int64_t slot = f8_slot(a.r, blockIdx.y, (int)n), row = f8_row(a.r, blockIdx.y, (int)n, a.out_tok);
  if (row < 0) return;
  float s[8] = {};
  if (a.res) unpack8(*(const uint4*)(a.res + row * a.h + c), s);
  const uint16_t* y = a.y + slot * a.top_k * a.h + c;
  for (int j = 0; j < a.top_k; ++j) {
    const float w = a.weights[slot * a.top_k + j];
    if (w == 0.0f) continue;
    float f[8];
    unpack8(*(const uint4*)(y + (int64_t)j * a.h), f);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = __builtin_fmaf(w, f[i], s[i]);
  }
  *(uint4*)(a.out + row * a.h + c) = pack8(s);
}

}  // namespace

hipError_t launch_add_rmsnorm_f8(const F8NormK& a, hipStream_t s) {
  const unsigned rows = (unsigned)a.r.max_rows, req = (unsigned)a.r.n_req;
  if (a.h <= 1024)
    hipLaunchKernelGGL((add_rmsnorm_f8_kernel<64, 2>), dim3((rows + 3) / 4, req), dim3(256), 0, s, a);
  else if (a.h <= 4096)
    hipLaunchKernelGGL((add_rmsnorm_f8_kernel<256, 2>), dim3(rows, req), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((add_rmsnorm_f8_kernel<256, 4>), dim3(rows, req), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_silu_mul_f8(const F8SiluK& a, hipStream_t s) {
  const int64_t pieces = (int64_t)a.r.max_rows * ((a.f + 511) / 512);
  if (pieces >= kSiluTwo)
    hipLaunchKernelGGL(silu_mul_f8_kernel<2>, dim3((unsigned)((pieces + 7) / 8), (unsigned)a.r.n_req), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(silu_mul_f8_kernel<1>, dim3((unsigned)((pieces + 3) / 4), (unsigned)a.r.n_req), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_f8_pack_weight(const uint16_t* w, int64_t n, int k, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  // (at most 65535 rows of blocks a launch)
  for (int64_t n0 = 0; n0 < n; n0 += 65535 * 128ll) {
    const int64_t nb = (n - n0 < 65535 * 128ll ? n - n0 : 65535 * 128ll) / 128;
    hipLaunchKernelGGL(f8_pack_weight_kernel, dim3((unsigned)(k / kF8Group), (unsigned)nb), dim3(256), 0, s, w + n0 * k, k,
                       codes + n0 * k, scales + n0 / 128 * f8_ld(k), f8_ld(k));
  }
  return hipGetLastError();
}

hipError_t launch_moe_combine(const MoeCombineK& a, hipStream_t s) {
  const int64_t threads = (int64_t)a.r.max_rows * (a.h / 8);
  hipLaunchKernelGGL(moe_combine_kernel, dim3((unsigned)((threads + 255) / 256), (unsigned)a.r.n_req), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace sx
