// Routing of a mixture of experts (include/sx_f8.h): the top experts of every row, their weights, and the rows' places
// grouped by expert.
#include "sx_f8_device.h"

namespace sx {
namespace {

constexpr int kRouteThreads = 1024;

// Bits of a float in the order of its value; a NaN counts as -inf, -0 as +0.
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t u = __float_as_uint(v != v ? -INFINITY : v + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false); }

// A logit's key: its order above the expert's, the lower expert larger, so that a row's keys differ and the largest says
// whose it is; 0 for what is no candidate (any more).  Of bfloat16 logits 16 + 16 bits; of float32 ones 32 + 30 bits in a
// positive float64 below 2, whose order is that of its bits and whose maximum is one instruction.
struct Key16 {
  typedef uint32_t T;
  typedef uint16_t Logit;
  static __device__ __forceinline__ T make(Logit x, int e) {
    return (order_bits(__uint_as_float((uint32_t)x << 16)) & 0xffff0000u) | (uint32_t)(0xffff - e);
  }
  static __device__ __forceinline__ T none() { return 0; }
  static __device__ __forceinline__ T larger(T a, T b) { return max(a, b); }
  static __device__ __forceinline__ T row_max(T v) { return row16_max(v); }
  static __device__ __forceinline__ T across(T v, int m) { return (T)__shfl_xor((int)v, m, 64); }
  static __device__ __forceinline__ int expert(T v) { return 0xffff - (int)(v & 0xffff); }
  static __device__ __forceinline__ float value(T v) { return order_value(v & 0x80000000u ? v & 0xffff0000u : v | 0xffffu); }
};
struct Key32 {
  typedef double T;
  static __device__ __forceinline__ T of(uint32_t hi, uint32_t lo) { return __hiloint2double((int)hi, (int)lo); }
  typedef float Logit;
  static __device__ __forceinline__ T make(Logit x, int e) {
    const uint32_t k = order_bits(x);
    return of(k >> 2, k << 30 | (uint32_t)(0x3fffffff - e));
  }
  static __device__ __forceinline__ T none() { return 0.0; }
  // (no key is a NaN or a subnormal number: nothing to make canonical, as fmax would first)
  static __device__ __forceinline__ T larger(T a, T b) {
    T m;
    asm("v_max_f64 %0, %1, %2" : "=v"(m) : "v"(a), "v"(b));
    return m;
  }
  template <int CTRL>
  static __device__ __forceinline__ T step(T v) {
    return larger(v, of(dpp<CTRL>((uint32_t)__double2hiint(v)), dpp<CTRL>((uint32_t)__double2loint(v))));
  }
  static __device__ __forceinline__ T row_max(T v) { return step<0x121>(step<0x122>(step<0x124>(step<0x128>(v)))); }
  static __device__ __forceinline__ T across(T v, int m) { return __shfl_xor(v, m, 64); }
  static __device__ __forceinline__ int expert(T v) { return 0x3fffffff - (__double2loint(v) & 0x3fffffff); }
  static __device__ __forceinline__ float value(T v) {
    return order_value((uint32_t)__double2hiint(v) << 2 | (uint32_t)__double2loint(v) >> 30);
  }
};

__device__ __forceinline__ float row16_sum(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, false));
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, false));
}

// exp(v - m), 1 for v == m also where both are infinite
__device__ __forceinline__ float share(float v, float m) { return v == m ? 1.0f : expf(v - m); }

// ---------------------------------------------------------------------------------------------
// Top experts.  LPR lanes share a row, lane l of them the NV logits from l NV on.  A round finds a row's largest remaining
// key in every one of its lanes and takes it out; lane j keeps the j-th.  Rows n0 .. n0 + 63 of request r, found ids to
// LDS too.
//
// Grouping.  A workgroup counts its rows' experts (LDS atomics on whole numbers, whose sums have no order).  Once all
// counts are there, a second pass places the rows, 64 at a time: no row takes an expert twice, so 64 bits an expert say
// which rows take it, and the number of bits below a row's own is its rank.  With one workgroup both passes are one
// launch.
//
// Bound by latency: 64 rows x 128 experts of float32 6.5 us, of which top_k rounds of a maximum over 16 lanes are most;
// 32767 rows of bfloat16 8.2 + 7.8 us (11.5 MB), 256 workgroups, each of which sums all workgroups' counts.  64 rows a
// workgroup where 256 of them are enough: 4096 rows x 256 of float32 14 us, 33 with 256 rows a workgroup.
// ---------------------------------------------------------------------------------------------
struct RouteLds {
  int base[kMoeMaxExperts];              // counts, later the next place of every expert
  unsigned long long rows[kMoeMaxExperts];
  int sums[16];
  uint16_t ids[64][kMoeMaxTop];
};

template <int NV, int LPR, typename Key>
__device__ __forceinline__ void top_of_rows(const MoeRouteK& a, int r, int n0, int count, RouteLds& l) {
  constexpr int RPP = kRouteThreads / LPR;   // rows of a pass of the workgroup
  const int lane = threadIdx.x & 63, sub = lane % LPR, in_wave = lane / LPR;
  const int E = a.n_experts;
  typedef typename Key::T T;
  auto row_sum = [&](float s) {
    s = row16_sum(s);
    if constexpr (LPR == 64) {
      s += __shfl_xor(s, 16, 64);
      s += __shfl_xor(s, 32, 64);
    }
    return s;
  };
  for (int p = 0; p < 64 / RPP; ++p) {
    const int i = p * RPP + threadIdx.x / LPR, n = n0 + i;
    if (n - in_wave >= count) break;   // (no row of the wave is left; its lanes run together)
    const bool live = n < count;
    const int64_t slot = f8_slot(a.r, r, live ? n : n - in_wave);
    const int e0 = sub * NV;
    T key[NV];
    const typename Key::Logit* x = (const typename Key::Logit*)a.logits + slot * E + e0;
    if (E % NV == 0) {   // a lane's logits are all there, in one piece, or none is
      struct __attribute__((aligned(sizeof(typename Key::Logit) * NV < 16 ? sizeof(typename Key::Logit) * NV : 16))) Piece {
        typename Key::Logit x[NV];
      } piece{};
      if (e0 < E) piece = *(const Piece*)x;
#pragma unroll
      for (int v = 0; v < NV; ++v) key[v] = e0 < E ? Key::make(piece.x[v], e0 + v) : Key::none();
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) key[v] = e0 + v < E ? Key::make(x[v], e0 + v) : Key::none();
    }
    T mine = Key::none();
    float top = 0, all = 0;
    for (int j = 0; j < a.top_k; ++j) {
      T m = key[0];
#pragma unroll
      for (int v = 1; v < NV; ++v) m = Key::larger(m, key[v]);
      m = Key::row_max(m);
      if constexpr (LPR == 64) {
        m = Key::larger(m, Key::across(m, 16));
        m = Key::larger(m, Key::across(m, 32));
      }
      if (j == 0) {
        top = Key::value(m);
        if (!a.renormalise) {
#pragma unroll
          for (int v = 0; v < NV; ++v) all += key[v] != Key::none() ? share(Key::value(key[v]), top) : 0.0f;
          all = row_sum(all);
        }
      }
      if (sub == j) mine = m;
#pragma unroll
      for (int v = 0; v < NV; ++v) key[v] = key[v] == m ? Key::none() : key[v];
    }
    const float w = sub < a.top_k ? share(Key::value(mine), top) : 0.0f;
    if (a.renormalise) all = row_sum(w);
    if (sub < a.top_k && live) {
      const int id = Key::expert(mine);
      l.ids[i][sub] = (uint16_t)id;
      a.ids[slot * a.top_k + sub] = id;
      a.weights[slot * a.top_k + sub] = top == -INFINITY ? 0.0f : w / all;
      atomicAdd(&l.base[id], 1);
    }
  }
}

// Exclusive prefix sums of v over the workgroup's threads.
__device__ __forceinline__ int block_prefix(int v, int* sums, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kRouteThreads / 64; ++i) {
    const int s = sums[i];
    before += i < wave ? s : 0;
    all += s;
  }
  *total = all;
  return before + x - v;
}

// Places of rows n0 .. n0 + 63 of request r, whose ids are in LDS; l.base holds the experts' next places.
__device__ __forceinline__ void place_rows(const MoeRouteK& a, int r, int n0, int count, RouteLds& l) {
  const int k = a.top_k, rows = min(64, count - n0);
  __syncthreads();
  for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) l.rows[e] = 0;
  __syncthreads();
  const int i = threadIdx.x / kMoeMaxTop, j = threadIdx.x % kMoeMaxTop;   // 64 rows x 16
  const bool live = i < rows && j < k;
  const int id = live ? l.ids[i][j] : 0;
  if (live) atomicOr(&l.rows[id], 1ull << i);
  __syncthreads();
  if (live) {
    const unsigned long long bits = l.rows[id];
    const int at = l.base[id] + __popcll(bits & ((1ull << i) - 1));
    a.order[at] = (int)(f8_slot(a.r, r, n0 + i) * k + j);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) l.base[e] += __popcll(l.rows[e]);
}

// The workgroup's rows, 64 at a time: f(request, first row, rows of the request).
template <typename F>
__device__ __forceinline__ void for_rows(const MoeRouteK& a, F f) {
  const int b = blockIdx.x;
  if (a.per_req > 1) {
    const int r = b / a.per_req, n0 = (b - r * a.per_req) * a.rows_per_block;
    const int count = f8_count(a.r, r), end = min(count, n0 + a.rows_per_block);
    for (int n = n0; n < end; n += 64) f(r, n, count);
  } else {
    const int r0 = b * a.reqs_per_block, r1 = min(r0 + a.reqs_per_block, a.r.n_req);
    for (int r = r0; r < r1; ++r) {
      const int count = f8_count(a.r, r);
      for (int n = 0; n < count; n += 64) f(r, n, count);
    }
  }
}

template <int NV, int LPR, typename Key, bool ONE>
__global__ __launch_bounds__(kRouteThreads) void route_top_kernel(MoeRouteK a) {
  __shared__ RouteLds l;
  for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) l.base[e] = 0;
  __syncthreads();
  int last_r = 0, last_n = 0, last_count = 0, chunks = 0;
  for_rows(a, [&](int r, int n0, int count) {
    top_of_rows<NV, LPR, Key>(a, r, n0, count, l);
    last_r = r;
    last_n = n0;
    last_count = count;
    ++chunks;
  });
  __syncthreads();
  if constexpr (ONE) {   // (at most 64 rows: their ids are still in LDS)
    int total;
    const int c = (int)threadIdx.x < a.n_experts ? l.base[threadIdx.x] : 0;
    const int at = block_prefix(c, l.sums, &total);
    if ((int)threadIdx.x < a.n_experts) {
      l.base[threadIdx.x] = at;
      a.offsets[threadIdx.x] = at;
    }
    if (threadIdx.x == 0) a.offsets[a.n_experts] = total;
    if (chunks > 0) place_rows(a, last_r, last_n, last_count, l);
  } else {
    for (int e = threadIdx.x; e < a.n_experts; e += kRouteThreads) a.counts[(int64_t)blockIdx.x * a.n_experts + e] = l.base[e];
  }
}

__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(MoeRouteK a) {
  __shared__ RouteLds l;
  __shared__ int mine[kMoeMaxExperts], all[kMoeMaxExperts];
  const int E = a.n_experts;
  for (int e = threadIdx.x; e < E; e += kRouteThreads) mine[e] = all[e] = 0;
  __syncthreads();
  // sums over the workgroups before this one, and over all
  const int per = kRouteThreads / E > 1 ? kRouteThreads / E : 1;   // threads an expert
  if ((int)threadIdx.x < per * E) {
    const int e = threadIdx.x % E;
    int before = 0, sum = 0;
    for (int b0 = threadIdx.x / E; b0 < a.blocks; b0 += 8 * per) {
      int c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = b0 + i * per < a.blocks ? a.counts[(int64_t)(b0 + i * per) * E + e] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        before += b0 + i * per < (int)blockIdx.x ? c[i] : 0;
        sum += c[i];
      }
    }
    atomicAdd(&mine[e], before);
    atomicAdd(&all[e], sum);
  }
  __syncthreads();
  int total;
  const int at = block_prefix((int)threadIdx.x < E ? all[threadIdx.x] : 0, l.sums, &total);
  if ((int)threadIdx.x < E) {
    l.base[threadIdx.x] = at + mine[threadIdx.x];
    if (blockIdx.x == 0) a.offsets[threadIdx.x] = at;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[E] = total;
  for_rows(a, [&](int r, int n0, int count) {
    const int i = threadIdx.x / kMoeMaxTop, j = threadIdx.x % kMoeMaxTop;
    __syncthreads();
    if (n0 + i < count && j < a.top_k) l.ids[i][j] = (uint16_t)a.ids[f8_slot(a.r, r, n0 + i) * a.top_k + j];
    place_rows(a, r, n0, count, l);
  });
}

template <int NV, int LPR>
hipError_t launch_top(const MoeRouteK& a, bool f32, hipStream_t s) {
  const bool one = a.blocks == 1 && a.r.n_req == 1 && a.r.max_rows <= 64;
  const dim3 grid((unsigned)a.blocks), block(kRouteThreads);
  if (one) {
    if (f32) hipLaunchKernelGGL((route_top_kernel<NV, LPR, Key32, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((route_top_kernel<NV, LPR, Key16, true>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  if (f32) hipLaunchKernelGGL((route_top_kernel<NV, LPR, Key32, false>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((route_top_kernel<NV, LPR, Key16, false>), grid, block, 0, s, a);
  hipLaunchKernelGGL(route_place_kernel, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_moe_route(const MoeRouteK& a, bool f32, hipStream_t s) {
  const int E = a.n_experts;
  if (E <= 16) return launch_top<1, 16>(a, f32, s);
  if (E <= 64) return launch_top<4, 16>(a, f32, s);
  if (E <= 128) return launch_top<8, 16>(a, f32, s);
  if (E <= 256) return launch_top<16, 16>(a, f32, s);
  if (E <= 512) return launch_top<8, 64>(a, f32, s);
  return launch_top<16, 64>(a, f32, s);
}

}  // namespace sx
