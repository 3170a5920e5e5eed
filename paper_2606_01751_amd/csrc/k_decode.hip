// What a decoding step runs before its attention (include/sx_decode.h):
//
//   append_slots_kernel   block tables and slot maps of the appended tokens
//   qk_norm_rope_kernel   per-head RMSNorm of queries and keys with the position rotation
#include "sx_kv4_device.h"

namespace sx {
namespace {

// ---------------------------------------------------------------------------------------------
// Slot maps.  With have_r = ceil(ctx_r / b) and need_r = min(ceil((ctx_r + new_r) / b), width) - have_r,
// token j of request r has index i = C_r + j in the step (C = exclusive prefix sums of new) and position
// p = ctx_r + j; its block is table[r][p / b] below have_r, else free[head + N_r + p / b - have_r] (N =
// exclusive prefix sums of need).
// One launch: every workgroup forms the two prefix sums by itself, in runs of 256 requests, and serves its
// own range of token indices from the run in LDS; workgroup 0 writes what there is one of per request, looks over the
// entries that the step takes from the free list, and only where one of them gives no slots goes over the requests
// once more to count its tokens.
// ---------------------------------------------------------------------------------------------
constexpr int kSlotRun = 256;    // requests a run, and threads
constexpr int kSlotTokens = 1;   // tokens per thread (300 requests, 131072 tokens: 6.9 us; 6.8 with 2, 7.6 with 4)

struct SlotRun {
  int64_t tok0, blk0;             // prefix sums before the run
  int tok[kSlotRun + 1];          // exclusive prefix sums inside the run
  int blk[kSlotRun + 1];
  int ctx[kSlotRun];
  int64_t wave_tok[4], wave_blk[4];
};

__device__ __forceinline__ int64_t wave_scan(int64_t v, int lane) {   // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  return v;
}

// ceil(n / b)
__device__ __forceinline__ int64_t blocks_of(uint32_t n, uint32_t b) {
  const uint32_t q = n / b;
  return (int64_t)q + (q * b != n);
}

// How many of a block's `b` slots int32 holds: none of a block that is not there.
__device__ __forceinline__ int64_t slots_of(int id, uint32_t b) {
  return id < 0 ? 0 : max(min(((int64_t)1 << 31) - (int64_t)id * b, (int64_t)b), (int64_t)0);
}

__global__ __launch_bounds__(kSlotRun) void append_slots_kernel(AppendSlotsK a, int per_wg) {
  __shared__ SlotRun run;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool per_request = blockIdx.x == 0;
  const int64_t t0 = (int64_t)(blockIdx.x - 1) * per_wg;   // this workgroup's token indices (not workgroup 0)
  const int64_t t1 = min(t0 + per_wg, (int64_t)a.max_tokens);
  const int64_t head = a.free_head ? max(a.free_head[0], 0) : 0;
  const uint32_t b = a.block;
  int64_t tok = 0, blk = 0, missing = 0;
  bool again = false;   // (workgroup 0's second time over the requests)
over_requests:
  for (int r0 = 0; r0 < a.n_req && (per_request || tok < t1); r0 += kSlotRun) {   // (uniform)
    const int r = r0 + tid;
    const int ctx = r < a.n_req ? max(a.ctx[r], 0) : 0;
    const int add = r < a.n_req ? (a.add ? max(a.add[r], 0) : 1) : 0;
    const int64_t len = (int64_t)ctx + add;   // (below 2^32)
    const int64_t have = blocks_of((uint32_t)ctx, b);
    const int64_t need = max(min(blocks_of((uint32_t)len, b), (int64_t)a.max_blocks) - have, (int64_t)0);
    int64_t st = wave_scan(add, lane), sb = wave_scan(need, lane);
    if (lane == 63) {
      run.wave_tok[wave] = st;
      run.wave_blk[wave] = sb;
    }
    __syncthreads();
    int64_t all_tok = 0, all_blk = 0;
#pragma unroll
    for (int w = 0; w < kSlotRun / 64; ++w) {
      if (w < wave) {
        st += run.wave_tok[w];
        sb += run.wave_blk[w];
      }
      all_tok += run.wave_tok[w];
      all_blk += run.wave_blk[w];
    }
    if (per_request) {
      const int64_t c = tok + st - add, f = head + blk + sb - need;   // first token index, first free entry
      const int64_t got = max(min((int64_t)a.n_free - f, need), (int64_t)0);
      const int64_t room = max(min((int64_t)a.max_tokens - c, (int64_t)add), (int64_t)0);
      // tokens from `upto` on have no slot: no block left, or no room in the table
      const int64_t upto = max(min(min(have + got, (int64_t)a.max_blocks) * b - ctx, (int64_t)add), (int64_t)0);
      if (again) {   // tokens that were counted as served, in blocks that the list does not give in full
        for (int64_t bi = have; bi < have + got && bi * b - ctx < min(upto, room); ++bi)
          missing += max(min((bi + 1) * b - ctx, min(upto, room)) - (bi * b - ctx + slots_of(a.free_blocks[f + bi - have], b)), (int64_t)0);
      } else if (r < a.n_req) {
        a.seq[r] = (int)min(len, (int64_t)INT32_MAX);
        a.cu[r] = (int)min(c, (int64_t)INT32_MAX);
        // the open block takes the tokens before `open`, as many as its entry has slots for
        const int64_t open = min(have * b - ctx, (int64_t)add);
        int64_t held = 0;
        if (open > 0 && have <= a.max_blocks)
          held = max(min(slots_of(a.table[(int64_t)r * a.max_blocks + have - 1], b) - (ctx - (have - 1) * b), open), (int64_t)0);
        missing += add - min(held, room) - max(min(upto, room) - open, (int64_t)0);
        if (c + add > a.max_tokens)   // blocks that open behind the room
          for (int64_t bi = max(have, ((int64_t)a.max_tokens - c + ctx + b - 1) / b); bi < have + need; ++bi) {
            const int64_t e = f + bi - have;
            a.table[(int64_t)r * a.max_blocks + bi] = e < a.n_free ? a.free_blocks[e] : -1;
          }
      }
    } else if (tok + all_tok > t0 && tok < t1) {   // (uniform)
      run.tok[tid] = (int)min(st - add, (int64_t)INT32_MAX);
      run.blk[tid] = (int)min(sb - need, (int64_t)INT32_MAX);
      run.ctx[tid] = ctx;
      __syncthreads();
      for (int64_t i = max(t0, tok) + tid; i < min(t1, tok + all_tok); i += kSlotRun) {
        const int x = (int)min(i - tok, (int64_t)INT32_MAX);
        int lo = 0;   // last request of the run that starts at or before token x
#pragma unroll
        for (int o = kSlotRun / 2; o >= 1; o >>= 1)
          if (run.tok[lo + o] <= x) lo += o;
        const uint32_t p = (uint32_t)run.ctx[lo] + (uint32_t)(x - run.tok[lo]);   // (below 2^32)
        const int64_t bi = p / b, hv = blocks_of((uint32_t)run.ctx[lo], b);
        const uint32_t off = p - (uint32_t)bi * b;
        int32_t* row = a.table + (int64_t)(r0 + lo) * a.max_blocks;
        int id = -1;
        if (bi < a.max_blocks) {
          if (bi < hv) {
            id = row[bi];
          } else {
            const int64_t f = head + blk + run.blk[lo] + bi - hv;
            if (f >= 0 && f < a.n_free) id = a.free_blocks[f];
            if (off == 0) row[bi] = id;
          }
        }
        const int64_t slot = (int64_t)id * b + off;
        a.pos[i] = (int)min(p, (uint32_t)INT32_MAX);
        a.slots[i] = id >= 0 && slot <= INT32_MAX ? (int)slot : -1;
      }
    }
    tok += all_tok;
    blk += all_blk;
    __syncthreads();   // the run's LDS is free again
  }
  if (per_request && !again) {
    const uint32_t most = 0x80000000u / b - 1;   // the last id all of whose slots int32 holds
    const int64_t end = min(head + blk, (int64_t)a.n_free);
    uint32_t bad = 0;
    for (int64_t e0 = head + tid; e0 - tid < end; e0 += 8 * kSlotRun) {   // (eight loads at once)
      uint32_t id[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) id[i] = a.free_blocks[min(e0 + i * kSlotRun, end - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) bad |= id[i] > most;
    }
    if (__syncthreads_or(bad)) {
      again = true;
      tok = blk = 0;
      goto over_requests;
    }
  }
  if (per_request) {
    const int64_t m = wave_scan(missing, lane);
    if (lane == 63) run.wave_tok[wave] = m;
    __syncthreads();
    if (tid == 0) {
      a.cu[a.n_req] = (int)min(tok, (int64_t)INT32_MAX);
      a.state[0] = (int)max(min(head + blk, (int64_t)a.n_free), min(head, (int64_t)INT32_MAX));
      a.state[1] = (int)min(run.wave_tok[0] + run.wave_tok[1] + run.wave_tok[2] + run.wave_tok[3], (int64_t)INT32_MAX);
    }
  } else {
    for (int64_t i = max(t0, tok) + tid; i < t1; i += kSlotRun) {
      a.pos[i] = -1;
      a.slots[i] = -1;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Q/K norm and rotation.  y = x / sqrt(mean x^2 + eps) * gamma over a head's D elements, then the pair
// (y1, y2) with frequency theta_p goes to (y1 c - y2 s, y2 c + y1 s), c, s = cos, sin(pos theta_p) formed in
// float64 once per (token, pair) and shared by the token's heads through LDS.  D / 8 lanes hold a head, 8
// elements each; with NEOX pairs a lane's partner elements sit D / 16 lanes away.
// A workgroup takes 256 / (D / 2) tokens and, of their heads, one of `parts` shares: few tokens are bound by latency
// (the first share of the rows is loaded before the angles are formed), many by HBM: 32768 rows of 28 / 4 heads of 128
// (bfloat16) 106 us, 5.1 TB/s read and written, 109 without the next head's load ahead of a head's arithmetic.
// ---------------------------------------------------------------------------------------------

// cos and sin of phi >= 0, rounded to float32.  phi = n pi/2 + r with |r| <= pi/4, pi/2 in two float64 parts (the first
// is off by 2^-54, the second makes up for n times that; good for phi below 2^52, which the host's bound of the base keeps);
// the Taylor polynomials of r up to r^13 and r^14 are off by less than 2^-45, far below half a unit of float32.
__device__ __forceinline__ void cos_sin(double phi, float* c, float* s) {
  const double n = __builtin_rint(phi * 0.63661977236758134308);
  double r = __builtin_fma(n, -1.57079632679489655800, phi);
  r = __builtin_fma(n, -6.12323399573676603587e-17, r);
  const double z = r * r;
  double ps = 1.0 / 6227020800.0, pc = -1.0 / 87178291200.0;
  ps = __builtin_fma(ps, z, -1.0 / 39916800.0);
  pc = __builtin_fma(pc, z, 1.0 / 479001600.0);
  ps = __builtin_fma(ps, z, 1.0 / 362880.0);
  pc = __builtin_fma(pc, z, -1.0 / 3628800.0);
  ps = __builtin_fma(ps, z, -1.0 / 5040.0);
  pc = __builtin_fma(pc, z, 1.0 / 40320.0);
  ps = __builtin_fma(ps, z, 1.0 / 120.0);
  pc = __builtin_fma(pc, z, -1.0 / 720.0);
  ps = __builtin_fma(ps, z, -1.0 / 6.0);
  pc = __builtin_fma(pc, z, 1.0 / 24.0);
  pc = __builtin_fma(pc, z, -0.5);
  const float fs = (float)__builtin_fma(ps * z, r, r), fc = (float)__builtin_fma(pc, z, 1.0);
  const int q = (int)__builtin_fma(-4.0, __builtin_floor(n * 0.25), n);   // quadrant
  const float a = q & 1 ? fs : fc, b = q & 1 ? fc : fs;
  *c = (q + 1) & 2 ? -a : a;
  *s = q & 2 ? -b : b;
}

template <typename T, int D, bool NEOX, bool ROWS>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNormRopeK a, int parts) {
  constexpr int TB = 256 / (D / 2);   // tokens per workgroup
  constexpr int LPH = D / 8;          // lanes per head
  constexpr int HPW = 256 / LPH;      // heads a pass of the workgroup
  __shared__ __attribute__((aligned(16))) float cs[TB][D / 2], sn[TB][D / 2];
  __shared__ int64_t rows[TB];        // token rows, -1: none
  const int part = blockIdx.x % (uint32_t)parts, n0 = blockIdx.x / (uint32_t)parts * TB;
  const int live = ROWS ? min(min(a.n_rows[blockIdx.y], a.max_rows), a.reqs[blockIdx.y].T) : a.n;   // rows of the call
  if (ROWS && n0 >= live) return;
  auto token = [&](int tb, int* pos) {   // token row of the workgroup's tb-th row, -1: none
    int64_t t = -1;
    if (n0 + tb < live) {
      if constexpr (ROWS) {
        const ReqDev rq = a.reqs[blockIdx.y];
        const int row = a.rows[rq.tok_off + n0 + tb];
        if ((uint32_t)row >= (uint32_t)rq.T) return t;
        t = (int64_t)rq.tok_off + row;
        *pos = a.tok_pos[t];
      } else {
        t = n0 + tb;
        *pos = a.pos[t];
      }
      if (*pos < 0) t = -1;
    }
    return t;
  };
  const int H = a.Hq + a.Hkv;
  const int hl = threadIdx.x % LPH;   // lane of its head
  const int items = TB * H, per = (items + parts * HPW - 1) / (parts * HPW) * HPW;   // (token, head) items of a share
  const int x0 = part * per + threadIdx.x / LPH, x1 = min(part * per + per, items);
  struct Item {
    int64_t t;   // token row, -1: none
    int h, tb;
    Raw8<T> raw;
  };
  auto fetch = [&](int x, Item& it, auto row_of) __attribute__((always_inline)) {   // (always loads: row 0 where there is none)
    const bool on = x < x1;
    x = on ? x : 0;
    it.tb = x / (uint32_t)H;
    it.h = x - it.tb * H;
    it.t = on ? row_of(it.tb) : -1;
    const int64_t row = it.t < 0 ? 0 : it.t;
    it.raw.load((it.h < a.Hq ? (const T*)a.q + row * a.q_ld + it.h * D : (const T*)a.k + row * a.k_ld + (it.h - a.Hq) * D) + hl * 8);
  };
  Item even, odd;
  fetch(x0, even, [&](int i) {
    int pos;
    return token(i, &pos);
  });
  float gq[8], gk[8];
  if (a.gq) load8((const T*)a.gq + hl * 8, gq);
  if (a.gk) load8((const T*)a.gk + hl * 8, gk);
  {
    const int pr = threadIdx.x % (D / 2), mine = threadIdx.x / (D / 2);
    int pos = 0;
    const int64_t row = token(mine, &pos);
    if (pr == 0) rows[mine] = row;
    cos_sin((double)max(pos, 0) * (ROWS ? a.d_theta[pr] : a.theta[pr]), &cs[mine][pr], &sn[mine][pr]);
  }
  __syncthreads();
  auto finish = [&](const Item& it) __attribute__((always_inline)) {
    const bool isq = it.h < a.Hq;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = it.raw.at(e);
    if (isq ? a.gq != nullptr : a.gk != nullptr) {
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
#pragma unroll
      for (int o = LPH / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
      const float inv = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * inv * (isq ? gq[e] : gk[e]);
    }
    float o8[8];
    if constexpr (NEOX) {
      const bool second = hl >= LPH / 2;
      const int p0 = (hl % (LPH / 2)) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = __shfl_xor(y[e], LPH / 2, 64);
        const float c = cs[it.tb][p0 + e], s = sn[it.tb][p0 + e];
        o8[e] = second ? y[e] * c + z * s : y[e] * c - z * s;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float c = cs[it.tb][hl * 4 + e], s = sn[it.tb][hl * 4 + e];
        o8[2 * e] = y[2 * e] * c - y[2 * e + 1] * s;
        o8[2 * e + 1] = y[2 * e + 1] * c + y[2 * e] * s;
      }
    }
    T* dst = isq ? (T*)a.qo + it.t * a.qo_ld + it.h * D : (T*)a.ko + it.t * a.ko_ld + (it.h - a.Hq) * D;
    if (it.t >= 0) store8(dst + hl * 8, o8);
  };
  auto row_at = [&](int i) { return rows[i]; };
  for (int x = x0 - (int)threadIdx.x / LPH; x < x1; x += 2 * HPW) {   // (uniform; an item's lanes stay together)
    const int mine = x + (int)threadIdx.x / LPH;
    fetch(mine + HPW, odd, row_at);
    finish(even);
    if (x + HPW < x1) {
      fetch(mine + 2 * HPW, even, row_at);
      finish(odd);
    }
  }
}

}  // namespace

hipError_t launch_append_slots(const AppendSlotsK& a, hipStream_t s) {
  const int64_t least = (int64_t)kSlotRun * kSlotTokens;
  const int per_wg = (int)least;
  const int64_t wgs = 1 + (a.max_tokens + least - 1) / least;
  hipLaunchKernelGGL(append_slots_kernel, dim3((unsigned)wgs), dim3(kSlotRun), 0, s, a, per_wg);
  return hipGetLastError();
}

template <typename T, int D, bool NEOX>
static void launch_qk(const QkNormRopeK& a, hipStream_t s) {
  constexpr int TB = 256 / (D / 2), HPW = 256 / (D / 8);
  const int rows = a.rows ? a.max_rows : a.n;
  const int64_t groups = (int64_t)((rows + TB - 1) / TB) * (a.rows ? a.n_req : 1);
  // shares of a group's heads: up to 2048 workgroups, one pass of the workgroup each at the least.  256 tokens of 32 / 8
  // heads (d = 128): 4.9 us in ten shares, 11.4 in one.
  const int passes = (TB * (a.Hq + a.Hkv) + HPW - 1) / HPW;
  const int64_t want = groups > 0 ? 2048 / groups : 1;
  const int parts = (int)(want < 1 ? 1 : want > passes ? passes : want);
  if (a.rows)
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, NEOX, true>), dim3((unsigned)((rows + TB - 1) / TB * parts), (unsigned)a.n_req),
                       dim3(256), 0, s, a, parts);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, NEOX, false>), dim3((unsigned)((rows + TB - 1) / TB * parts)), dim3(256), 0, s,
                       a, parts);
}

hipError_t launch_qk_norm_rope(const QkNormRopeK& a, int D, bool f32, bool neox, hipStream_t s) {
#define SX_QK(T_)                                                                    \
  do {                                                                               \
    if (D == 128) { if (neox) launch_qk<T_, 128, true>(a, s); else launch_qk<T_, 128, false>(a, s); } \
    else { if (neox) launch_qk<T_, 64, true>(a, s); else launch_qk<T_, 64, false>(a, s); }            \
  } while (0)
  if (f32) SX_QK(float); else SX_QK(uint16_t);
#undef SX_QK
  return hipGetLastError();
}

}  // namespace sx
