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
// own range of token indices from the run in LDS; workgroup 0 writes what there is one of per request.
// ---------------------------------------------------------------------------------------------
constexpr int kSlotRun = 256;    // requests a run, and threads
constexpr int kSlotTokens = 4;   // tokens per thread and workgroup at the least

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

__global__ __launch_bounds__(kSlotRun) void append_slots_kernel(AppendSlotsK a, int per_wg) {
  __shared__ SlotRun run;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool per_request = blockIdx.x == 0;
  const int64_t t0 = (int64_t)(blockIdx.x - 1) * per_wg;   // this workgroup's token indices (not workgroup 0)
  const int64_t t1 = min(t0 + per_wg, (int64_t)a.max_tokens);
  const int64_t head = a.free_head ? max(a.free_head[0], 0) : 0;
  const int b = a.block;
  int64_t tok = 0, blk = 0, missing = 0;
  for (int r0 = 0; r0 < a.n_req; r0 += kSlotRun) {
    const int r = r0 + tid;
    const int ctx = r < a.n_req ? max(a.ctx[r], 0) : 0;
    const int add = r < a.n_req ? (a.add ? max(a.add[r], 0) : 1) : 0;
    const int64_t len = (int64_t)ctx + add;
    const int64_t have = ((int64_t)ctx + b - 1) / b;
    const int64_t need = max(min((len + b - 1) / b, (int64_t)a.max_blocks) - have, (int64_t)0);
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
      if (r < a.n_req) {
        a.seq[r] = (int)min(len, (int64_t)INT32_MAX);
        a.cu[r] = (int)min(c, (int64_t)INT32_MAX);
        // tokens without a slot: all before `from` (the open block's entry is missing) and all from `upto`
        // on (no block left, or no room in the table)
        const int64_t got = max(min((int64_t)a.n_free - f, need), (int64_t)0);
        int64_t from = 0;
        if (have * b > ctx && add > 0)
          if (have > a.max_blocks || a.table[(int64_t)r * a.max_blocks + have - 1] < 0) from = min(have * b - ctx, (int64_t)add);
        const int64_t upto = max(min(min(have + got, (int64_t)a.max_blocks) * b - ctx, (int64_t)add), (int64_t)0);
        const int64_t room = max(min((int64_t)a.max_tokens - c, (int64_t)add), (int64_t)0);
        missing += add - max(min(upto, room) - from, (int64_t)0);
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
        const int64_t p = (int64_t)run.ctx[lo] + (x - run.tok[lo]);
        const int64_t bi = p / b, hv = ((int64_t)run.ctx[lo] + b - 1) / b;
        int32_t* row = a.table + (int64_t)(r0 + lo) * a.max_blocks;
        int id = -1;
        if (bi < a.max_blocks) {
          if (bi < hv) {
            id = row[bi];
          } else {
            const int64_t f = head + blk + run.blk[lo] + bi - hv;
            if (f >= 0 && f < a.n_free) id = a.free_blocks[f];
            if (p % b == 0) row[bi] = id;
          }
        }
        const int64_t slot = (int64_t)id * b + p % b;
        a.pos[i] = (int)min(p, (int64_t)INT32_MAX);
        a.slots[i] = id >= 0 && slot <= INT32_MAX ? (int)slot : -1;
      }
    }
    tok += all_tok;
    blk += all_blk;
    __syncthreads();   // the run's LDS is free again
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
// ---------------------------------------------------------------------------------------------
template <typename T, int D, bool NEOX, bool ROWS>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNormRopeK a) {
  constexpr int TB = 256 / (D / 2);   // tokens per workgroup
  constexpr int LPH = D / 8;          // lanes per head
  __shared__ __attribute__((aligned(16))) float cs[TB][D / 2], sn[TB][D / 2];
  __shared__ int64_t trow[TB];        // token row, -1: none
  const int n0 = blockIdx.x * TB;
  const int tb0 = threadIdx.x / (D / 2), pr = threadIdx.x % (D / 2);
  {
    int64_t t = -1;
    int p = -1;
    if constexpr (ROWS) {
      const ReqDev rq = a.reqs[blockIdx.y];
      if (n0 >= min(a.n_rows[blockIdx.y], a.max_rows)) return;
      if (n0 + tb0 < min(a.n_rows[blockIdx.y], a.max_rows)) {
        t = (int64_t)rq.tok_off + a.rows[rq.tok_off + n0 + tb0];
        p = a.tok_pos[t];
      }
    } else if (n0 + tb0 < a.n) {
      t = n0 + tb0;
      p = a.pos[t];
    }
    if (p < 0) t = -1;
    const double phi = (double)max(p, 0) * (ROWS ? a.d_theta[pr] : a.theta[pr]);
    cs[tb0][pr] = (float)cos(phi);
    sn[tb0][pr] = (float)sin(phi);
    if (pr == 0) trow[tb0] = t;
  }
  __syncthreads();
  const int H = a.Hq + a.Hkv;
  const int hl = threadIdx.x % LPH;   // lane of its head
  for (int x = threadIdx.x / LPH; x < TB * H; x += 256 / LPH) {
    const int tb = x / H, h = x - tb * H;
    const int64_t t = trow[tb];
    const bool isq = h < a.Hq;
    const bool live = t >= 0;
    float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (live) {
      const T* src = isq ? (const T*)a.q + t * a.q_ld + h * D : (const T*)a.k + t * a.k_ld + (h - a.Hq) * D;
      load8(src + hl * 8, y);
    }
    const void* gamma = isq ? a.gq : a.gk;
    if (gamma) {
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
#pragma unroll
      for (int o = LPH / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
      const float inv = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
      float g[8];
      load8((const T*)gamma + hl * 8, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * inv * g[e];
    }
    float o8[8];
    if constexpr (NEOX) {
      const bool second = hl >= LPH / 2;
      const int p0 = (hl % (LPH / 2)) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = __shfl_xor(y[e], LPH / 2, 64);
        const float c = cs[tb][p0 + e], s = sn[tb][p0 + e];
        o8[e] = second ? y[e] * c + z * s : y[e] * c - z * s;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float c = cs[tb][hl * 4 + e], s = sn[tb][hl * 4 + e];
        o8[2 * e] = y[2 * e] * c - y[2 * e + 1] * s;
        o8[2 * e + 1] = y[2 * e + 1] * c + y[2 * e] * s;
      }
    }
    if (live) {
      T* dst = isq ? (T*)a.qo + t * a.qo_ld + h * D : (T*)a.ko + t * a.ko_ld + (h - a.Hq) * D;
      store8(dst + hl * 8, o8);
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
  constexpr int TB = 256 / (D / 2);
  if (a.rows)
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, NEOX, true>), dim3((unsigned)((a.max_rows + TB - 1) / TB), (unsigned)a.n_req),
                       dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, NEOX, false>), dim3((unsigned)((a.n + TB - 1) / TB)), dim3(256), 0, s, a);
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
