// Attention over the 4-bit cache (include/sx_decode.h).
//
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_16x16x32_bf16 with 16 query rows (token x head of the group)
// as the columns, so a lane owns one row throughout: lane l holds row l % 16 of S^T for the keys 4 (l / 16) ..
// + 3 of each of two blocks, and takes exactly these keys' probabilities as its part of the P^T operand (the
// keys of a step are numbered (l / 16, block, i) for the second product; any order gives the same sum).  The
// record's byte order makes a block's K and V one consecutive load per lane each, and K's scale one byte per
// lane; the codes become bfloat16 in registers, two elements an instruction, exactly.  Nothing goes through
// LDS until the waves of a workgroup, which take the steps of a chunk of keys in turn, add up their parts.
// Softmax statistics and sums are float32; a probability goes into the product as two bfloat16 parts (float32
// q: three, and q itself in three), so what is lost there is below the rounding of the output.
#include "sx_kv4_device.h"

namespace sx {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
constexpr float kNegInf = -__builtin_huge_valf();
// Requests of more rows per KV head than this take the kernel for many rows (bfloat16).
constexpr int kKv4FewRows = 64;

__device__ __forceinline__ bf16x8_t as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8_t, (u32x4_t){a, b, c, d});
}
__device__ __forceinline__ f32x4_t mfma16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Workgroup barrier that orders LDS only: global loads stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A float32 as a sum of N bfloat16 parts, each the rounding of what the others leave (an infinity or NaN
// stands in the first alone): part i of x[0..8).
template <int N>
__device__ __forceinline__ void split_parts(const float (&x)[8], bf16x8_t (&part)[N]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(rest[2 * e], rest[2 * e + 1]);
    part[i] = as_bf16x8(w[0], w[1], w[2], w[3]);
#pragma unroll
    for (int e = 0; e < 4 && i + 1 < N; ++e) {
      const float lo = bf16_lo(w[e]), hi = bf16_hi(w[e]);
      rest[2 * e] = __builtin_isfinite(lo) ? rest[2 * e] - lo : 0.0f;
      rest[2 * e + 1] = __builtin_isfinite(hi) ? rest[2 * e + 1] - hi : 0.0f;
    }
  }
}

// A lane's bytes of one block: D / 32 dwords of K (token l % 16, elements D / 4 (l / 16) ..) and of V (tokens
// 4 (l / 16) .. + 3, the column group l % 16), and their scale bytes.
template <int D>
struct Page {
  uint32_t k[D / 32], v[D / 32];
  uint32_t ks, vs;
  __device__ __forceinline__ void load(const uint8_t* rec, int lane) {
    const int tok = lane & 15, lg = lane >> 4;
    if constexpr (D == 128) {
      const uint4 x = *(const uint4*)(rec + lane * 16), y = *(const uint4*)(rec + kv4_v_codes(D) + lane * 16);
      k[0] = x.x; k[1] = x.y; k[2] = x.z; k[3] = x.w;
      v[0] = y.x; v[1] = y.y; v[2] = y.z; v[3] = y.w;
    } else {
      const uint2 x = *(const uint2*)(rec + lane * 8), y = *(const uint2*)(rec + kv4_v_codes(D) + lane * 8);
      k[0] = x.x; k[1] = x.y;
      v[0] = y.x; v[1] = y.y;
    }
    ks = rec[kv4_k_scales(D) + lg * (D / 4) / kKv4Group * 16 + tok];
    vs = *(const uint32_t*)(rec + kv4_v_scales(D) + tok * (D / 16) / kKv4Group * 16 + 4 * lg);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) k[i] = v[i] = 0;
    ks = 127;
    vs = 0x7f7f7f7fu;
  }
  // values of the keys n .. 15 become zero: a NaN there would pass through a zero probability
  __device__ __forceinline__ void drop_values_from(int n, int lane) {
    const int t = n - 4 * (lane >> 4);   // this lane's first dropped token
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i >= t) {
        vs = (vs & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));
        if constexpr (D == 128) v[i] = 0;
        else v[i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
      }
  }
  // K operand of elements 8 c .. 8 c + 7 of the lane's quarter
  __device__ __forceinline__ bf16x8_t k_part(int c) const {
    const float s = kv4_scale(ks);
    return as_bf16x8(kv4_pair<0>(k[c], s), kv4_pair<1>(k[c], s), kv4_pair<2>(k[c], s), kv4_pair<3>(k[c], s));
  }
  // V of the lane's four tokens: w[token][pair of columns]
  __device__ __forceinline__ void values(uint32_t (&w)[4][D / 32]) const {
    const float s[4] = {kv4_scale(vs & 0xff), kv4_scale(vs >> 8 & 0xff), kv4_scale(vs >> 16 & 0xff), kv4_scale(vs >> 24)};
    if constexpr (D == 128) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i][0] = kv4_pair<0>(v[i], s[i]);
        w[i][1] = kv4_pair<1>(v[i], s[i]);
        w[i][2] = kv4_pair<2>(v[i], s[i]);
        w[i][3] = kv4_pair<3>(v[i], s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        w[i][0] = kv4_pair<0>(v[i / 2], s[i]);
        w[i][1] = kv4_pair<1>(v[i / 2], s[i]);
        w[i + 1][0] = kv4_pair<2>(v[i / 2], s[i + 1]);
        w[i + 1][1] = kv4_pair<3>(v[i / 2], s[i + 1]);
      }
    }
  }
  // a NaN group among the values of the lane's tokens
  __device__ __forceinline__ bool bad_values() const {
    return (vs & 0xff) == 0xff || (vs & 0xff00) == 0xff00 || (vs & 0xff0000) == 0xff0000 || vs >> 24 == 0xff;
  }
};

// What the kernels derive from a request's lengths, each cut to the call's bounds.
struct Request {
  int q0, nq, len, rows, off;   // first query row, query tokens, keys, rows per KV head, position of the first query
  Kv4Split split;
  __device__ __forceinline__ Request(const Kv4AttnK& a, int r) {
    const int G = a.Hq / a.Hkv;
    q0 = min(max(a.cu[r], 0), a.total_q);
    nq = max(min(min(a.cu[r + 1], a.total_q) - q0, a.max_q), 0);
    len = max(min(a.lens[r], (int)min((int64_t)a.max_seqlen, (int64_t)a.max_blocks * kBlock)), 0);
    rows = nq * G;
    off = len - nq;
    split = kv4_split(rows, len);
  }
};

// ---------------------------------------------------------------------------------------------
// One workgroup: 16 rows of one KV head over one chunk of keys, its NW waves taking steps of two blocks in
// turn.  Writes the rows' results, or their parts where the request's keys are split.
// ---------------------------------------------------------------------------------------------
template <typename T, int D, int NW>
__global__ __launch_bounds__(NW * 64) void kv4_attn_kernel(Kv4AttnK a, int tiles) {
  constexpr int NC = D / 32;                  // 32-element pieces of a row
  constexpr int NU = D / 16;                  // 16-column tiles of V
  constexpr int NQ = sizeof(T) == 4 ? 3 : 1;  // bfloat16 parts of a query element, and of a probability
  constexpr int NP = sizeof(T) == 4 ? 3 : 2;
  constexpr int OP = D + 4;                   // LDS row pitch
  __shared__ __attribute__((aligned(16))) float so[NW][16][OP];
  __shared__ float sm[NW][16], sl[NW][16];
  int idx = blockIdx.x;
  const int h = idx % a.Hkv;
  idx /= a.Hkv;
  const int c = idx / tiles, tile = idx % tiles, r = blockIdx.y;   // (chunks slowest, as below)
  const Request q(a, r);
  const int row0 = tile * 16;
  if (row0 >= q.rows || c >= q.split.n || (sizeof(T) == 2 && q.rows > kKv4FewRows)) return;
  const int G = a.Hq / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = min(row0 + (lane & 15), q.rows - 1), lg = lane >> 4;
  const int lim = q.off + row / G;            // last key that this lane's row sees
  const int lim_min = q.off + row0 / G, lim_max = q.off + min(row0 + 15, q.rows - 1) / G;
  const int k0 = c * q.split.keys;            // (c < n: below len)
  const int k1 = min(min(k0 + (int64_t)q.split.keys, (int64_t)q.len), (int64_t)lim_max + 1);
  const int32_t* table = a.table + (int64_t)r * a.max_blocks;

  bf16x8_t qf[NC][NQ];
  {
    const T* src = (const T*)a.q + (int64_t)(q.q0 + row / G) * a.q_ld + (h * G + row % G) * D + lg * (D / 4);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if constexpr (NQ == 1) {
        qf[i][0] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(src + i * 8));
      } else {
        float x[8];
        load8(src + i * 8, x);
        split_parts<NQ>(x, qf[i]);
      }
    }
  }
  f32x4_t o[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) o[u] = (f32x4_t){0, 0, 0, 0};
  float m = kNegInf, l = 0.0f;

  for (int kb = k0 + wave * 32; kb < k1; kb += NW * 32) {
    Page<D> pg[2];
    bool have[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int p = kb / kBlock + j;
      const int id = p * kBlock < k1 ? table[p] : -1;
      have[j] = id >= 0 && id < a.n_blocks;
      if (have[j]) pg[j].load(a.pool + ((int64_t)id * a.Hkv + h) * kv4_record(D), lane);
      else pg[j].clear();
      if ((p + 1) * kBlock > q.len) pg[j].drop_values_from(q.len - p * kBlock, lane);
    }
    float s[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f32x4_t acc = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const bf16x8_t kf = pg[j].k_part(i);
#pragma unroll
        for (int n = NQ - 1; n >= 0; --n) acc = mfma16(kf, qf[i][n], acc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * j + i] = acc[i];
    }
    const bool edge = kb + 31 > lim_min;       // some row does not see every key of the step
    if (edge || !have[0] || !have[1]) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!have[j] || kb + 16 * j + 4 * lg + i > lim) s[4 * j + i] = kNegInf;
    }
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i]);
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float mn = fmaxf(m, top * a.scale);
    const float base = mn == kNegInf ? 0.0f : mn;
    if (__any(mn > m)) {
      const float f = __builtin_amdgcn_exp2f(m - base);
      l *= f;
#pragma unroll
      for (int u = 0; u < NU; ++u) o[u] *= f;
      m = mn;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale, -base));
      l += p[i];
    }
    bf16x8_t pf[NP];
    split_parts<NP>(p, pf);
    // a NaN group among the values of keys that some rows see and some do not: these rows get it, the others
    // nothing
    if (edge && __any(pg[0].bad_values() || pg[1].bad_values())) {
      float nan = 0.0f;
      const int grp = lg * (D / 4) / kKv4Group;   // of the output elements that this lane holds
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int pbase = kb + 16 * j;
        if (have[j]) {
          const uint8_t* sc = a.pool + ((int64_t)table[pbase / kBlock] * a.Hkv + h) * kv4_record(D) + kv4_v_scales(D) + grp * 16;
          for (int t = 0; t < 16 && pbase + t < q.len; ++t)
            if (sc[t] == 255 && pbase + t <= lim) nan = __builtin_nanf("");
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((pg[j].vs >> (8 * i) & 0xff) == 0xff) {
            pg[j].vs = (pg[j].vs & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));   // (its codes are zero)
          }
      }
#pragma unroll
      for (int u = 0; u < NU; ++u) o[u] += nan;
    }
    uint32_t w0[4][NC], w1[4][NC];
    pg[0].values(w0);
    pg[1].values(w1);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      // element u of every token: the low or high half of its pair u / 2
      const uint32_t sel = u % 2 ? 0x07060302u : 0x05040100u;
      const int b = u / 2;
      const bf16x8_t vf = as_bf16x8(__builtin_amdgcn_perm(w0[1][b], w0[0][b], sel), __builtin_amdgcn_perm(w0[3][b], w0[2][b], sel),
                                    __builtin_amdgcn_perm(w1[1][b], w1[0][b], sel), __builtin_amdgcn_perm(w1[3][b], w1[2][b], sel));
#pragma unroll
      for (int n = NP - 1; n >= 0; --n) o[u] = mfma16(vf, pf[n], o[u]);
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);

  // the waves' parts: lane l holds row l % 16, columns D / 4 (l / 16) + (D / 16) i + u
  {
    float* dst = &so[wave][lane & 15][lg * (D / 4)];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < NU; u += 4)
        *(float4*)(dst + i * NU + u) = make_float4(o[u][i], o[u + 1][i], o[u + 2][i], o[u + 3][i]);
    if (lg == 0) {
      sm[wave][lane & 15] = m;
      sl[wave][lane & 15] = l;
    }
  }
  __syncthreads();
  constexpr int TPR = NW * 64 / 16;           // threads per row
  constexpr int EPT = D / TPR;                // elements per thread
  const int rr = tid / TPR, d0 = tid % TPR * EPT;
  if (row0 + rr >= q.rows) return;
  float mt = sm[0][rr];
#pragma unroll
  for (int w = 1; w < NW; ++w) mt = fmaxf(mt, sm[w][rr]);
  const float base = mt == kNegInf ? 0.0f : mt;
  float lt = 0.0f, acc[EPT];
#pragma unroll
  for (int e = 0; e < EPT; ++e) acc[e] = 0.0f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float f = __builtin_amdgcn_exp2f(sm[w][rr] - base);
    lt = __builtin_fmaf(sl[w][rr], f, lt);
#pragma unroll
    for (int e = 0; e < EPT; ++e) acc[e] = __builtin_fmaf(so[w][rr][d0 + e], f, acc[e]);
  }
  const int orow = row0 + rr;
  if (q.split.n == 1) {
    const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
    const int64_t at = (int64_t)(q.q0 + orow / G) * a.Hq + h * G + orow % G;
    T* dst = (T*)a.out + at * D + d0;
#pragma unroll
    for (int e = 0; e < EPT; e += 2) {
      if constexpr (sizeof(T) == 2) *(uint32_t*)(dst + e) = pack_bf16x2(acc[e] * inv, acc[e + 1] * inv);
      else *(float2*)(dst + e) = make_float2(acc[e] * inv, acc[e + 1] * inv);
    }
    if (a.lse && d0 == 0) a.lse[at] = (mt + __builtin_amdgcn_logf(lt)) * 0.69314718055994530942f;
  } else {
    const int64_t at = ((int64_t)r * a.Hkv + h) * a.part_rows + (int64_t)c * q.rows + orow;
    float* dst = a.part + at * D + d0;
#pragma unroll
    for (int e = 0; e < EPT; e += 2) *(float2*)(dst + e) = make_float2(acc[e], acc[e + 1]);
    if (d0 == 0) a.part_ml[at] = make_float2(mt, lt);
  }
}

// ---------------------------------------------------------------------------------------------
// Many query rows (bfloat16): one workgroup of 8 waves takes 256 columns (32 a wave) of one KV head over one
// chunk of keys, in tiles of 64 keys = 4 blocks.  Each wave turns the K or the V of one block of the tile into
// bfloat16 operands of v_mfma_f32_32x32x16_bf16 and leaves them in LDS in lane order, so that every operand is
// one conflict-free 16-byte read; the conversion is paid once for 256 columns instead of once for 16.
// S^T = K Q^T: a lane owns one column, its keys 8 (e / 4) + 4 hg + e % 4 of each 32; these registers are the
// P^T operand of O^T += V^T P^T as they stand (the V operand is laid out for this key order, and for columns
// d = (D / 16) (m % 16) + 2 dt + m / 16 of tile dt).
// Two groups of four waves, one of each per SIMD, alternate a matrix phase (P V of tile j - 1, S of tile j) and
// a vector phase (conversion of tile j + 1, softmax of tile j), a barrier after each: the matrix cores run while
// the other group's exponentials do.  Writes of tile T end before the barrier that precedes the first reads;
// with three buffers its predecessor there, T - 3, was last read (its V) in iteration T - 2, while the earliest
// write of T comes in iteration T - 1.
// Probabilities are rounded to bfloat16 once, as in full and sparse attention: the error of a result, 2^-9 of its
// typical size, is that of its own rounding (0.0024 relative with both, 0.0017 with the output's alone), and two
// parts cost 1378 us where one costs 964.  Sums and statistics are float32; the running maximum is raised only
// when a probability would reach 2^64.
// 2048 tokens of 32 / 8 heads over 32768 keys (d = 128): 964 us, 1.10 PFLOP/s; the kernel for few rows took 11.4 ms.
// ---------------------------------------------------------------------------------------------
constexpr int kWideCols = 256;
constexpr int kWideKeys = 64;

template <int D>
__global__ __launch_bounds__(512, 1) void kv4_attn_wide_kernel(Kv4AttnK a, int tiles) {
  constexpr int NS = D / 16;          // 16-element slices of a key
  constexpr int ND = D / 32;          // 32-column tiles of the output; dwords of codes per lane
  constexpr int TILEB = kWideKeys * D * 2;
  constexpr int NBUF = 3;
  __shared__ __attribute__((aligned(1024))) char smem[2 * NBUF * TILEB];   // [buffer][K], [buffer][V]
  __shared__ int s_nan[NBUF];         // NaN groups among the values of the buffer's tile (replaced by zero)
  int idx = blockIdx.x;
  const int h = idx % a.Hkv;
  idx /= a.Hkv;
  // chunks slowest: workgroups beyond a request's last chunk end at once, and between live ones they would put
  // these on a few shader engines; later rows see more keys and come first
  const int c = idx / tiles, tile = tiles - 1 - idx % tiles, r = blockIdx.y;
  const Request q(a, r);
  const int row0 = tile * kWideCols;
  if (q.rows <= kKv4FewRows || row0 >= q.rows || c >= q.split.n) return;
  const int G = a.Hq / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hg = lane >> 5;
  const int wrow = row0 + wave * 32;
  const int row = min(wrow + l32, q.rows - 1);
  const bool valid = wrow + l32 < q.rows;
  const int lim = q.off + row / G;
  const int lim0 = q.off + row0 / G, lim1 = q.off + min(row0 + kWideCols - 1, q.rows - 1) / G;   // of the workgroup
  const int wave_min = q.off + min(wrow, q.rows - 1) / G;
  const int wave_max = wrow < q.rows ? q.off + min(wrow + 31, q.rows - 1) / G : -1;
  const int k0 = c * q.split.keys;    // (a multiple of kKv4Step = 128)
  const int k1 = (int)min(min(k0 + (int64_t)q.split.keys, (int64_t)q.len), (int64_t)lim1 + 1);
  const int nkt = k1 > k0 ? (k1 - k0 + kWideKeys - 1) / kWideKeys : 0;
  const int32_t* table = a.table + (int64_t)r * a.max_blocks;
  const float c2 = a.scale;

  bf16x8_t qb[NS];
  {
    const uint16_t* src = (const uint16_t*)a.q + (int64_t)(q.q0 + row / G) * a.q_ld + (h * G + row % G) * D + hg * 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) qb[s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(src + s * 16));
  }
  f32x16_t o[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;
  float m_run = kNegInf, l_run = 0.0f;

  // ---- staging: this wave's block and matrix of every tile ----
  const int grp = wave >> 2;
  const int sj = wave >> 1;
  const bool sv = wave & 1;
  // block ids of 16 tiles at a time, one a lane (-1: not there), the next 16 tiles' on their way
  auto load_ids = [&](int run) {
    const int page = k0 / kBlock + run * 64 + lane;
    const int id = (int64_t)page * kBlock < k1 ? table[page] : -1;
    return id < a.n_blocks ? id : -1;
  };
  int ids = load_ids(0), next_ids = load_ids(1);
  uint64_t gone_ids = __ballot(ids < 0), gone_tiles = 0;   // missing blocks: of `ids`; four bits a fetched tile
  uint32_t code[ND], scale = 0;
  bool there = false;
  auto fetch = [&](int t) {           // its codes and scales of tile t (called for 0, 1, 2, ...)
    if (t > 0 && (t & 15) == 0) {
      ids = next_ids;
      next_ids = load_ids((t >> 4) + 1);
      gone_ids = __ballot(ids < 0);
    }
    const int at = (t & 15) * 4;
    gone_tiles = gone_tiles << 4 | (gone_ids >> at & 15);
    const int id = __builtin_amdgcn_readlane(ids, at + sj);
    there = id >= 0;
    if (!there) return;
    const uint8_t* rec = a.pool + ((int64_t)id * a.Hkv + h) * kv4_record(D);
    const uint8_t* src = rec + (sv ? kv4_v_codes(D) : 0) + lane * (D / 8);
    if constexpr (D == 128) {
      const uint4 x = *(const uint4*)src;
      code[0] = x.x; code[1] = x.y; code[2] = x.z; code[3] = x.w;
    } else {
      const uint2 x = *(const uint2*)src;
      code[0] = x.x; code[1] = x.y;
    }
    const int tok = lane & 15, lg = lane >> 4;
    if (sv) scale = *(const uint32_t*)(rec + kv4_v_scales(D) + tok * (D / 16) / kKv4Group * 16 + 4 * lg);
    else scale = rec[kv4_k_scales(D) + lg * (D / 4) / kKv4Group * 16 + tok];
  };
  auto stage = [&](int t, int buf) {  // ... as operands in LDS
    if (t >= nkt) return;
    Page<D> p;
    p.clear();
    const int key = k0 + t * kWideKeys + sj * kBlock;
    const int tok = lane & 15, lg = lane >> 4;
    if (sv) {
      if (there) {
#pragma unroll
        for (int i = 0; i < ND; ++i) p.v[i] = code[i];
        p.vs = scale;
      }
      if (key + kBlock > q.len) p.drop_values_from(q.len - key, lane);
      if (k0 + t * kWideKeys + kWideKeys - 1 > lim0) {   // some row does not see every key of the tile
        const bool bad = p.bad_values();
        if (__any(bad)) {
          if (lane == 0) s_nan[buf] = 1;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((p.vs >> (8 * i) & 0xff) == 0xff) p.vs = (p.vs & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));
        }
      }
      uint32_t w[4][ND];
      p.values(w);
      char* dst = smem + (NBUF + buf) * TILEB + sj * ND * 1024 + ((lg & 1) * 32 + tok) * 16 + (lg >> 1) * 8;
#pragma unroll
      for (int u = 0; u < 2 * ND; ++u) {
        const uint32_t sel = u % 2 ? 0x07060302u : 0x05040100u;
        *(uint2*)(dst + u / 2 * 1024 + u % 2 * 256) = make_uint2(__builtin_amdgcn_perm(w[1][u / 2], w[0][u / 2], sel),
                                                                __builtin_amdgcn_perm(w[3][u / 2], w[2][u / 2], sel));
      }
    } else {
      if (there) {
#pragma unroll
        for (int i = 0; i < ND; ++i) p.k[i] = code[i];
        p.ks = scale;
      }
      char* dst = smem + buf * TILEB + (sj >> 1) * NS * 1024 + ((sj & 1) * 16 + tok) * 16;
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        const int id = lg * ND + i;   // elements 8 id ..
        *(bf16x8_t*)(dst + (id >> 1) * 1024 + (id & 1) * 512) = p.k_part(i);
      }
    }
  };

  // ---- tile computations ----
  f32x16_t sacc[2];
  bf16x8_t pb[4];
  auto s_tile = [&](const char* kb) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int e = 0; e < 16; ++e) sacc[mt][e] = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
        sacc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t*)(kb + (mt * NS + s) * 1024 + lane * 16), qb[s],
                                                           sacc[mt], 0, 0, 0);
    sched_pipelined<2 * NS, 1, 4>();
  };
  auto pv_tile = [&](const char* vb) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t*)(vb + (kk * ND + dt) * 1024 + lane * 16), pb[kk],
                                                        o[dt], 0, 0, 0);
    sched_pipelined<4 * ND, 1, 4>();
  };
  auto softmax_tile = [&](int j, int buf) {
    const int kbase = k0 + j * kWideKeys;
    // blocks of the tile that are not there (its group has fetched 2, or 3, tiles since)
    const int gone = (int)(gone_tiles >> (4 * (2 + grp)) & 15);
    const bool edge = kbase + kWideKeys - 1 > wave_min;
    if (edge || gone) {
      const int last = lim - kbase - hg * 4;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = mt * 32 + (e >> 2) * 8 + (e & 3);   // (+ 4 hg; the block is key / 16)
          if (key > last || (gone >> (mt * 2 + (e >> 3)) & 1)) sacc[mt][e] = kNegInf;
        }
    }
    float psum = 0.0f;
    auto expo = [&](float mneg) {
      psum = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        float x[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          x[t] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[kk >> 1][(kk & 1) * 8 + t], c2, mneg));
          psum += x[t];
        }
        pb[kk] = as_bf16x8(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
      }
    };
    expo(-m_run);
    if (__ballot(!(psum < 0x1p64f))) {
      float mx = sacc[0][0];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sacc[mt][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = fmaxf(m_run, mx * c2);
      const float f = m_new == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= f;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] *= f;
      m_run = m_new;
      expo(m_new == kNegInf ? 0.0f : -m_new);
    }
    l_run += psum;
    if (kbase + kWideKeys - 1 > lim0 && s_nan[buf]) {   // rows that see a NaN group get it (its values went into LDS as zeros)
      float nan[2] = {0.0f, 0.0f};   // groups of this lane's columns: D = 128: hg, 2 + hg; D = 64: 0, 1
      for (int b = 0; b < 4; ++b) {
        const int key = kbase + b * kBlock;
        if (gone >> b & 1) continue;
        const uint8_t* sc = a.pool + ((int64_t)table[key / kBlock] * a.Hkv + h) * kv4_record(D) + kv4_v_scales(D);
        for (int t = 0; t < kBlock && key + t < q.len; ++t)
#pragma unroll
          for (int n = 0; n < 2; ++n)
            if (sc[(D == 128 ? 2 * n + hg : n) * 16 + t] == 255 && key + t <= lim) nan[n] = __builtin_nanf("");
      }
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] += nan[e >> 2 & 1];
    }
  };

  // ---- schedule (see above): U(j) = matrix phase j | barrier | vector phase | barrier ----
  if (tid < NBUF) s_nan[tid] = 0;
  lds_barrier();
  fetch(0);
  stage(0, 0);
  fetch(1);
  lds_barrier();
  auto matrix_phase = [&](int j, int ph) {
    __builtin_amdgcn_s_setprio(2);
    if (j >= 1 && j - 1 < nkt && k0 + (j - 1) * kWideKeys <= wave_max) pv_tile(smem + (NBUF + (ph + NBUF - 1) % NBUF) * TILEB);
    if (j < nkt && k0 + j * kWideKeys <= wave_max) s_tile(smem + ph * TILEB);
    __builtin_amdgcn_s_setprio(0);
  };
  auto stage_phase = [&](int j, int ph) {   // tile j + 1; codes of tile j + 2 on their way
    stage(j + 1, (ph + 1) % NBUF);
    fetch(j + 2);
  };
  auto iter_u = [&](int j, int ph) {
    matrix_phase(j, ph);
    lds_barrier();
    stage_phase(j + grp, (ph + grp) % NBUF);
    if (j < nkt && k0 + j * kWideKeys <= wave_max) softmax_tile(j, ph);
    lds_barrier();
  };
  if (grp) {
    stage_phase(0, 0);
    lds_barrier();
  }
  for (int j = 0; j <= nkt; j += 3) {
    iter_u(j, 0);
    iter_u(j + 1, 1);
    iter_u(j + 2, 2);
  }
  if (!grp) lds_barrier();

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if (!valid) return;
  // columns (D / 16) cg + 2 dt + n of the lane: cg = 8 g + 4 hg + i, element e = 8 n + 4 g + i
  if (q.split.n == 1) {
    const float inv = l_tot == 0.0f ? 0.0f : 1.0f / l_tot;
    const int64_t at = (int64_t)(q.q0 + row / G) * a.Hq + h * G + row % G;
    uint16_t* dst = (uint16_t*)a.out + at * D;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[ND];
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) w[dt] = pack_bf16x2(o[dt][4 * g + i] * inv, o[dt][8 + 4 * g + i] * inv);
        uint16_t* p = dst + (8 * g + 4 * hg + i) * (D / 16);
        if constexpr (D == 128) *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
        else *(uint2*)p = make_uint2(w[0], w[1]);
      }
    if (a.lse && hg == 0) a.lse[at] = (m_run + __builtin_amdgcn_logf(l_tot)) * 0.69314718055994530942f;
  } else {
    const int64_t at = ((int64_t)r * a.Hkv + h) * a.part_rows + (int64_t)c * q.rows + row;
    float* dst = a.part + at * D;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
          *(float2*)(dst + (8 * g + 4 * hg + i) * (D / 16) + 2 * dt) = make_float2(o[dt][4 * g + i], o[dt][8 + 4 * g + i]);
    if (hg == 0) a.part_ml[at] = make_float2(m_run, l_tot);
  }
}

// The parts of split requests, chunk after chunk: one wave per row.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_merge_kernel(Kv4AttnK a) {
  const int r = blockIdx.y, h = blockIdx.x % a.Hkv;
  const Request q(a, r);
  if (q.split.n == 1) return;
  const int G = a.Hq / a.Hkv, lane = threadIdx.x & 63, n = q.split.n;   // n <= 64: a chunk per lane
  for (int row = blockIdx.x / a.Hkv * 4 + (threadIdx.x >> 6); row < q.rows; row += gridDim.x / a.Hkv * 4) {
    const int64_t at = ((int64_t)r * a.Hkv + h) * a.part_rows + row;
    const float2 ml = lane < n ? a.part_ml[at + (int64_t)lane * q.rows] : make_float2(kNegInf, 0.0f);
    const float mt = wave_max(ml.x);
    const float base = mt == kNegInf ? 0.0f : mt;
    const float f = __builtin_amdgcn_exp2f(ml.x - base);
    float lt = 0.0f, acc[D / 64];
#pragma unroll
    for (int e = 0; e < D / 64; ++e) acc[e] = 0.0f;
    for (int c = 0; c < n; ++c) {
      const float fc = __shfl(f, c, 64);
      lt = __builtin_fmaf(__shfl(ml.y, c, 64), fc, lt);
      const float* src = a.part + (at + (int64_t)c * q.rows) * D + lane * (D / 64);
#pragma unroll
      for (int e = 0; e < D / 64; ++e) acc[e] = __builtin_fmaf(src[e], fc, acc[e]);
    }
    const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
    const int64_t to = (int64_t)(q.q0 + row / G) * a.Hq + h * G + row % G;
    T* dst = (T*)a.out + to * D + lane * (D / 64);
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
      if constexpr (sizeof(T) == 2) dst[e] = (uint16_t)pack_bf16x2(acc[e] * inv, 0.0f);
      else dst[e] = acc[e] * inv;
    }
    if (a.lse && lane == 0) a.lse[to] = (mt + __builtin_amdgcn_logf(lt)) * 0.69314718055994530942f;
  }
}

}  // namespace

template <typename T, int D>
static hipError_t launch_kv4(const Kv4AttnK& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.max_q * (a.Hq / a.Hkv);
  const int splits = kv4_max_chunks(a.max_seqlen);
  if constexpr (sizeof(T) == 2) {
    if (rows > kKv4FewRows) {
      const int wide = (int)((rows + kWideCols - 1) / kWideCols);
      hipLaunchKernelGGL((kv4_attn_wide_kernel<D>), dim3((unsigned)(wide * splits * a.Hkv), (unsigned)a.n_req), dim3(512), 0, s, a,
                         wide);
    }
  }
  const int64_t few = sizeof(T) == 2 && rows > kKv4FewRows ? kKv4FewRows : rows;
  const int tiles = (int)((few + 15) / 16);
  hipLaunchKernelGGL((kv4_attn_kernel<T, D, 4>), dim3((unsigned)(tiles * splits * a.Hkv), (unsigned)a.n_req), dim3(256), 0, s,
                     a, tiles);
  if (splits > 1) {
    const int64_t part = rows < kKv4PartRows ? rows : kKv4PartRows;
    const unsigned wgs = (unsigned)((part + 3) / 4 < 64 ? (part + 3) / 4 : 64);
    hipLaunchKernelGGL((kv4_merge_kernel<T, D>), dim3(wgs * a.Hkv, (unsigned)a.n_req), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_attn(const Kv4AttnK& a, int D, bool f32, hipStream_t s) {
  if (f32) return D == 128 ? launch_kv4<float, 128>(a, s) : launch_kv4<float, 64>(a, s);
  return D == 128 ? launch_kv4<uint16_t, 128>(a, s) : launch_kv4<uint16_t, 64>(a, s);
}

}  // namespace sx
