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

__device__ __forceinline__ bf16x8_t as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8_t, (u32x4_t){a, b, c, d});
}
__device__ __forceinline__ f32x4_t mfma16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
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
__global__ __launch_bounds__(NW * 64) void kv4_attn_kernel(Kv4AttnK a, int tiles, int splits) {
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
  const int c = idx % splits, tile = idx / splits, r = blockIdx.y;
  const Request q(a, r);
  const int row0 = tile * 16;
  if (row0 >= q.rows || c >= q.split.n) return;
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
  const int tiles = (int)((rows + 15) / 16), splits = kv4_max_chunks(a.max_seqlen);
  hipLaunchKernelGGL((kv4_attn_kernel<T, D, 4>), dim3((unsigned)(tiles * splits * a.Hkv), (unsigned)a.n_req), dim3(256), 0, s,
                     a, tiles, splits);
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
