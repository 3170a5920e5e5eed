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
// q: three, and q itself in three), so what is lost there is below the rounding of the output.  The kernel for many
// rows, further down, has another layout, and one part.
#include <algorithm>
#include <type_traits>

#include "sx_kv4_device.h"

namespace sx {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
constexpr float kNegInf = -__builtin_huge_valf();
// Requests of more rows per KV head than this take the kernel for many rows (bfloat16).  Measured on both, few / many:
// 80 rows over 16384 keys (2 requests of 8 heads) 36 / 40 us, 128 over 16384 (8 of 2) 43 / 44, 128 over 4096 (16 of 8)
// 80 / 89, 160 over 8192 (4 of 8) 49 / 51, 192 over 32768 (1 of 8) 55 / 54, 256 over 32768 (1 of 8) 70 / 61.
constexpr int kKv4FewRows = 128;

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

// The two bfloat16 values of w added to c.
__device__ __forceinline__ float sum_bf16x2(uint32_t w, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), (bf16x2_t){1.0f, 1.0f}, c, false);
}

// A float32 as a sum of N bfloat16 parts, each the rounding of what the others leave: part i of x[0..8).  FINITE:
// no infinities among them (otherwise one stands in the first part alone).
template <int N, bool FINITE = false>
__device__ __forceinline__ void split_parts(const float (&x)[8], bf16x8_t (&part)[N]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
  // the largest bfloat16: a finite value above it must not round to infinity
  auto first = [](float v) { return FINITE || !__builtin_isfinite(v) ? v : fminf(fmaxf(v, -0x1.fep127f), 0x1.fep127f); };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = i > 0 ? pack_bf16x2(rest[2 * e], rest[2 * e + 1]) : pack_bf16x2(first(rest[2 * e]), first(rest[2 * e + 1]));
      if (i + 1 < N) asm("" : "+v"(w[e]));   // (the halves are taken from here, not rounded once more)
    }
    part[i] = as_bf16x8(w[0], w[1], w[2], w[3]);
#pragma unroll
    for (int e = 0; e < 4 && i + 1 < N; ++e) {
      const float lo = bf16_lo(w[e]), hi = bf16_hi(w[e]);
      rest[2 * e] = FINITE || __builtin_isfinite(lo) ? rest[2 * e] - lo : 0.0f;
      rest[2 * e + 1] = FINITE || __builtin_isfinite(hi) ? rest[2 * e + 1] - hi : 0.0f;
    }
  }
}

// A lane's bytes of one block: D / 32 dwords of K (token l % 16, elements D / 4 (l / 16) ..) and of V (tokens
// 4 (l / 16) .. + 3, the column group l % 16), and their scale bytes.
template <int D>
struct Page {
  uint32_t k[D / 32], v[D / 32];
  uint32_t ks, vs;
  // byte offsets in a record; kept apart from the record's address, which is uniform: a load takes both as they are
  struct At {
    uint32_t code, ks, vs;
    __device__ __forceinline__ explicit At(uint32_t lane)
        : code(lane * (D / 8)), ks(kv4_k_scales(D) + (lane >> 4) * (D / 4) / kKv4Group * 16 + (lane & 15)),
          vs(kv4_v_scales(D) + (lane & 15) * (D / 16) / kKv4Group * 16 + 4 * (lane >> 4)) {}
    __device__ __forceinline__ void here() { asm volatile("" : "+v"(code), "+v"(ks), "+v"(vs)); }
  };
  __device__ __forceinline__ void load(const uint8_t* rec, At at) {
    if constexpr (D == 128) {
      const uint4 x = *(const uint4*)(rec + at.code), y = *(const uint4*)(rec + at.code + kv4_v_codes(D));
      k[0] = x.x; k[1] = x.y; k[2] = x.z; k[3] = x.w;
      v[0] = y.x; v[1] = y.y; v[2] = y.z; v[3] = y.w;
    } else {
      const uint2 x = *(const uint2*)(rec + at.code), y = *(const uint2*)(rec + at.code + kv4_v_codes(D));
      k[0] = x.x; k[1] = x.y;
      v[0] = y.x; v[1] = y.y;
    }
    ks = rec[at.ks];
    vs = *(const uint32_t*)(rec + at.vs);
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
  // V of the lane's four tokens, columns 2 B and 2 B + 1 of the column group
  template <int B>
  __device__ __forceinline__ void value_pair(uint32_t (&w)[4]) const {
    const float s[4] = {kv4_scale(vs & 0xff), kv4_scale(vs >> 8 & 0xff), kv4_scale(vs >> 16 & 0xff), kv4_scale(vs >> 24)};
    if constexpr (D == 128) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = kv4_pair<B>(v[i], s[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        w[i] = kv4_pair<B>(v[i / 2], s[i]);
        w[i + 1] = kv4_pair<B + 2>(v[i / 2], s[i + 1]);
      }
    }
  }
  // a NaN group's scale as 1 (its codes are zero)
  __device__ __forceinline__ void drop_bad_values() {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((vs >> (8 * i) & 0xff) == 0xff) vs = (vs & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));
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
  __device__ __forceinline__ Request(const Kv4AttnK& a, int r) : Request(a, a.cu[r], a.cu[r + 1], a.lens[r]) {}
  __device__ __forceinline__ Request(const Kv4AttnK& a, int from, int to, int keys) {
    q0 = min(max(from, 0), a.total_q);
    nq = max(min(min(to, a.total_q) - q0, a.max_q), 0);
    len = max(min(keys, a.max_keys), 0);
    rows = nq * a.G;
    off = len - nq;
    split = kv4_split(rows, len, a.Hkv, a.most16, a.most256);
  }
};

// What a workgroup does: items are (request, chunk of its keys, tile of its rows) of one KV head, numbered request by
// request, a request's tiles fastest.  The host knows bounds only, and a workgroup without an item costs its dispatch
// and its look at the lengths, so where a launch for every possible item would be large, a smaller one finds its items
// by the requests' item counts.  Every thread of the workgroup calls this; false: no such item.
template <int THREADS, typename CountF>
__device__ __forceinline__ bool find_item(const Kv4AttnK& a, uint32_t item, CountF count, int* request, uint32_t* in_request) {
  __shared__ uint32_t total[THREADS / 64];
  __shared__ int s_request;
  __shared__ uint32_t s_item;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t base = 0;
  for (int r0 = 0; r0 < a.n_req; r0 += THREADS) {
    const int r = r0 + (int)threadIdx.x;
    const uint32_t n = r < a.n_req ? count(Request(a, r)) : 0;
    uint32_t x = n;   // inclusive prefix over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    if (lane == 63) total[wave] = x;
    __syncthreads();
    uint32_t before = base, all = base;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) before += total[w];
      all += total[w];
    }
    if (item - (before + x - n) < n) {   // (unsigned: item below its first wraps)
      s_request = r;
      s_item = item - (before + x - n);
    }
    __syncthreads();
    if (item < all) {
      *request = __builtin_amdgcn_readfirstlane(s_request);
      *in_request = __builtin_amdgcn_readfirstlane(s_item);
      return true;
    }
    base = all;
  }
  return false;
}

// The kernel's first argument, read from the kernel-argument segment through a pointer the compiler cannot follow, so
// that a kernel that loops over items keeps nothing of it in registers from one to the next.
__device__ __forceinline__ Kv4AttnK item_args() {
  typedef const __attribute__((address_space(4))) char* ArgPtr;
  ArgPtr p = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const Kv4AttnK*)(const char*)p;
}

// Halves of the pairs (x: one of two keys, y: the other) as the two keys of one column: the low or high ones.
template <int ODD>
__device__ __forceinline__ uint32_t halves(uint32_t x, uint32_t y) {
  return __builtin_amdgcn_perm(y, x, ODD ? 0x07060302u : 0x05040100u);
}

// for_each<N>(f): f(integral constant 0) .. f(N - 1)
template <int N, int I = 0, typename F>
__device__ __forceinline__ void for_each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    for_each<N, I + 1>(f);
  }
}

// ---------------------------------------------------------------------------------------------
// Few query rows: one workgroup takes 16 MT rows of one KV head over one chunk of keys, its NW waves steps of
// two blocks in turn; the next step's codes are loaded while a step is computed, the block ids of 32 steps at
// once.  Writes the rows' results, or their parts where the request's keys are split.  (Adding them up in the
// workgroup that ends last saved nothing over the merge launch: 38.6 us for 34.6, 50.2 for 47.5 on the two cases
// below.)  16 rows are bound by HBM where there is work for every compute unit: 64 requests of up to 8192 keys (28 / 4
// heads, d = 128) 44.6 us with the merge, 3.6 TB/s; 256 of 1024 keys (32 / 8) 58 us, 5.0 TB/s; 256 of 8192 keys 468 us,
// 5.0 TB/s; one of 131072 keys 34.5 us, 4.1 TB/s; a plain streaming read reaches 5.5 - 6.  32 rows are bound by the
// vector ALU (two thirds of its cycles; conversions, exponentials and the parts of the probabilities): 128 requests of 5
// tokens over 4608 keys (32 / 8 heads) 205 us, 3.1 TB/s.
// ---------------------------------------------------------------------------------------------
template <typename T, int D, int MT, int NW>
__device__ __forceinline__ void few_rows_item(const Kv4AttnK& a, const Request& q, int r, int h, int tile, int c) {
  constexpr int NC = D / 32;                  // 32-element pieces of a row
  constexpr int NU = D / 16;                  // 16-column tiles of V
  constexpr int NQ = sizeof(T) == 4 ? 3 : 1;  // bfloat16 parts of a query element, and of a probability
  constexpr int NP = sizeof(T) == 4 ? 3 : 2;
  constexpr int OP = D + 4;                   // LDS row pitch
  __shared__ __attribute__((aligned(16))) float so[NW][16][OP];
  __shared__ float sm[NW][16], sl[NW][16];
  __shared__ bf16x8_t sq[MT][NC][NQ][64];     // the rows' operands, in lane order
  const int row0 = tile * 16 * MT;
  const int G = a.G;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));               // (nothing derived from it is kept from one item to the next)
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4;
  int row[MT], token[MT], lim[MT];            // this lane's rows, their tokens, and the last key each sees
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    row[t] = min(row0 + 16 * t + (lane & 15), q.rows - 1);
    token[t] = a.group.of(row[t]);
    lim[t] = q.off + token[t];
  }
  const int lim_min = q.off + a.group.of(row0), lim_max = q.off + a.group.of(min(row0 + 16 * MT - 1, q.rows - 1));
  const int k0 = c * q.split.keys;            // (c < n: below len)
  const int k1 = (int)min(min(k0 + (int64_t)q.split.keys, (int64_t)q.len), (int64_t)lim_max + 1);
  const int32_t* table = a.table + (int64_t)r * a.max_blocks;
  const uint8_t* pool = a.pool + (int64_t)h * kv4_record(D);
  const int64_t block_bytes = (int64_t)a.Hkv * kv4_record(D);

  // this wave's steps: keys k0 + 32 (wave + NW i) ..; block ids of steps 32 run .. + 31, two a step
  const int steps = k1 > k0 ? ((k1 - k0 + 31) / 32 - wave + NW - 1) / NW : 0;
  auto load_ids = [&](int run) {
    const int page = k0 / kBlock + 2 * (wave + NW * (32 * run + (lane >> 1))) + (lane & 1);
    const int id = (int64_t)page * kBlock < k1 ? table[page] : -1;
    return id < a.n_blocks ? id : -1;
  };
  int ids = load_ids(0);
  // codes of the current and the next step: the loop below names the slots in turn, since a register copy would
  // wait for its load.  Every step fetches, the last one block 0 (all its pages are missing): were the loads skipped
  // on a path, each step would have to wait for all that are under way.  (Two steps ahead were no faster: 121 us
  // for 121 for 64 requests of 8192 keys.)
  Page<D> page[2][2];
  int page_id[2][2];
  typename Page<D>::At at(lane);
  auto fetch = [&](int i, Page<D> (&pg)[2], int (&id)[2]) __attribute__((always_inline)) {
    if (i > 0 && (i & 31) == 0) ids = load_ids(i >> 5);
    at.here();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      id[j] = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + j);
      pg[j].load(pool + max(id[j], 0) * block_bytes, at);   // (a missing block: any bytes, dropped below)
    }
  };
  fetch(0, page[0], page_id[0]);

#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const T* src = (const T*)a.q + (int64_t)(q.q0 + token[t]) * a.q_ld + (h * G + row[t] - token[t] * G) * D + lg * (D / 4);
    for (int i = wave; i < NC; i += NW) {
      bf16x8_t qf[NQ];
      if constexpr (NQ == 1) {
        qf[0] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(src + i * 8));
      } else {
        float x[8];
        load8(src + i * 8, x);
        split_parts<NQ>(x, qf);
      }
#pragma unroll
      for (int p = 0; p < NQ; ++p) sq[t][i][p][lane] = qf[p];
    }
  }
  lds_barrier();
  f32x4_t o[MT][NU];
  float m[MT], l[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    m[t] = kNegInf;
    l[t] = 0.0f;
#pragma unroll
    for (int u = 0; u < NU; ++u) o[t][u] = (f32x4_t){0, 0, 0, 0};
  }

  auto step = [&](int i, Page<D> (&pg)[2], const int (&id)[2], Page<D> (&next)[2], int (&next_id)[2]) __attribute__((always_inline)) {
    const int kb = k0 + 32 * (wave + NW * i);
    fetch(i + 1, next, next_id);
    if (kb + 32 > q.len || id[0] < 0 || id[1] < 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) pg[j].drop_values_from(id[j] < 0 ? 0 : q.len - kb - 16 * j, lane);
    }
    f32x4_t sc[MT][2];
#pragma unroll
    for (int t = 0; t < MT; ++t) sc[t][0] = sc[t][1] = (f32x4_t){0, 0, 0, 0};
    int l64 = lane;
    asm volatile("" : "+v"(l64));              // (read again in every step: the registers go to more waves)
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const bf16x8_t k0f = pg[0].k_part(n), k1f = pg[1].k_part(n);
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int p = NQ - 1; p >= 0; --p) {
          const bf16x8_t qf = sq[t][n][p][l64];
          sc[t][0] = mfma16(k0f, qf, sc[t][0]);
          sc[t][1] = mfma16(k1f, qf, sc[t][1]);
        }
    }
    const bool edge = kb + 31 > lim_min;       // some row does not see every key of the step
    bf16x8_t pf[MT][NP];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      float s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = sc[t][e >> 2][e & 3];
      if (edge || id[0] < 0 || id[1] < 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (id[e >> 2] < 0 || kb + 16 * (e >> 2) + 4 * lg + (e & 3) > lim[t]) s[e] = kNegInf;
      }
      // the maximum is raised only when a probability would reach 2^24 (or is not a number): the same softmax,
      // and no maximum over the lanes in most steps.  Only for the rows that need it: another row's keys, which this one
      // may not see, leave its bits alone
      float p[8], psum;
      auto expo = [&](float neg) {
        psum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.scale, neg));
          psum += p[e];
        }
      };
      expo(-m[t]);
      if (const uint64_t high = __ballot(!(psum < 0x1p24f))) {
        const bool raise = high >> (lane & 15) & 0x0001000100010001;   // (any of the row's four lanes)
        float top = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = raise ? fmaxf(m[t], top * a.scale) : m[t];
        const float f = !raise || mn == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[t] - mn);
        l[t] *= f;
#pragma unroll
        for (int u = 0; u < NU; ++u) o[t][u] *= f;
        m[t] = mn;
        expo(mn == kNegInf ? 0.0f : -mn);
      }
      l[t] += psum;
      split_parts<NP, true>(p, pf[t]);
    }
    // a NaN group among the values of keys that some rows see and some do not: these rows get it, the others
    // nothing
    if (edge && __any(pg[0].bad_values() || pg[1].bad_values())) {
      const int grp = lg * (D / 4) / kKv4Group;   // of the output elements that this lane holds
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        float nan = 0.0f;
        for (int k = kb; k < min(kb + 32, q.len); ++k) {
          const int b = (k - kb) >> 4;
          if (id[b] >= 0 && k <= lim[t] && pool[id[b] * block_bytes + kv4_v_scales(D) + grp * 16 + (k & 15)] == 255)
            nan = __builtin_nanf("");
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) o[t][u] += nan;
      }
      pg[0].drop_bad_values();
      pg[1].drop_bad_values();
    }
    for_each<NC>([&](auto bc) {
      constexpr int B = decltype(bc)::value;
      uint32_t w0[4], w1[4];
      pg[0].template value_pair<B>(w0);
      pg[1].template value_pair<B>(w1);
      for_each<2>([&](auto odd) {
        constexpr int O = decltype(odd)::value, u = 2 * B + O;
        const bf16x8_t vf = as_bf16x8(halves<O>(w0[0], w0[1]), halves<O>(w0[2], w0[3]), halves<O>(w1[0], w1[1]),
                                      halves<O>(w1[2], w1[3]));
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int n = NP - 1; n >= 0; --n) o[t][u] = mfma16(vf, pf[t][n], o[t][u]);
      });
    });
  };
  for (int i = 0; i < steps; i += 2) {
    step(i, page[0], page_id[0], page[1], page_id[1]);
    if (i + 1 < steps) step(i + 1, page[1], page_id[1], page[0], page_id[0]);
  }

#pragma unroll
  for (int t = 0; t < MT; ++t) {
    // the waves' parts: lane l holds row l % 16, columns D / 4 (l / 16) + (D / 16) i + u
    if (t > 0) __syncthreads();
    float lw = l[t];
    lw += __shfl_xor(lw, 16, 64);
    lw += __shfl_xor(lw, 32, 64);
    float* dst = &so[wave][lane & 15][lg * (D / 4)];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < NU; u += 4)
        *(float4*)(dst + i * NU + u) = make_float4(o[t][u][i], o[t][u + 1][i], o[t][u + 2][i], o[t][u + 3][i]);
    if (lg == 0) {
      sm[wave][lane & 15] = m[t];
      sl[wave][lane & 15] = lw;
    }
    __syncthreads();
    constexpr int TPR = NW * 64 / 16;           // threads per row
    constexpr int EPT = D / TPR;                // elements per thread
    const int rr = tid / TPR, d0 = tid % TPR * EPT;
    const int orow = row0 + 16 * t + rr;
    if (orow >= q.rows) continue;
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
    if (q.split.n == 1) {
      const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
      const int otoken = a.group.of(orow);
      const int64_t at = (int64_t)(q.q0 + otoken) * a.Hq + h * G + orow - otoken * G;
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
}

template <typename T, int MT>
__device__ __forceinline__ uint32_t few_tiles(const Request& q) {   // (0: the request is not for this kernel)
  return sizeof(T) == 2 && q.rows > kKv4FewRows ? 0u : (uint32_t)(q.rows + 16 * MT - 1) / (16 * MT);
}

// A workgroup for every possible item: x = KV head, y = tile, request, z = chunk.  Chunks slowest: workgroups beyond a
// request's last chunk end at once, and between live ones they would put these on a few shader engines.
template <typename T, int D, int MT, int NW, int WAVES>
__global__ __launch_bounds__(NW * 64, WAVES) void kv4_attn_kernel(Kv4AttnK a, int tiles) {
  const int h = blockIdx.x, c = blockIdx.z;
  const uint32_t r = tiles > 1 ? blockIdx.y / (uint32_t)tiles : blockIdx.y, tile = blockIdx.y - r * tiles;
  const Request q(a, r);
  if (tile < few_tiles<T, MT>(q) && c < q.split.n) few_rows_item<T, D, MT, NW>(a, q, r, h, tile, c);
}

// Workgroups that take items in turn.  (bfloat16, two tiles of d = 128: 9 registers of a lane are spilled for a third wave a
// SIMD, as in the direct form.)
template <typename T, int D, int MT, int NW>
__global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 3 : 2) void kv4_attn_items_kernel(Kv4AttnK ka) {
  const int h = blockIdx.x % (uint32_t)ka.Hkv;
  for (uint32_t item = blockIdx.x / (uint32_t)ka.Hkv;; item += gridDim.x / (uint32_t)ka.Hkv) {
    const Kv4AttnK a = item_args();
    int r;
    uint32_t at;
    if (!find_item<NW * 64>(a, item, [&](const Request& q) { return few_tiles<T, MT>(q) * q.split.n; }, &r, &at)) return;
    const Request q(a, r);
    const uint32_t n = few_tiles<T, MT>(q);
    few_rows_item<T, D, MT, NW>(a, q, r, h, at % n, at / n);
    __syncthreads();   // (the item's LDS is free again)
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
// parts cost 1378 us where one costs 964.  A row is divided by the sum of the rounded probabilities, so a rounding
// moves its result by 2^-8 w |v - result| at the most, w the key's weight, and nothing where one key has all of it (divided
// by the exact sum: 2^-8 |v|); the exact sum, for the lse and the weights of parts, is kept beside it.  That costs 3 %
// (945 us to 972; 979 with the sum formed in the vector phase).  Sums and statistics are float32; the running maximum is
// raised only when a probability would reach 2^24.
// 2048 tokens of 32 / 8 heads over 32768 keys (d = 128): 970 us, 1.10 PFLOP/s (a plain 8192^3 bfloat16 product reaches
// 1.26); the kernel for few rows took 11.4 ms.  Deeper operand reads (2 to 8 MFMAs ahead) change nothing, without its
// softmax or its conversion the loop takes 970 and 837 us: bound by the matrix phase, whose MFMAs run at about that rate.
// ---------------------------------------------------------------------------------------------
constexpr int kWideCols = 256;
constexpr int kWideKeys = 64;

template <int D>
__device__ __forceinline__ void many_rows_item(const Kv4AttnK& a, const Request& q, int r, int h, int tile, int c) {
  constexpr int NS = D / 16;          // 16-element slices of a key
  constexpr int ND = D / 32;          // 32-column tiles of the output; dwords of codes per lane
  constexpr int TILEB = kWideKeys * D * 2;
  constexpr int NBUF = 3;
  __shared__ __attribute__((aligned(1024))) char smem[2 * NBUF * TILEB];   // [buffer][K], [buffer][V]
  __shared__ int s_nan[NBUF];         // NaN groups among the values of the buffer's tile (replaced by zero)
  const int row0 = tile * kWideCols;
  const int G = a.G;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hg = lane >> 5;
  const int wrow = row0 + wave * 32;
  const int row = min(wrow + l32, q.rows - 1);
  const bool valid = wrow + l32 < q.rows;
  const int token = a.group.of(row), lim = q.off + token;
  const int lim0 = q.off + a.group.of(row0), lim1 = q.off + a.group.of(min(row0 + kWideCols - 1, q.rows - 1));   // of the workgroup
  const int wave_min = q.off + a.group.of(min(wrow, q.rows - 1));
  const int wave_max = wrow < q.rows ? q.off + a.group.of(min(wrow + 31, q.rows - 1)) : -1;
  const int k0 = c * q.split.keys;    // (a multiple of kKv4Step = 128)
  const int k1 = (int)min(min(k0 + (int64_t)q.split.keys, (int64_t)q.len), (int64_t)lim1 + 1);
  const int nkt = k1 > k0 ? (k1 - k0 + kWideKeys - 1) / kWideKeys : 0;
  const int32_t* table = a.table + (int64_t)r * a.max_blocks;
  const float c2 = a.scale;

  bf16x8_t qb[NS];
  {
    const uint16_t* src = (const uint16_t*)a.q + (int64_t)(q.q0 + token) * a.q_ld + (h * G + row - token * G) * D + hg * 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) qb[s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(src + s * 16));
  }
  f32x16_t o[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;
  float m_run = kNegInf, l_run = 0.0f, r_run = 0.0f;   // maximum; sum of the probabilities, and of their roundings

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
        if (__any(p.bad_values())) {
          if (lane == 0) s_nan[buf] = 1;
          p.drop_bad_values();
        }
      }
      char* dst = smem + (NBUF + buf) * TILEB + sj * ND * 1024 + ((lg & 1) * 32 + tok) * 16 + (lg >> 1) * 8;
      for_each<ND>([&](auto bc) {
        constexpr int B = decltype(bc)::value;
        uint32_t w[4];
        p.template value_pair<B>(w);
        *(uint2*)(dst + B * 1024) = make_uint2(halves<0>(w[0], w[1]), halves<0>(w[2], w[3]));
        *(uint2*)(dst + B * 1024 + 256) = make_uint2(halves<1>(w[0], w[1]), halves<1>(w[2], w[3]));
      });
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
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int t = 0; t < 4; ++t) r_run = sum_bf16x2(__builtin_bit_cast(u32x4_t, pb[kk])[t], r_run);
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
    if (const uint64_t high = __ballot(!(psum < 0x1p24f))) {
      const bool raise = high >> l32 & 0x100000001;   // (for the columns that need it, either of whose lanes says so)
      float mx = sacc[0][0];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sacc[mt][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = raise ? fmaxf(m_run, mx * c2) : m_run;
      const float f = !raise || m_new == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= f;
      r_run *= f;
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

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64), r_tot = r_run + __shfl_xor(r_run, 32, 64);
  if (!valid) return;
  // columns (D / 16) cg + 2 dt + n of the lane: cg = 8 g + 4 hg + i, element e = 8 n + 4 g + i
  if (q.split.n == 1) {
    const float inv = l_tot == 0.0f ? 0.0f : 1.0f / r_tot;
    const int64_t at = (int64_t)(q.q0 + token) * a.Hq + h * G + row - token * G;
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
    const float f = l_tot == 0.0f ? 0.0f : l_tot / r_tot;   // (the merge divides by the sum of all l)
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
          *(float2*)(dst + (8 * g + 4 * hg + i) * (D / 16) + 2 * dt) = make_float2(o[dt][4 * g + i] * f, o[dt][8 + 4 * g + i] * f);
    if (hg == 0) a.part_ml[at] = make_float2(m_run, l_tot);
  }
}

// A workgroup for every possible item, or (LOOP) fewer that take items in turn.
template <int D, bool LOOP>
__global__ __launch_bounds__(512, 1) void kv4_attn_wide_kernel(Kv4AttnK ka) {
  const int h = blockIdx.x % (uint32_t)ka.Hkv;
  auto tiles_of = [](const Request& q) {
    return q.rows > kKv4FewRows ? (uint32_t)(q.rows + kWideCols - 1) / kWideCols : 0u;
  };
  auto run = [&](const Kv4AttnK& a, uint32_t item) __attribute__((always_inline)) {
    int r;
    uint32_t at;
    if (!find_item<512>(a, item, [&](const Request& q) { return tiles_of(q) * q.split.n; }, &r, &at)) return false;
    const Request q(a, r);
    const uint32_t n = tiles_of(q);
    many_rows_item<D>(a, q, r, h, n - 1 - at % n, at / n);   // later rows see more keys: first
    return true;
  };
  if constexpr (LOOP) {
    for (uint32_t item = blockIdx.x / (uint32_t)ka.Hkv; run(item_args(), item); item += gridDim.x / (uint32_t)ka.Hkv) __syncthreads();
  } else {
    run(ka, blockIdx.x / (uint32_t)ka.Hkv);
  }
}

// The parts of split requests: a wave per (token, head), up to 32 chunks' loads in flight at once (none for the runs of 8
// that there are no chunks for), or (FOUR) four waves, a workgroup, with 16 each.  The chunks c, c + 4, .. are added in
// order, then the four sums, in both.
template <typename T, int D, bool FOUR>
__global__ __launch_bounds__(256) void kv4_merge_kernel(Kv4AttnK a) {
  constexpr int E = D / 64;                  // elements per lane
  constexpr int STEP = FOUR ? 4 : 1, BATCH = FOUR ? kKv4Splits / 4 : 32, RUN = FOUR ? BATCH : 8;
  __shared__ float so[FOUR ? 4 : 1][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = FOUR ? blockIdx.y : blockIdx.y * 4 + wave;
  if (head >= a.Hq) return;
  const int h = a.group.of(head);
  for (int token = blockIdx.x; token < a.total_q; token += gridDim.x) {
    int r, q0, q1, keys;                   // the token's request
    if (a.n_req <= 64) {                     // a lane each: one round of loads
      q1 = lane < a.n_req ? a.cu[lane + 1] : INT32_MAX;
      keys = lane < a.n_req ? a.lens[lane] : 0;
      q0 = a.cu[0];
      r = __popcll(__ballot(q1 <= token));
      if (r >= a.n_req) return;              // behind the last sequence
      if (r > 0) q0 = __builtin_amdgcn_readlane(q1, r - 1);
      q1 = __builtin_amdgcn_readlane(q1, r);
      keys = __builtin_amdgcn_readlane(keys, r);
    } else {
      r = __builtin_amdgcn_readfirstlane(lower_bound_wave(a.cu + 1, a.n_req, token + 1, lane));
      if (r >= a.n_req) return;
      q0 = a.cu[r];
      q1 = a.cu[r + 1];
      keys = a.lens[r];
    }
    const Request q(a, q0, q1, keys);
    const int i = token - q.q0, n = q.split.n;
    if (n == 1) {                            // on to the next request's tokens
      if (q.nq - i > (int)gridDim.x) token += (q.nq - i - 1) / gridDim.x * gridDim.x;
      continue;
    }
    if (i < 0 || i >= q.nq) continue;
    const int64_t at = ((int64_t)r * a.Hkv + h) * a.part_rows + i * a.G + head - h * a.G;
    const float2 ml = lane < n ? a.part_ml[at + (int64_t)lane * q.rows] : make_float2(kNegInf, 0.0f);   // n <= 64: a chunk per lane
    const float* src = a.part + at * D + lane * E;
    const float mt = wave_max(ml.x);
    const float f = __builtin_amdgcn_exp2f(ml.x - (mt == kNegInf ? 0.0f : mt));
    float lt = ml.y * f;                     // (a fixed tree over the lanes)
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) lt += __shfl_xor(lt, s, 64);
    float acc[4][E];                         // (FOUR: the first of them)
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[w][e] = 0.0f;
    for (int c0 = FOUR ? wave : 0; c0 < n; c0 += BATCH * STEP) {
      float x[BATCH][E];
#pragma unroll
      for (int p0 = 0; p0 < BATCH; p0 += RUN) {
        if (c0 + p0 * STEP >= n) break;
#pragma unroll
        for (int p = p0; p < p0 + RUN; ++p)
#pragma unroll
          for (int e = 0; e < E; ++e) x[p][e] = c0 + p * STEP < n ? src[(int64_t)(c0 + p * STEP) * q.rows * D + e] : 0.0f;
      }
#pragma unroll
      for (int p0 = 0; p0 < BATCH; p0 += RUN) {
        if (c0 + p0 * STEP >= n) break;
#pragma unroll
        for (int p = p0; p < p0 + RUN; ++p) {  // (behind the last chunk: f = 2^-inf = 0)
          const float fc = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), c0 + p * STEP));
#pragma unroll
          for (int e = 0; e < E; ++e) acc[FOUR ? 0 : p & 3][e] = __builtin_fmaf(x[p][e], fc, acc[FOUR ? 0 : p & 3][e]);
        }
      }
    }
    if constexpr (FOUR) {
#pragma unroll
      for (int e = 0; e < E; ++e) so[wave][lane * E + e] = acc[0][e];
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[w][e] = so[w][lane * E + e];
      __syncthreads();
      if (wave != 0) continue;
    }
    const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
    const int64_t to = (int64_t)token * a.Hq + head;
    T* dst = (T*)a.out + to * D + lane * E;
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = ((acc[0][e] + acc[1][e]) + (acc[2][e] + acc[3][e])) * inv;
    if constexpr (E == 1) {
      if constexpr (sizeof(T) == 2) *dst = (uint16_t)pack_bf16x2(v[0], 0.0f);
      else *dst = v[0];
    } else {
      if constexpr (sizeof(T) == 2) *(uint32_t*)dst = pack_bf16x2(v[0], v[1]);
      else *(float2*)dst = make_float2(v[0], v[1]);
    }
    if (a.lse && lane == 0) a.lse[to] = (mt + __builtin_amdgcn_logf(lt)) * 0.69314718055994530942f;
  }
}

}  // namespace

// Workgroups of a launch.  64 requests of 1000 keys cost 15.6 us where the host says 1000 keys, but took 43 where it
// says 131072 and every possible chunk had a workgroup, 305 with bounds of 512 queries beside it.
constexpr int64_t kDirectGroups = 4096;   // most workgroups launched for possible items
constexpr int64_t kWaves3Groups = 1024;   // workgroups from which three waves of two tiles a SIMD pay
constexpr int64_t kFewGroups = 2048;      // ... that take items in turn: a few a compute unit
constexpr int64_t kWideDirect = 2048;     // the same of the kernel for many rows, of which one fits a compute unit
constexpr int64_t kWideGroups = 512;
constexpr int64_t kMergeGroups = 4096;

template <typename T, int D, int MT>
static void launch_few(const Kv4AttnK& a, int64_t rows, int splits, hipStream_t s) {
  const int64_t tiles = (rows + 16 * MT - 1) / (16 * MT), all = tiles * a.Hkv * a.n_req;
  if (all * splits <= kDirectGroups) {
    // waves a SIMD.  Two tiles of d = 128 take 183 registers: three cost a few spills, which pays where there is work for
    // them (64 requests of 16 tokens, 28 / 4 heads, over 4096 keys 151 us for 160), not in smaller launches (8 requests
    // of 8192 keys 20.9 us for 20.4).
    constexpr int W = sizeof(T) == 2 && MT == 1 ? 3 : 2;
    const dim3 grid((unsigned)a.Hkv, (unsigned)(tiles * a.n_req), (unsigned)splits);
    if constexpr (sizeof(T) == 2 && MT == 2 && D == 128) {
      if (all * splits >= kWaves3Groups) {
        hipLaunchKernelGGL((kv4_attn_kernel<T, D, MT, 4, 3>), grid, dim3(256), 0, s, a, (int)tiles);
        return;
      }
    }
    hipLaunchKernelGGL((kv4_attn_kernel<T, D, MT, 4, W>), grid, dim3(256), 0, s, a, (int)tiles);
    return;
  }
  // at most so many tiles by the rows of q, too
  const int64_t most = std::min(tiles * a.n_req, (int64_t)a.total_q * a.G / (16 * MT) + a.n_req) * splits;
  const int64_t items = std::max<int64_t>(1, std::min(most, kFewGroups / a.Hkv));
  hipLaunchKernelGGL((kv4_attn_items_kernel<T, D, MT, 4>), dim3((unsigned)(items * a.Hkv)), dim3(256), 0, s, a);
}

template <typename T, int D>
static hipError_t launch_kv4(const Kv4AttnK& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.max_q * a.G;
  const int splits = kv4_max_chunks(a.max_keys);
  if constexpr (sizeof(T) == 2) {
    if (rows > kKv4FewRows) {
      // a request of t tiles in n > 1 chunks has rows x heads x n <= kKv4Parts, so t n <= 2 x 256 / heads
      const int64_t requests = std::min<int64_t>(a.n_req, (int64_t)a.total_q * a.G / (kKv4FewRows + 1) + 1);
      const int64_t all_tiles = (int64_t)a.total_q * a.G / kWideCols + requests;
      const int64_t n = std::min<int64_t>(splits, kv4_most_chunks(kKv4FewRows + 1, a.Hkv));
      const int64_t most = std::min(all_tiles * n, all_tiles + requests * (2 * kKv4Parts / kWideCols / a.Hkv + 1)) * a.Hkv;
      if (most <= kWideDirect)
        hipLaunchKernelGGL((kv4_attn_wide_kernel<D, false>), dim3((unsigned)most), dim3(512), 0, s, a);
      else
        hipLaunchKernelGGL((kv4_attn_wide_kernel<D, true>), dim3((unsigned)(std::max<int64_t>(1, kWideGroups / a.Hkv) * a.Hkv)),
                           dim3(512), 0, s, a);
    }
  }
  const int64_t few = sizeof(T) == 2 ? std::min<int64_t>(rows, kKv4FewRows) : rows;
  if (few <= 16) launch_few<T, D, 1>(a, few, splits, s);
  else launch_few<T, D, 2>(a, few, splits, s);
  if (splits > 1) {
    // few rows of many chunks: four waves each (one token of 32 heads in 64 chunks: 4.5 us, 8.6 in one)
    const bool four = splits > kKv4Splits / 4 && (int64_t)a.total_q * a.Hq <= kMergeGroups / 4;
    const int64_t groups = four ? a.Hq : (a.Hq + 3) / 4;
    const int64_t tokens = std::max<int64_t>(1, std::min<int64_t>(a.total_q, kMergeGroups / groups));
    const dim3 grid((unsigned)tokens, (unsigned)groups);
    if (four) hipLaunchKernelGGL((kv4_merge_kernel<T, D, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv4_merge_kernel<T, D, false>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_attn(const Kv4AttnK& a, int D, bool f32, hipStream_t s) {
  if (f32) return D == 128 ? launch_kv4<float, 128>(a, s) : launch_kv4<float, 64>(a, s);
  return D == 128 ? launch_kv4<uint16_t, 128>(a, s) : launch_kv4<uint16_t, 64>(a, s);
}

}  // namespace sx
