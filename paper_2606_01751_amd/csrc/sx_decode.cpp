// Host side of the decoding calls (include/sx_decode.h): argument validation and dispatch.
#include "sx_decode.h"

#include <algorithm>
#include <cmath>

#include "sx_args.h"
#include "sx_kv4.h"

#ifndef SX_DEVICE_CHECKS
#define SX_DEVICE_CHECKS 0
#endif

namespace {

using sx::aligned16;
using sx::overlap;
using sx::reportf;
using sx::Rows;
using sx::rows_overlap;
using sx::whole;

constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - ((int64_t)1 << 16);   // of a one-dimensional launch
constexpr int kMaxRequests = 65535;
constexpr int kMaxSlotRequests = 65536;

int esize(const sx_layer_desc* d) { return d->dtype == SX_F32 ? 4 : 2; }

// Rows of `heads` heads each, ld elements apart.
sx_status check_rows_arg(const sx_layer_desc* d, const char* name, const void* p, int64_t ld, int heads) {
  if (!p) return reportf(SX_EINVAL, "%s is NULL", name);
  if (!aligned16(p)) return reportf(SX_EINVAL, "%s is not 16-byte aligned", name);
  if (ld < (int64_t)heads * d->head_dim || ld % 8 != 0 || ld > ((int64_t)1 << 40))
    return reportf(SX_ESHAPE, "%s: %lld elements between rows (a multiple of 8, at least %d heads x %d)", name,
                   (long long)ld, heads, d->head_dim);
  return SX_OK;
}

const char* kWhat[] = {"", "", "", "", "cu_q[0] is not 0", "a request's query tokens are negative or above max_q",
                       "a length is negative or out of range", "an index is out of range",
                       "a block table entry is below -1 or out of range", "cu_q ends behind total_q"};

sx_status verdict_status(hipError_t e, const int v[4], const char* who) {
  if (e != hipSuccess) return reportf(SX_EHIP, "%s: device check: %s", who, hipGetErrorString(e));
  if (v[0] != 0)
    return reportf(SX_EDEVICE, "%s: %s (request %d, entry %d, value %d)", who, kWhat[v[0] < 10 ? v[0] : 0], v[1], v[2], v[3]);
  return SX_OK;
}

sx_status index_ok(const int32_t* idx, int32_t n, int64_t limit, void* stream, const char* who, int32_t low = -1) {
  if (!SX_DEVICE_CHECKS || n == 0) return SX_OK;
  int v[4] = {0, 0, 0, 0};
  const hipError_t e = sx::device_check_index(idx, n, low, limit, (hipStream_t)stream, v);
  return verdict_status(e, v, who);
}

sx_status check_pool(const void* pool, int64_t n_blocks) {
  if (!pool) return reportf(SX_EINVAL, "pool is NULL");
  if (!aligned16(pool)) return reportf(SX_EINVAL, "pool is not 16-byte aligned");
  // (slots are int32)
  if (n_blocks < 1 || n_blocks > INT32_MAX / sx::kBlock)
    return reportf(SX_ESHAPE, "n_blocks %lld outside 1 .. %d", (long long)n_blocks, INT32_MAX / sx::kBlock);
  return SX_OK;
}

sx_status check_move(const sx_layer_desc* d, const void* pool, int64_t n_blocks, const int32_t* idx, int32_t n, bool blocks,
                     const char* who) {
  sx_status st = sx::check_desc(d);
  if (st != SX_OK) return st;
  if ((st = check_pool(pool, n_blocks)) != SX_OK) return st;
  if (n < 0) return reportf(SX_EINVAL, "%s: negative count %d", who, n);
  if (n == 0) return SX_OK;
  if (!idx) return reportf(SX_EINVAL, "%s: index array is NULL", who);
  const int64_t tiles = blocks ? n : ((int64_t)n + sx::kBlock - 1) / sx::kBlock;
  if (n > INT32_MAX - sx::kBlock || tiles * d->n_kv_heads * 64 >= kMaxThreads)
    return reportf(SX_EUNSUPPORTED, "%s: %d rows or blocks x %d heads exceed one launch", who, n, d->n_kv_heads);
  return SX_OK;
}

Rows pool_blocks(const sx_layer_desc* d, const void* pool, int64_t n_blocks) {
  const int64_t block = (int64_t)d->n_kv_heads * sx::kv4_record(d->head_dim);
  return {pool, n_blocks, block, block};
}

// What a move writes (the pool, or k and v) must not overlap anything else of the call.
sx_status check_apart(Rows k, Rows v, Rows pool, Rows idx, Rows idx2, bool write, const char* who) {
  if (write ? rows_overlap(pool, k) || rows_overlap(pool, v) || rows_overlap(pool, idx) || rows_overlap(pool, idx2)
            : rows_overlap(k, v) || rows_overlap(k, pool) || rows_overlap(v, pool) || rows_overlap(k, idx) || rows_overlap(v, idx) ||
                  rows_overlap(k, idx2) || rows_overlap(v, idx2))
    return reportf(SX_EINVAL, "%s: an output overlaps another argument", who);
  return SX_OK;
}

sx_status move_rows(const sx_layer_desc* d, const void* k, int64_t k_ld, const void* v, int64_t v_ld, const int32_t* slots,
                    int32_t n, const void* pool, int64_t n_blocks, bool write, void* stream, const char* who) {
  sx_status st = check_move(d, pool, n_blocks, slots, n, false, who);
  if (st != SX_OK || n == 0) return st;
  if ((st = check_rows_arg(d, "k", k, k_ld, d->n_kv_heads)) != SX_OK) return st;
  if ((st = check_rows_arg(d, "v", v, v_ld, d->n_kv_heads)) != SX_OK) return st;
  if ((st = index_ok(slots, n, n_blocks * sx::kBlock, stream, who)) != SX_OK) return st;
  const int64_t es = esize(d), width = d->n_kv_heads * d->head_dim * es;
  if ((st = check_apart({k, n, width, k_ld * es}, {v, n, width, v_ld * es}, pool_blocks(d, pool, n_blocks), whole(slots, 4ll * n),
                        whole(nullptr, 0), write, who)) != SX_OK)
    return st;
  sx::Kv4MoveK a{};
  a.k = const_cast<void*>(k);
  a.v = const_cast<void*>(v);
  a.k_ld = k_ld;
  a.v_ld = v_ld;
  a.idx = slots;
  a.pool = (uint8_t*)const_cast<void*>(pool);
  a.n_blocks = n_blocks;
  a.n = n;
  a.Hkv = d->n_kv_heads;
  const bool f32 = d->dtype == SX_F32;
  return sx::launch_status(write ? sx::launch_kv4_write(a, d->head_dim, f32, false, (hipStream_t)stream)
                                 : sx::launch_kv4_read(a, d->head_dim, f32, false, (hipStream_t)stream), who);
}

sx_status move_blocks(const sx_layer_desc* d, const void* kc, const void* vc, int64_t n_cache_blocks, const int32_t* cb,
                      int32_t n, const void* pool, int64_t n_blocks, const int32_t* pb, bool write, void* stream,
                      const char* who) {
  sx_status st = check_move(d, pool, n_blocks, pb, n, true, who);
  if (st != SX_OK || n == 0) return st;
  if (!kc || !vc || !cb) return reportf(SX_EINVAL, "%s: NULL argument", who);
  if (!aligned16(kc) || !aligned16(vc)) return reportf(SX_EINVAL, "%s: the cache is not 16-byte aligned", who);
  if (n_cache_blocks < 1 || n_cache_blocks > INT32_MAX) return reportf(SX_ESHAPE, "%s: n_cache_blocks %lld", who, (long long)n_cache_blocks);
  if ((st = index_ok(pb, n, n_blocks, stream, who)) != SX_OK) return st;
  if ((st = index_ok(cb, n, n_cache_blocks, stream, who)) != SX_OK) return st;
  const int64_t block = (int64_t)d->n_kv_heads * sx::kBlock * d->head_dim * esize(d);
  if ((st = check_apart({kc, n_cache_blocks, block, block}, {vc, n_cache_blocks, block, block}, pool_blocks(d, pool, n_blocks),
                        whole(pb, 4ll * n), whole(cb, 4ll * n), write, who)) != SX_OK)
    return st;
  sx::Kv4MoveK a{};
  a.k = const_cast<void*>(kc);
  a.v = const_cast<void*>(vc);
  a.idx = pb;
  a.cache_blocks = cb;
  a.pool = (uint8_t*)const_cast<void*>(pool);
  a.n_blocks = n_blocks;
  a.n_cache_blocks = n_cache_blocks;
  a.n = n;
  a.Hkv = d->n_kv_heads;
  const bool f32 = d->dtype == SX_F32;
  return sx::launch_status(write ? sx::launch_kv4_write(a, d->head_dim, f32, true, (hipStream_t)stream)
                                 : sx::launch_kv4_read(a, d->head_dim, f32, true, (hipStream_t)stream), who);
}

// RoPE frequencies base^(-2i/d), the last (base, d) of the thread kept: 64 powers cost more than a launch.
const double* frequencies(double base, int d) {
  thread_local double table[64];
  thread_local double of_base = 0.0;
  thread_local int of_d = 0;
  if (of_base != base || of_d != d) {
    for (int i = 0; i < d / 2; ++i) table[i] = std::pow(base, -2.0 * i / d);
    of_base = base;
    of_d = d;
  }
  return table;
}

sx_status check_norm(const sx_layer_desc* d, const void* gamma_q, const void* gamma_k, float eps) {
  // (the kernel's cos and sin hold for angles below 2^52; frequencies are at most 1 / base, positions below 2^31)
  if (d->rope_base < 0x1p-20) return reportf(SX_EUNSUPPORTED, "rope_base %g below 2^-20", d->rope_base);
  if (!aligned16(gamma_q) || !aligned16(gamma_k)) return reportf(SX_EINVAL, "gamma is not 16-byte aligned");
  if ((gamma_q || gamma_k) && (!(eps > 0.0f) || !std::isfinite(eps))) return reportf(SX_EINVAL, "eps must be finite and > 0");
  return SX_OK;
}

int64_t workspace_of(const sx_layer_desc* d, int32_t n_requests, int32_t max_q, int32_t max_seqlen, int64_t* part_rows) {
  const int64_t rows = sx::kv4_part_rows((int64_t)max_q * (d->n_q_heads / d->n_kv_heads), max_seqlen, d->n_kv_heads);
  *part_rows = rows;
  return (int64_t)n_requests * d->n_kv_heads * rows * (d->head_dim * 4 + 8);
}

}  // namespace

extern "C" {

sx_status sx_append_slots(const int32_t* ctx_lens, const int32_t* new_lens, int32_t n_requests, int32_t block_size,
                          const int32_t* free_blocks, int32_t n_free, const int32_t* free_head, int32_t* block_table,
                          int32_t max_blocks, int32_t max_tokens, int32_t* seq_lens, int32_t* cu_new,
                          int32_t* positions, int32_t* slots, int32_t* state, void* stream) {
  if (!ctx_lens || !block_table || !seq_lens || !cu_new || !state || (max_tokens > 0 && (!positions || !slots)))
    return reportf(SX_EINVAL, "sx_append_slots: NULL argument");
  if (n_free < 0 || (n_free > 0 && !free_blocks)) return reportf(SX_EINVAL, "sx_append_slots: bad free list");
  if (n_requests < 1 || block_size < 1 || max_blocks < 1 || max_tokens < 0)
    return reportf(SX_EINVAL, "sx_append_slots: n_requests, block_size and max_blocks must be >= 1, max_tokens >= 0");
  if (n_requests > kMaxSlotRequests)
    return reportf(SX_EUNSUPPORTED, "sx_append_slots: more than %d requests", kMaxSlotRequests);
  if (max_tokens > (1 << 30)) return reportf(SX_EUNSUPPORTED, "sx_append_slots: max_tokens above 2^30");
  const struct {
    const void* p;
    int64_t bytes;
  } arr[] = {{ctx_lens, 4ll * n_requests}, {new_lens, 4ll * n_requests}, {free_blocks, 4ll * n_free}, {free_head, 4},
             {block_table, 4ll * n_requests * max_blocks}, {seq_lens, 4ll * n_requests}, {cu_new, 4ll * (n_requests + 1ll)},
             {positions, 4ll * max_tokens}, {slots, 4ll * max_tokens}, {state, 8}};
  for (int i = 4; i < 10; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(arr[i].p, arr[i].bytes, arr[j].p, arr[j].bytes))
        return reportf(SX_EINVAL, "sx_append_slots: an output overlaps another argument");
  if (SX_DEVICE_CHECKS) {
    int v[4] = {0, 0, 0, 0};
    hipError_t e = sx::device_check_lengths(ctx_lens, new_lens, n_requests, (hipStream_t)stream, v);
    sx_status st = verdict_status(e, v, "sx_append_slots");
    if (st != SX_OK) return st;
    if ((st = index_ok(free_blocks, n_free, (int64_t)INT32_MAX / block_size, stream, "sx_append_slots", 0)) != SX_OK) return st;
  }
  sx::AppendSlotsK a{};
  a.ctx = ctx_lens;
  a.add = new_lens;
  a.free_blocks = free_blocks;
  a.free_head = free_head;
  a.table = block_table;
  a.seq = seq_lens;
  a.cu = cu_new;
  a.pos = positions;
  a.slots = slots;
  a.state = state;
  a.n_req = n_requests;
  a.block = block_size;
  a.n_free = n_free;
  a.max_blocks = max_blocks;
  a.max_tokens = max_tokens;
  return sx::launch_status(sx::launch_append_slots(a, (hipStream_t)stream), "sx_append_slots launch");
}

sx_status sx_qk_norm_rope(const sx_layer_desc* desc, const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                          const void* gamma_q, const void* gamma_k, float eps, const int32_t* positions,
                          int32_t n_tokens, void* q_out, int64_t q_out_ld, void* k_out, int64_t k_out_ld,
                          void* stream) {
  sx_status st = sx::check_desc(desc);
  if (st != SX_OK) return st;
  if (n_tokens < 0) return reportf(SX_EINVAL, "n_tokens must be >= 0");
  if (n_tokens == 0) return SX_OK;
  // (a workgroup of 256 threads takes 512 / head_dim tokens)
  if ((int64_t)n_tokens * (desc->head_dim / 2) >= kMaxThreads) return reportf(SX_EUNSUPPORTED, "%d tokens exceed one launch", n_tokens);
  if ((st = check_rows_arg(desc, "q", q, q_ld, desc->n_q_heads)) != SX_OK) return st;
  if ((st = check_rows_arg(desc, "k", k, k_ld, desc->n_kv_heads)) != SX_OK) return st;
  if ((st = check_rows_arg(desc, "q_out", q_out, q_out_ld, desc->n_q_heads)) != SX_OK) return st;
  if ((st = check_rows_arg(desc, "k_out", k_out, k_out_ld, desc->n_kv_heads)) != SX_OK) return st;
  if ((st = check_norm(desc, gamma_q, gamma_k, eps)) != SX_OK) return st;
  if (!positions) return reportf(SX_EINVAL, "positions is NULL");
  if ((q_out == q && q_out_ld != q_ld) || (k_out == k && k_out_ld != k_ld))
    return reportf(SX_EINVAL, "in place, the rows must be as far apart in the output as in the input");
  const int64_t es = esize(desc), head = desc->head_dim * es;
  const Rows in[] = {{q, n_tokens, desc->n_q_heads * head, q_ld * es}, {k, n_tokens, desc->n_kv_heads * head, k_ld * es},
                     whole(gamma_q, head), whole(gamma_k, head), whole(positions, 4ll * n_tokens)};
  const Rows to[] = {{q_out, n_tokens, in[0].width, q_out_ld * es}, {k_out, n_tokens, in[1].width, k_out_ld * es}};
  if (rows_overlap(to[0], to[1])) return reportf(SX_EINVAL, "q_out and k_out overlap");
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 5; ++i)
      if (!(i == o && to[o].p == in[i].p) && rows_overlap(to[o], in[i]))
        return reportf(SX_EINVAL, "%s overlaps another argument (it may be %s itself)", o ? "k_out" : "q_out", o ? "k" : "q");
  sx::QkNormRopeK a{};
  a.q = q;
  a.k = k;
  a.qo = q_out;
  a.ko = k_out;
  a.q_ld = q_ld;
  a.k_ld = k_ld;
  a.qo_ld = q_out_ld;
  a.ko_ld = k_out_ld;
  a.gq = gamma_q;
  a.gk = gamma_k;
  a.eps = eps;
  a.n = n_tokens;
  a.Hq = desc->n_q_heads;
  a.Hkv = desc->n_kv_heads;
  a.pos = positions;
  const double* th = frequencies(desc->rope_base, desc->head_dim);
  for (int i = 0; i < desc->head_dim / 2; ++i) a.theta[i] = th[i];
  return sx::launch_status(sx::launch_qk_norm_rope(a, desc->head_dim, desc->dtype == SX_F32,
                                                   desc->rope_style == SX_ROPE_NEOX, (hipStream_t)stream),
                           "sx_qk_norm_rope launch");
}

sx_status sx_qk_norm_rope_rows(const sx_plan* p, const int32_t* rows, const int32_t* n_rows, int32_t max_rows, void* q,
                               void* k, const void* gamma_q, const void* gamma_k, float eps, void* stream) {
  if (!p) return reportf(SX_EINVAL, "plan is NULL");
  if (!rows || !n_rows) return reportf(SX_EINVAL, "NULL row list");
  if (!q || !k) return reportf(SX_EINVAL, "NULL tensor argument");
  if (!aligned16(q) || !aligned16(k)) return reportf(SX_EINVAL, "q or k is not 16-byte aligned");
  if (max_rows < 0) return reportf(SX_EINVAL, "max_rows must be >= 0");
  if (max_rows > p->max_T) return reportf(SX_ESHAPE, "max_rows %d exceeds the longest request (%d)", max_rows, p->max_T);
  sx_status st = check_norm(&p->desc, gamma_q, gamma_k, eps);
  if (st != SX_OK) return st;
  if (max_rows == 0) return SX_OK;
  if ((st = sx::check_row_list(p, rows, n_rows, max_rows, stream, "sx_qk_norm_rope_rows")) != SX_OK) return st;
  const sx_layer_desc& d = p->desc;
  const int64_t head = d.head_dim * esize(&d);
  const Rows arr[] = {whole(q, p->total * d.n_q_heads * head), whole(k, p->total * d.n_kv_heads * head), whole(gamma_q, head),
                      whole(gamma_k, head), whole(rows, 4 * p->total), whole(n_rows, 4ll * p->n_req)};
  for (int o = 0; o < 2; ++o)
    for (int i = o + 1; i < 6; ++i)
      if (rows_overlap(arr[o], arr[i])) return reportf(SX_EINVAL, "%s overlaps another argument", o ? "k" : "q");
  sx::QkNormRopeK a{};
  a.q = a.qo = q;
  a.k = a.ko = k;
  a.q_ld = a.qo_ld = (int64_t)d.n_q_heads * d.head_dim;
  a.k_ld = a.ko_ld = (int64_t)d.n_kv_heads * d.head_dim;
  a.gq = gamma_q;
  a.gk = gamma_k;
  a.eps = eps;
  a.Hq = d.n_q_heads;
  a.Hkv = d.n_kv_heads;
  a.reqs = p->d_req;
  a.rows = rows;
  a.n_rows = n_rows;
  a.tok_pos = p->d_tok_pos;
  a.d_theta = p->d_theta;
  a.max_rows = max_rows;
  a.n_req = p->n_req;
  return sx::launch_status(sx::launch_qk_norm_rope(a, d.head_dim, d.dtype == SX_F32, d.rope_style == SX_ROPE_NEOX,
                                                   (hipStream_t)stream),
                           "sx_qk_norm_rope_rows launch");
}

sx_status sx_kv4_record_bytes(const sx_layer_desc* desc, int64_t* bytes) {
  sx_status st = sx::check_desc(desc);
  if (st != SX_OK) return st;
  if (!bytes) return reportf(SX_EINVAL, "bytes is NULL");
  *bytes = sx::kv4_record(desc->head_dim);
  return SX_OK;
}

sx_status sx_kv4_write(const sx_layer_desc* desc, const void* k, int64_t k_ld, const void* v, int64_t v_ld,
                       const int32_t* slots, int32_t n_tokens, void* pool, int64_t n_blocks, void* stream) {
  return move_rows(desc, k, k_ld, v, v_ld, slots, n_tokens, pool, n_blocks, true, stream, "sx_kv4_write");
}

sx_status sx_kv4_read(const sx_layer_desc* desc, const void* pool, int64_t n_blocks, const int32_t* slots,
                      int32_t n_tokens, void* k, int64_t k_ld, void* v, int64_t v_ld, void* stream) {
  return move_rows(desc, k, k_ld, v, v_ld, slots, n_tokens, pool, n_blocks, false, stream, "sx_kv4_read");
}

sx_status sx_kv4_pack(const sx_layer_desc* desc, const void* k_cache, const void* v_cache, int64_t n_cache_blocks,
                      const int32_t* cache_blocks, int32_t n, void* pool, int64_t n_blocks,
                      const int32_t* pool_blocks, void* stream) {
  return move_blocks(desc, k_cache, v_cache, n_cache_blocks, cache_blocks, n, pool, n_blocks, pool_blocks, true, stream,
                     "sx_kv4_pack");
}

sx_status sx_kv4_unpack(const sx_layer_desc* desc, const void* pool, int64_t n_blocks, const int32_t* pool_blocks,
                        int32_t n, void* k_cache, void* v_cache, int64_t n_cache_blocks, const int32_t* cache_blocks,
                        void* stream) {
  return move_blocks(desc, k_cache, v_cache, n_cache_blocks, cache_blocks, n, pool, n_blocks, pool_blocks, false, stream,
                     "sx_kv4_unpack");
}

sx_status sx_kv4_attn_workspace(const sx_layer_desc* desc, int32_t n_requests, int32_t max_q, int32_t max_seqlen,
                                int64_t* bytes) {
  sx_status st = sx::check_desc(desc);
  if (st != SX_OK) return st;
  if (!bytes) return reportf(SX_EINVAL, "bytes is NULL");
  if (n_requests < 0 || max_q < 0 || max_seqlen < 0) return reportf(SX_EINVAL, "negative size");
  int64_t rows;
  *bytes = workspace_of(desc, n_requests, max_q, max_seqlen, &rows);
  return SX_OK;
}

sx_status sx_kv4_attn(const sx_layer_desc* desc, const void* q, int64_t q_ld, const int32_t* cu_q,
                      const int32_t* seq_lens, const int32_t* block_table, int32_t max_blocks, int32_t n_requests,
                      int32_t total_q, int32_t max_q, int32_t max_seqlen, const void* pool, int64_t n_blocks, void* out,
                      float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  sx_status st = sx::check_desc(desc);
  if (st != SX_OK) return st;
  if (n_requests < 0 || total_q < 0 || max_q < 0 || max_seqlen < 0 || max_blocks < 0)
    return reportf(SX_EINVAL, "sx_kv4_attn: negative size");
  if (n_requests == 0 || total_q == 0 || max_q == 0) return SX_OK;
  if ((st = check_rows_arg(desc, "q", q, q_ld, desc->n_q_heads)) != SX_OK) return st;
  if ((st = check_pool(pool, n_blocks)) != SX_OK) return st;
  if (!cu_q || !seq_lens || (max_blocks > 0 && !block_table) || !out) return reportf(SX_EINVAL, "sx_kv4_attn: NULL argument");
  if (!aligned16(out)) return reportf(SX_EINVAL, "out is not 16-byte aligned");
  const int64_t G = desc->n_q_heads / desc->n_kv_heads;
  if (max_q > total_q) max_q = total_q;
  if ((int64_t)max_q * G >= ((int64_t)1 << 30)) return reportf(SX_EUNSUPPORTED, "sx_kv4_attn: max_q %d too large", max_q);
  if (max_seqlen > ((int64_t)1 << 30)) return reportf(SX_EUNSUPPORTED, "sx_kv4_attn: max_seqlen above 2^30");
  if (n_requests > kMaxRequests) return reportf(SX_EUNSUPPORTED, "sx_kv4_attn: more than %d requests", kMaxRequests);
  int64_t part_rows;
  const int64_t need = workspace_of(desc, n_requests, max_q, max_seqlen, &part_rows);
  if (need > 0 && !workspace) return reportf(SX_EINVAL, "workspace is NULL");
  if (workspace_bytes < need)
    return reportf(SX_ESHAPE, "sx_kv4_attn needs %lld bytes of workspace, got %lld", (long long)need, (long long)workspace_bytes);
  if (!aligned16(workspace)) return reportf(SX_EINVAL, "workspace is not 16-byte aligned");
  // (a workgroup reads the rows of q that it writes before it writes them, and no other reads them: out may be q)
  const int64_t es = esize(desc), width = desc->n_q_heads * desc->head_dim * es, floats = 4ll * desc->n_q_heads;
  const Rows arr[] = {{out, total_q, width, width}, {lse, total_q, floats, floats}, whole(workspace, need),
                      {q, total_q, width, q_ld * es}, whole(cu_q, 4ll * (n_requests + 1ll)), whole(seq_lens, 4ll * n_requests),
                      whole(block_table, 4ll * n_requests * max_blocks), pool_blocks(desc, pool, n_blocks)};
  const char* const names[] = {"out", "lse", "workspace"};
  for (int o = 0; o < 3; ++o)
    for (int i = o + 1; i < 8; ++i)
      if (!(o == 0 && i == 3 && out == q && q_ld * es == width) && rows_overlap(arr[o], arr[i]))
        return reportf(SX_EINVAL, "sx_kv4_attn: %s overlaps another argument (out may be q itself, with contiguous rows)", names[o]);
  sx::Kv4AttnK a{};
  a.q = q;
  a.q_ld = q_ld;
  a.cu = cu_q;
  a.lens = seq_lens;
  a.table = block_table;
  a.pool = (const uint8_t*)pool;
  a.out = out;
  a.lse = lse;
  a.part = (float*)workspace;
  a.part_ml = (float2*)((char*)workspace + (int64_t)n_requests * desc->n_kv_heads * part_rows * desc->head_dim * 4);
  a.n_blocks = n_blocks;
  a.part_rows = part_rows;
  a.max_blocks = max_blocks;
  a.n_req = n_requests;
  a.total_q = total_q;
  a.max_q = max_q;
  a.max_keys = (int)std::min<int64_t>(max_seqlen, (int64_t)max_blocks * sx::kBlock);
  a.Hq = desc->n_q_heads;
  a.Hkv = desc->n_kv_heads;
  a.G = (int)G;
  a.most16 = (int)sx::kv4_most_chunks(16, (uint32_t)a.Hkv);
  a.most256 = (int)sx::kv4_most_chunks(256, (uint32_t)a.Hkv);
  a.group = sx::kv4_heads((uint32_t)a.G);
  a.scale = (float)((double)sx::softmax_scale(desc) * 1.4426950408889634074);
  if (SX_DEVICE_CHECKS) {
    int v[4] = {0, 0, 0, 0};
    const hipError_t e = sx::device_check_kv4(a, (hipStream_t)stream, v);
    if ((st = verdict_status(e, v, "sx_kv4_attn")) != SX_OK) return st;
  }
  return sx::launch_status(sx::launch_kv4_attn(a, desc->head_dim, desc->dtype == SX_F32, (hipStream_t)stream),
                           "sx_kv4_attn launch");
}

}  // extern "C"
