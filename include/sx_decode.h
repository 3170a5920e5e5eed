/* libsx decoding over a KV cache held in 4 bits: what a serving loop runs after the prefill of
 * include/sx.h.  One step of a layer, in this order:
 *
 *   sx_append_slots    block tables and slot maps of the tokens that every request appends (once per
 *                      step, for all layers)
 *   sx_qk_norm_rope    per-head RMSNorm of the fresh queries and keys and their rotation to the tokens'
 *                      positions, in one pass (sx_qk_norm_rope_rows: the same on a plan's row list,
 *                      beside sx_rope_rows)
 *   sx_kv4_write       the fresh keys and values into their slots, rounded to 4 bits (sx_kv4_read: back)
 *   sx_kv4_attn        attention of every request's last tokens over its 4-bit blocks
 *
 * and once per request, after its prefill, sx_kv4_pack: the blocks of its paged cache into 4-bit
 * blocks (sx_kv4_unpack: back, so that resident 4-bit blocks serve as sources of sx_rope_realign).
 *
 * Status, streams, memory ownership, dtypes and sx_last_error are as in include/sx.h: no call
 * allocates, synchronises the host, aborts or throws, every tensor is caller-owned DEVICE memory on
 * the current device, and desc.dtype is the type of q, k, v, gamma and out.  No call needs a plan but
 * sx_qk_norm_rope_rows, and none keeps anything between calls but the host thread's last table of RoPE
 * frequencies, which is a function of rope_base and head_dim: calls may run at the same time on any
 * streams when their outputs and workspaces differ, and any of them can be captured into a graph.
 * Index arrays in device memory are trusted to hold sensible lengths by the release library, but an
 * entry that is out of range is left out and never followed: the checked library (libsx_checked.so)
 * refuses it with SX_EDEVICE, which cannot be done while the stream is captured.
 *
 * The 4-bit pool is one array of bytes [n_blocks][Hkv][sx_kv4_record_bytes], 16-byte aligned.  A block
 * holds 16 tokens; slot s is token s % 16 of block s / 16.  32 consecutive elements of a row share a
 * power of two 2^e: the smallest with amax <= 7 * 2^e, -126 <= e <= 125, so no element is off by more
 * than half of the widest step.  An element is its sign and the nearest of {0, 0.5, 1, 1.5, 2, 3, 4, 6}
 * times 2^e (OCP e2m1), ties to the even code, saturating at 6 * 2^125.  A group with a NaN or an
 * infinity reads back as NaN in all its 32 elements; the rest of the row is not touched by it.  A
 * record, with d = head_dim:
 *   K codes   [4][16 tokens][d/8 bytes]                    two elements a byte, the even one low
 *   V codes   [4][16 column groups][4 tokens][d/32 bytes]
 *   K scales  [d / 32][16 tokens]                               bytes e + 127; 255 for a NaN group
 *   V scales  [d / 32][16 tokens]
 * (the order in which the attention's matrix instructions take them: a lane's operands are 16, or 8,
 * consecutive bytes).
 *
 * Results: a call gives the same bits every time, and a request's (or row's) results do not depend on
 * the other requests of the call, nor on how loose max_q and max_seqlen are.
 */
#ifndef SX_DECODE_H
#define SX_DECODE_H

#include "sx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Appends new_lens[r] tokens to every request r, which holds ctx_lens[r] tokens in the blocks
 * block_table[r][0 .. ceil(ctx_lens[r] / block_size)).  Missing blocks are taken from free_blocks in
 * request order, starting at entry *free_head.
 *   ctx_lens     [n_requests] int32
 *   new_lens     [n_requests] int32, or NULL: one token each.  Negative lengths count as 0.
 *   free_blocks  [n_free] int32, free_head [1] int32 or NULL (0)
 *   block_table  [n_requests][max_blocks] int32, in and out: entries of blocks that open are written
 *                (-1 if the list is used up), all others left as they are
 *   max_tokens   room of positions and slots
 * Outputs (int32):
 *   seq_lens     [n_requests] ctx + new
 *   cu_new       [n_requests + 1] prefix sums of the new tokens: the rows of request r's new tokens
 *   positions    [max_tokens] token index of every new token in its request; -1 behind the last one
 *   slots        [max_tokens] block * block_size + offset; -1 behind the last one, and for a token
 *                that has no block (list used up, table too narrow, a negative entry of table or list)
 *                or whose slot int32 does not hold
 *   state        [2] the free list's next entry, and the number of new tokens that got no slot (0: all
 *                is well; tokens that do not fit into max_tokens count, their blocks are taken and entered
 *                in block_table all the same)
 * A later step passes state as its free_head.  Outputs must not overlap the inputs or each other
 * (SX_EINVAL), so a loop in a graph copies seq_lens and state back before its next step.
 * One launch.  1 <= n_requests <= 65536 (an empty batch is refused), block_size >= 1. */
sx_status sx_append_slots(const int32_t* ctx_lens, const int32_t* new_lens, int32_t n_requests, int32_t block_size,
                          const int32_t* free_blocks, int32_t n_free, const int32_t* free_head, int32_t* block_table,
                          int32_t max_blocks, int32_t max_tokens, int32_t* seq_lens, int32_t* cu_new,
                          int32_t* positions, int32_t* slots, int32_t* state, void* stream);

/* Per-head RMSNorm and RoPE of n_tokens rows: for every head x of q [n_tokens][Hq][d] and k
 * [n_tokens][Hkv][d],
 *   y = x / sqrt(mean x^2 + eps) * gamma        (gamma_q or gamma_k [d]; NULL: y = x, eps not read)
 *   out = y rotated to positions[row]           (pairs and frequencies as in sx_rope_realign)
 * in float32 with one rounding at the end; angle and cos / sin in float64, rounded to float32 (rope_base of at
 * least 2^-20, SX_EUNSUPPORTED below).
 * positions [n_tokens] int32: a row with a negative position is neither computed nor written.
 * Rows are contiguous, ld elements apart (a multiple of 8, at least heads * d: the parts of a stacked
 * projection).  q_out, k_out may be q, k themselves with the same ld; otherwise their rows must not overlap
 * each other or another argument (SX_EINVAL).  Tensors are 16-byte aligned. */
sx_status sx_qk_norm_rope(const sx_layer_desc* desc, const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                          const void* gamma_q, const void* gamma_k, float eps, const int32_t* positions,
                          int32_t n_tokens, void* q_out, int64_t q_out_ld, void* k_out, int64_t k_out_ld,
                          void* stream);

/* The same for the listed rows of a plan, in place, each at its position in the new sequence
 * (new_pos of its segment + offset), as sx_rope_rows does without the norm: q [sum T][Hq][d],
 * k [sum T][Hkv][d], addressed by token; rows not listed are left alone, listed rows beyond their request
 * left out.  q and k must not overlap each other or another argument.  float32 and bfloat16. */
sx_status sx_qk_norm_rope_rows(const sx_plan* plan, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                               void* q, void* k, const void* gamma_q, const void* gamma_k, float eps, void* stream);

/* Bytes of one KV head of one block in the 4-bit pool: 17 * head_dim (2176 or 1088). */
sx_status sx_kv4_record_bytes(const sx_layer_desc* desc, int64_t* bytes);

/* The four moves below: what a call writes must not overlap its other arguments (SX_EINVAL). */

/* Rounds rows k, v [n_tokens][Hkv][d] (rows ld elements apart as above) to 4 bits into slots[i] of the
 * pool; a row whose slot is negative (or beyond the pool) is skipped.  The slots of one call are
 * distinct.  Nothing else in the pool is written. */
sx_status sx_kv4_write(const sx_layer_desc* desc, const void* k, int64_t k_ld, const void* v, int64_t v_ld,
                       const int32_t* slots, int32_t n_tokens, void* pool, int64_t n_blocks, void* stream);

/* The rows that slots[i] hold, exactly (every 4-bit value is a bfloat16 value): k, v [n_tokens][Hkv][d];
 * rows whose slot is negative (or beyond the pool) are left as they were. */
sx_status sx_kv4_read(const sx_layer_desc* desc, const void* pool, int64_t n_blocks, const int32_t* slots,
                      int32_t n_tokens, void* k, int64_t k_ld, void* v, int64_t v_ld, void* stream);

/* Rounds whole blocks of a paged cache ([n_cache_blocks][Hkv][16][d], include/sx.h) to 4 bits: block
 * cache_blocks[i] into pool block pool_blocks[i], i < n.  Pairs with an id out of range are skipped;
 * the pool blocks of one call are distinct. */
sx_status sx_kv4_pack(const sx_layer_desc* desc, const void* k_cache, const void* v_cache, int64_t n_cache_blocks,
                      const int32_t* cache_blocks, int32_t n, void* pool, int64_t n_blocks,
                      const int32_t* pool_blocks, void* stream);

/* The other way: pool block pool_blocks[i] into block cache_blocks[i] of a paged cache, exactly. */
sx_status sx_kv4_unpack(const sx_layer_desc* desc, const void* pool, int64_t n_blocks, const int32_t* pool_blocks,
                        int32_t n, void* k_cache, void* v_cache, int64_t n_cache_blocks, const int32_t* cache_blocks,
                        void* stream);

/* Bytes of workspace that sx_kv4_attn needs for n_requests requests of at most max_q query tokens and
 * max_seqlen keys (partial results of requests whose keys are split): room for every request at both
 * bounds, at most 65536 * (4 * head_dim + 8) bytes each (of up to 4096 KV heads). */
sx_status sx_kv4_attn_workspace(const sx_layer_desc* desc, int32_t n_requests, int32_t max_q, int32_t max_seqlen,
                                int64_t* bytes);

/* Causal attention of every request's last tokens over its 4-bit blocks.  Request r has the query rows
 * cu_q[r] .. cu_q[r + 1] of q [total_q][Hq][d] (rows q_ld elements apart) and seq_lens[r] keys, those
 * of the queries' own tokens included (write them first); its query i stands at position
 * p = seq_lens[r] - n_r + i with n_r = cu_q[r + 1] - cu_q[r] and sees the keys j <= p:
 *   out[cu_q[r] + i, h] = sum_j softmax_j(scale * q[cu_q[r] + i, h] . K[j]) V[j]
 *   lse[cu_q[r] + i, h] = log sum_j exp(scale * q . K[j])     (natural log; lse may be NULL)
 * A row that sees no key (p < 0, no keys at all, or all its blocks missing) gives 0 and lse -inf.
 * Keys in blocks whose table entry is negative or out of range are left out.  What stands behind a
 * request's last key, or behind a row's own position, does not change the row's result, NaN included.
 *   cu_q [n_requests + 1], seq_lens [n_requests], block_table [n_requests][max_blocks]: DEVICE int32
 *   max_q, max_seqlen: host bounds of every n_r and seq_lens[r] (they size the launch; a request is cut
 *   to them); rows of q and out from cu_q[n_requests] on are left as they were
 *   out [total_q][Hq][d], lse [total_q][Hq] float32.  out may be q itself (q_ld = Hq * d); otherwise out, lse and
 *   workspace must not overlap each other or another argument (SX_EINVAL)
 *   workspace: sx_kv4_attn_workspace bytes, 16-byte aligned, any content; calls in flight at the same
 *   time need one each.
 * Products run on the bfloat16 matrix cores with float32 accumulation: the 4-bit values are bfloat16
 * values, a float32 q and its probabilities go through as three bfloat16 parts, a bfloat16 call's
 * probabilities as two (requests of at most 128 rows, query tokens x heads of the group) or one, divided by the
 * sum of what was multiplied.  Sums are float32 and divided at the end, with weights below 2^24 in between: they
 * hold for values up to 2^72. */
sx_status sx_kv4_attn(const sx_layer_desc* desc, const void* q, int64_t q_ld, const int32_t* cu_q,
                      const int32_t* seq_lens, const int32_t* block_table, int32_t max_blocks, int32_t n_requests,
                      int32_t total_q, int32_t max_q, int32_t max_seqlen, const void* pool, int64_t n_blocks, void* out,
                      float* lse, void* workspace, int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SX_DECODE_H */
