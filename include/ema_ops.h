/*
 * ema_ops.h -- operators that bring prompts into the paged cache of a memory
 * slice and attend over it: tables and slot maps built on the GPU, the store
 * of a chunk's K and V, causal attention of prompt chunks, and differential
 * attention of single tokens and of chunks.
 *
 * Everything ema_slice.h says about handles, pools, unified ids, layouts,
 * return values, devices and streams holds here too. A call on a host-only
 * handle takes host arrays, validates them and launches nothing; on a
 * handle made with EMA_CREATE_CHECKED the device arrays are read back and
 * validated first (not while `stream` is capturing: INVAL). Otherwise kernels
 * skip what is out of range and count it (ema_slice_device_errors): a table entry,
 * a length, a request's starts each once a call, however many heads look at them.
 *
 * Workspaces belong to the caller: a call that needs one says how many bytes
 * (ema_*_workspace; 0: none, NULL will do), 16-byte aligned device memory that
 * nothing else uses until the call's work on `stream` is done. Nothing is kept
 * in it between calls and nothing in the handle is written, so calls on one
 * handle may run at once on different streams, each with its own workspace,
 * and graphs captured with different workspaces may be replayed at once.
 * No call here allocates or synchronizes (checked mode aside).
 */
#ifndef EMA_OPS_H
#define EMA_OPS_H

#include "ema_slice.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EMA_FULL_WEIGHTS 0x100   /* with an out_dtype: softmax weights of 32-bit accuracy */

/*
 * kv_tables -- the tables of a step for all layers, from the requests' lengths
 * (section 4: a request's logical blocks map to segments of the slice or to
 * local memory; section 5.1: the accessing GPU reads the prefetched copy). Request b
 * has seq_lens[b] tokens, the last new_lens[b] of them new in this step, in
 * n_b = ceil(seq_lens[b] / block_size) blocks; first_b is the sum of n_b' over
 * b' < b, and for layer l its block j is block_ids[l][first_b + j].
 *   canon_table[l][b][j]  that id, -1 for n_b <= j < max_blocks (may be NULL)
 *   block_table[l][b][j]  the same, with each slice id replaced by its staged copy
 *                         staging_ids[l % staging_slots][r], r the number of
 *                         slice ids before it in layer l in (b, j) order
 *   query_start[b]        sum of new_lens[b'] over b' < b; [batch] is the total
 *   slot_map[l][t]        block_table entry * block_size + row of the t-th new
 *                         token (request by request, in order); -1 from the
 *                         total on and for tokens whose block is not local
 *   prefetch_src/dst[l]   slice ids and staged copies of the slice blocks that
 *                         hold older tokens, in (b, j) order, what
 *                         ema_slice_prefetch takes; prefetch_n[l] of them, -1
 *                         behind (stage_n entries a layer)
 *   writeback_src/dst[l]  staged copies and slice ids of the slice blocks that
 *                         take new tokens, in order, what ema_slice_writeback
 *                         takes; writeback_n[l] of them, -1 behind
 *                         (writeback_cap entries a layer). A block without older
 *                         tokens was not prefetched: behind the request's length
 *                         it takes back whatever its staging block held
 * All arrays are device int32, written whole. Without staging (staging_slots
 * 0) block_table keeps slice ids, the lists are not touched and their pointers may be
 * NULL. The outputs must not overlap each other or the inputs. Lengths outside
 * [0, max_blocks * block_size], new lengths outside [0, length], ids
 * outside both pools, requests whose blocks lie past block_ids' `n_ids` per
 * layer, slice blocks past stage_n, write-backs past writeback_cap, new tokens
 * past n_slots or in a block that is not local: clamped or left out (-1), and
 * counted. Async on `stream`; `workspace` of ema_kv_tables_workspace bytes.
 * layers in [1, 65535], batch * max_blocks * block_size below 2^31.
 * Errors: INVAL (sizes, NULL arrays, workspace too small; in checked mode and
 * host-only also any of the violations above), HIP.
 */
typedef struct {
  const int32_t* block_ids;     /* [layers][n_ids] */
  const int32_t* seq_lens;      /* [batch] */
  const int32_t* new_lens;      /* [batch] */
  const int32_t* staging_ids;   /* [staging_slots][stage_n] local ids */
  int32_t* canon_table;         /* [layers][batch][max_blocks], or NULL */
  int32_t* block_table;         /* [layers][batch][max_blocks] */
  int32_t* query_start;         /* [batch + 1] */
  int32_t* slot_map;            /* [layers][n_slots] */
  int32_t* prefetch_src;        /* [layers][stage_n] */
  int32_t* prefetch_dst;
  int32_t* prefetch_n;          /* [layers] */
  int32_t* writeback_src;       /* [layers][writeback_cap] */
  int32_t* writeback_dst;
  int32_t* writeback_n;         /* [layers] */
  int32_t layers, batch, max_blocks;
  int32_t n_ids;                /* block ids a layer has */
  int32_t n_slots;              /* slot_map entries a layer has */
  int32_t staging_slots, stage_n, writeback_cap;
} ema_kv_tables_args;

int ema_kv_tables_workspace(ema_slice_t h, const ema_kv_tables_args* args, size_t* bytes);
int ema_kv_tables(ema_slice_t h, const ema_kv_tables_args* args, void* workspace,
                  size_t workspace_bytes, void* stream);

/*
 * kv_store -- the K and V of a chunk's tokens into their blocks (the many-token
 * form of ema_kv_append): token t goes to row slot_map[t] % block_size of local
 * block slot_map[t] / block_size; slot -1 stores nothing. k_new, v_new: device
 * [tokens][num_kv_heads][head_dim] in the slice's dtype, rows of a token
 * contiguous, tokens k_stride and v_stride elements apart (a fused projection's
 * output is read in place); 16-byte aligned, strides multiples of 8 elements and
 * at least num_kv_heads * head_dim.
 * No slot twice (which of the two tokens is stored, is not defined). Slots past
 * the local pool are skipped and counted. Async on `stream`. Errors: INVAL (also,
 * in checked mode and host-only, a slot past the pool or named twice), HIP.
 */
int ema_kv_store(ema_slice_t h, const void* k_new, int64_t k_stride, const void* v_new,
                 int64_t v_stride, const int32_t* slot_map, int32_t tokens, void* stream);

/*
 * paged_prompt_attention -- causal attention of prompt chunks over the paged cache
 * (the many-token form of ema_paged_decode_attention). Request b's queries are rows
 * [query_start[b], query_start[b + 1]) of q, n_b of them, its last n_b tokens: row i
 * of them sits at position p = seq_lens[b] - n_b + i and
 *   out[row][hq] = sum_t softmax_t(scale * q[row][hq] . K_t) V_t, t <= p,
 * with K and V read through the block table (the chunk's own tokens among
 * them: store them first). q: device [tokens][num_q_heads][head_dim] in the
 * slice's dtype, tokens q_stride elements apart, 16-byte aligned, q_stride a
 * multiple of 8 and at least num_q_heads * head_dim. query_start: device int32
 * [batch + 1], ascending from 0 to at most `tokens`; rows of out past its last
 * entry stay as they were. A row at a negative position (more queries than
 * tokens) gives zeros, and its request is counted. Starts that do not begin at 0,
 * descend or pass `tokens` are clamped and their requests counted; what rows hold
 * that then belong to no request, or to two, is not defined. What lies behind a
 * request's length and what a row's mask leaves out may hold anything, infinities
 * and NaN too. A row that attends an infinity or NaN in V gets something not
 * finite in its channel (NaN, or the infinity), one that attends NaN in K, or a
 * score of +infinity, NaN; one whose scores are all -infinity gives zeros.
 * The tokens are cut into parts by the sizes, types and max_blocks, not by the
 * lengths: the same call gives the same bits, one with a wider table may differ in
 * the last ones (and take longer: a table much wider than the lengths makes parts
 * without tokens).
 * out: device [tokens][num_q_heads][head_dim] of out_dtype, 16-byte aligned.
 * EMA_F32 keeps the softmax weights in as many 16-bit parts as 32-bit
 * accuracy takes (f16 two, in a power-of-two scale that keeps them from f16's
 * smallest steps; bf16 three); the 16-bit types use one part, rounded to nearest,
 * whose error is that of the output's own rounding (together 1.3 to 1.6 times it).
 * EMA_F16 and EMA_BF16 may be given with EMA_FULL_WEIGHTS: as EMA_F32, in its
 * time, and rounded once at the end.
 * Any whole number of query heads per KV head; tokens * num_q_heads below 2^29,
 * batch up to 65535. scale <= 0 means
 * 1/sqrt(head_dim). Async on `stream`; `workspace` of
 * ema_paged_prompt_workspace bytes for these sizes (it does not depend on the
 * lengths). Errors: INVAL (in checked mode and host-only also bad starts, lengths or
 * table entries), HIP.
 */
int ema_paged_prompt_workspace(ema_slice_t h, int32_t tokens, int32_t batch, int32_t num_q_heads,
                               int32_t max_blocks, size_t* bytes);
int ema_paged_prompt_attention(ema_slice_t h, const void* q, int64_t q_stride,
                               const int32_t* query_start, const int32_t* block_table,
                               const int32_t* seq_lens, int32_t tokens, int32_t batch,
                               int32_t num_q_heads, int32_t max_blocks, float scale, void* out,
                               int32_t out_dtype, void* workspace, size_t workspace_bytes,
                               void* stream);

/*
 * paged_diff_attention -- differential attention of one token per sequence: the
 * difference of two softmax maps, the second weighted by a learned factor per
 * head. Query heads 2i and 2i + 1 are the two maps of head i, KV heads 2j and
 * 2j + 1 their keys, j = i / (num_q_heads / num_kv_heads), and the two
 * KV heads' values side by side (2 * head_dim channels) the head's values:
 *   o = sum_t (softmax_t(scale * q[2i] . K[2j]_t)
 *              - lambda[i] * softmax_t(scale * q[2i + 1] . K[2j + 1]_t)) V[j]_t
 *   out[b][i] = o, or, with norm_weight, o / sqrt(mean(o^2) + norm_eps) * norm_weight
 *   (o = 0 stays 0 where norm_eps is 0)
 * for t < seq_lens[b]. lambda: device float [num_q_heads / 2]; norm_weight:
 * device float [2 * head_dim], 16-byte aligned, or NULL (a constant factor of the
 * layer is folded into it). out: device [batch][num_q_heads / 2][2 * head_dim] of out_dtype,
 * 16-byte aligned. q as for ema_paged_prompt_attention (row b is sequence b's);
 * block_table, seq_lens, scale as for ema_paged_decode_attention; length 0 gives zeros.
 * Tokens and values that are not finite, and bits and table widths, as above.
 * The 16-bit types use weights in two parts here (bf16: 16 bits), EMA_FULL_WEIGHTS as above.
 * num_kv_heads must be even, num_q_heads / num_kv_heads a whole number up to 16. Async
 * on `stream`; `workspace` of ema_paged_diff_workspace bytes. Errors: INVAL, HIP.
 */
int ema_paged_diff_workspace(ema_slice_t h, int32_t batch, int32_t num_q_heads,
                             int32_t max_blocks, size_t* bytes);
int ema_paged_diff_attention(ema_slice_t h, const void* q, int64_t q_stride,
                             const int32_t* block_table, const int32_t* seq_lens, int32_t batch,
                             int32_t num_q_heads, int32_t max_blocks, float scale,
                             const float* lambda, const float* norm_weight, float norm_eps,
                             void* out, int32_t out_dtype, void* workspace,
                             size_t workspace_bytes, void* stream);

/*
 * paged_diff_prompt_attention -- differential attention of prompt chunks: heads,
 * lambda and norm as for ema_paged_diff_attention, rows, positions and masks as
 * for ema_paged_prompt_attention (any whole number of query heads per KV head); out:
 * device [tokens][num_q_heads / 2][2 * head_dim]. `workspace` of
 * ema_paged_diff_prompt_workspace bytes. Errors: INVAL, HIP.
 */
int ema_paged_diff_prompt_workspace(ema_slice_t h, int32_t tokens, int32_t batch,
                                    int32_t num_q_heads, int32_t max_blocks, size_t* bytes);
int ema_paged_diff_prompt_attention(ema_slice_t h, const void* q, int64_t q_stride,
                                    const int32_t* query_start, const int32_t* block_table,
                                    const int32_t* seq_lens, int32_t tokens, int32_t batch,
                                    int32_t num_q_heads, int32_t max_blocks, float scale,
                                    const float* lambda, const float* norm_weight, float norm_eps,
                                    void* out, int32_t out_dtype, void* workspace,
                                    size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* EMA_OPS_H */
