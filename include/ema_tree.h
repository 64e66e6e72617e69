/*
 * ema_tree.h -- decoding with trees of drafted tokens over the paged cache of a
 * memory slice: the trees' masks and positions, attention of their nodes, the
 * path that the model's choices confirm, and the kept tokens moved together in the
 * cache.
 *
 * Everything ema_ops.h says about handles, devices, streams, host-only and
 * checked handles, counted errors and workspaces holds here too. No call here
 * allocates or synchronizes (checked mode aside), and nothing in the handle is written.
 *
 * A step: request b's last n_b tokens are the nodes of its tree, drafted from the
 * n tokens before them; they are rows [query_start[b], query_start[b + 1]) of the
 * step's arrays, a parent before its children. ema_kv_tables and ema_kv_store
 * bring them into the cache like a chunk of a prompt, ema_paged_tree_attention
 * attends layer by layer, ema_tree_accept finds the path to keep, ema_kv_compact moves
 * it behind the older tokens.
 */
#ifndef EMA_TREE_H
#define EMA_TREE_H

#include "ema_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EMA_TREE_WORDS 16        /* mask words of a node at most */
#define EMA_TREE_NODES 1024      /* nodes of a tree that tree_tables and tree_accept look at */

/*
 * tree_tables -- what the nodes of a step's trees attend and where they stand, for
 * all layers. parents[row]: the node's parent, counted from its request's first
 * row, below the node itself; -1: a root, which follows the request's older tokens
 * (there may be several).
 *   mask[row][w]     bit j: node 64 w + j of the request is the node itself or above it
 *   positions[row]   seq_lens[b] - n_b + the nodes above it (may be NULL)
 *   base[b]          seq_lens[b] - n_b, the tokens before the tree (may be NULL)
 * parents, query_start [batch + 1], seq_lens [batch]: device int32; mask: device
 * uint64 [tokens][mask_words], 8-byte aligned; positions [tokens], base [batch]: device
 * int32. Rows behind the last start stay as they were. Outputs must not overlap
 * each other or the inputs (INVAL). A parent that is not below its node, or below -1, makes a root,
 * counted; nodes from 64 * mask_words on get no bits and base as their position, their
 * request is counted; so is one with a length below n_b (base is negative then) and,
 * clamped, one whose starts are no range of the rows. mask_words in [1,
 * EMA_TREE_WORDS], batch up to 65535. Async on `stream`. Errors: INVAL (in
 * checked mode and host-only also any of the violations above), HIP.
 */
int ema_tree_tables(ema_slice_t h, const int32_t* parents, const int32_t* query_start,
                    const int32_t* seq_lens, int32_t tokens, int32_t batch, uint64_t* mask,
                    int32_t mask_words, int32_t* positions, int32_t* base, void* stream);

/*
 * paged_tree_attention -- attention of drafted nodes over the paged cache: row i of
 * request b attends every token before the drafted ones, t < seq_lens[b] - n_b, and
 * of these, at t = seq_lens[b] - n_b + j, those whose bit j of mask[row] is set:
 *   out[row][hq] = sum_t softmax_t(scale * q[row][hq] . K_t) V_t over them.
 * The mask need not be a tree's: any bits, the row's own set or not, of later nodes
 * too; bits from n_b on are not looked at, and nodes from 64 * mask_words on are attended by
 * none. A row that attends nothing gives zeros. q, query_start, block_table, seq_lens,
 * scale, out and out_dtype, rows that are no request's, what lies in places that a
 * row does not attend, values that are not finite, and the weights of 16-bit outputs
 * and EMA_FULL_WEIGHTS: as for ema_paged_prompt_attention. mask: device uint64
 * [tokens][mask_words], 8-byte aligned, mask_words in [1, EMA_TREE_WORDS]. A row whose
 * own token is at a negative position gives zeros, and its request is counted.
 * The work is cut by the lengths: the same call gives the same bits, other lengths in
 * the batch may change the last ones, a wider table does not where both hold more
 * than 512 tokens. The query heads of a KV head times a tree's nodes are best
 * up to 256: further ones read the request's K and V again. Any whole number of query heads per KV
 * head; tokens * num_q_heads below 2^29, batch up to 65535, and below 2^30: KV heads, times 64-token
 * tiles of max_blocks and four, times 64-row tiles of all requests' nodes and heads of a
 * group (INVAL otherwise). block_table may be NULL where max_blocks is 0. Async on `stream`;
 * `workspace` of ema_paged_tree_workspace bytes for these sizes. Errors: INVAL, HIP.
 */
int ema_paged_tree_workspace(ema_slice_t h, int32_t tokens, int32_t batch, int32_t num_q_heads,
                             int32_t max_blocks, size_t* bytes);
int ema_paged_tree_attention(ema_slice_t h, const void* q, int64_t q_stride,
                             const int32_t* query_start, const int32_t* block_table,
                             const int32_t* seq_lens, const uint64_t* mask, int32_t mask_words,
                             int32_t tokens, int32_t batch, int32_t num_q_heads,
                             int32_t max_blocks, float scale, void* out, int32_t out_dtype,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * tree_accept -- the path of each tree that the model's choices confirm. drafted[row]:
 * the node's token; choice[row]: the token the model gives after the node. From a
 * node, the path goes on to its lowest child whose token is the model's choice after it.
 * It begins at the lowest root whose token is root_choice[b], the model's choice after
 * the older tokens; where root_choice is NULL, at node 0, which is accepted as it is
 * (the token sampled last, whose K and V were not in the cache yet).
 *   path[b][k]   the path's k-th node, k < n_path[b]; -1 behind
 *   n_path[b]    its length, path_cap at most (the path ends there)
 *   next[b]      choice after its last node; root_choice[b] where there is none, -1
 *                without root_choice (a request without nodes)
 * All arrays are device int32: parents, drafted, choice [tokens], query_start [batch +
 * 1], root_choice [batch], path [batch][path_cap], n_path, next [batch]. Outputs must not
 * overlap each other or the inputs (INVAL). Parents as for ema_tree_tables, those out of range make
 * nodes that no path reaches, counted; nodes from EMA_TREE_NODES on are not looked
 * at and their request is counted. path_cap at least 1, batch up to 65535. Async on
 * `stream`. Errors: INVAL (in checked mode and host-only also bad parents or starts), HIP.
 */
int ema_tree_accept(ema_slice_t h, const int32_t* parents, const int32_t* query_start,
                    const int32_t* drafted, const int32_t* choice, const int32_t* root_choice,
                    int32_t tokens, int32_t batch, int32_t path_cap, int32_t* path,
                    int32_t* n_path, int32_t* next, void* stream);

/*
 * kv_compact -- moves the kept ones of a request's last tokens together, in all
 * layers and in place: token base[b] + k becomes what token base[b] + keep[b][k] was,
 * for k < n_keep[b], and
 *   new_lens[b] = base[b] + n_keep[b]   (may be NULL)
 * The K and V of an accepted path go behind the older tokens that way, as do those that a
 * context keeps of its tokens. keep[b] ascends (each entry above the one before);
 * what lies from new_lens[b] on, is whatever was there or was moved from there.
 * block_table: device int32 [layers][batch][max_blocks] unified ids of the canonical
 * tables: blocks are changed where they live, in either pool and the slice's
 * layout; staged copies stay as they were. No block may be named twice among those that
 * moved tokens come from or go to. base, n_keep [batch], keep [batch][keep_cap],
 * new_lens: device int32; new_lens must not overlap the inputs (INVAL). A negative base,
 * n_keep outside [0, keep_cap] (clamped), an entry that does not ascend or lies past the table, and a
 * table entry outside both pools that a moved token is in, are counted (the
 * entries once for every layer and moved token there) and those tokens not moved. Arrays of up to
 * nine columns (keep_cap) take a form for short lists that is several times faster.
 * layers in [1, 65535], batch up to 65535, batch * max_blocks * block_size below 2^31. Async
 * on `stream`. Errors: INVAL (in checked mode and host-only also any of the violations
 * above), HIP.
 */
int ema_kv_compact(ema_slice_t h, const int32_t* block_table, const int32_t* base,
                   const int32_t* keep, const int32_t* n_keep, int32_t layers, int32_t batch,
                   int32_t max_blocks, int32_t keep_cap, int32_t* new_lens, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* EMA_TREE_H */
