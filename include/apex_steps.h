/*
 * apex_steps.h -- C ABI of the calls for steps with several new tokens a
 * request (MI355X, gfx950): prompts, trees of drafted tokens, and the cache
 * blocks that new tokens take.
 *
 * The decode attention (apex_decode.h) attends one new token per request over
 * a paged fp16 cache whose blocks somebody gave out and whose rows a prompt
 * left there.  These calls are what comes before it and beside it:
 *     apex_steps_extend            blocks and slots for a batch's new tokens
 *     apex_steps_prompt_attention  the prompts over themselves
 *     apex_kv_append               (apex_kv_append.h) their rows into the slots
 *     apex_steps_tree_attention    drafted tokens over the cache and each other
 *     apex_steps_release           blocks of dropped tokens, given back
 *
 * A batch of B requests with several tokens each is packed: token_offsets
 * (int32 [B + 1], from 0, not descending) says that request b's tokens are the
 * rows token_offsets[b] .. token_offsets[b + 1] of every packed array of T rows.
 * Rows from token_offsets[B] on are padding: they are not read, and of what a
 * call writes they are left as they are (extend gives them the slot -1).
 * Offsets are cut to [0, T]; what comes of descending ones is unspecified, but
 * stays within the buffers.
 *
 * All buffers are device memory, row-major and contiguous unless a stride is
 * given.  q is fp16 [T][Hq][d] with q_token_stride elements between tokens, K
 * and V rows are fp16 [T][Hkv][d] with one stride between tokens for both (each
 * 0 for a tight array, otherwise a multiple of 8 and at least heads * d: views
 * of a fused projection's buffer); q, K, V, the caches and out are 16-byte
 * aligned, the other arrays to their element.  q-head h attends kv-head
 * h / (Hq / Hkv); any Hq that is a multiple of Hkv is supported.  lse_out (fp32
 * [T][Hq], may be NULL) is the natural-log log-sum-exp of the scaled logits.
 * Scores, softmax and sums are fp32.  The softmax's weights enter the product with
 * V as fp16: of the drafted tokens' attention in two parts, as the decode
 * attention's do, so that what is left is the output's own rounding; of the prompts'
 * in one, off by up to 2^-11 of a weight (and by 2^-36 of a row's largest).  A row
 * that attends nothing gives zeros and -inf.  What a row
 * does not attend has no influence on it, infinities and NaNs among it.
 * Supported: d = 128, B <= 2^22, Hq <= 2^16, (T + 256) * Hq < 2^30, B * Hkv + (T + 32) *
 * Hq / 32 < 2^30, strides < 2^31; block_size 16 for the attention, any for extend and release; anything else returns
 * APEX_ERR_UNSUPPORTED.
 *
 * Ownership and errors as in apex_decode.h: the caller owns every buffer, a
 * call validates on the host, enqueues its kernels on `stream` (NULL = the
 * legacy default stream) of the current device, which must be the buffers'
 * device, and returns without synchronising; on failure it enqueues nothing
 * and apex_steps_last_error() says why.  B == 0 or T == 0 is a successful no-op.
 */
#ifndef APEX_STEPS_H
#define APEX_STEPS_H

#include <stddef.h>
#include <stdint.h>

#include "apex_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Drafted tokens of a request that a tree_mask word can name. */
#define APEX_STEPS_MAX_NODES 64

/*
 * Gives a batch's new tokens their cache blocks and slots.  Request b has
 * L_b = context_lens[b] tokens in the blocks of its table row (int32
 * [B][block_table_stride]) and gets n_b = new_lens[b] more (negative values
 * count as 0).
 *
 * free_blocks (int32 [num_blocks]) is a stack of the ids of unused blocks,
 * free_state (int32 [2]) its height and a word that is 0 between calls.  Blocks
 * are taken from its top, for the requests in their order and a request's
 * positions upwards; the height is lowered by what was taken, free_blocks itself
 * is not written.
 *
 * A request is refused if its tokens would not fit its table row, if they end
 * behind row T of the packed batch, if L_b + n_b exceeds 2^31 - 1, or if it needs
 * blocks and those needed up to it (by requests that are not refused for one of
 * the other reasons) are more than there are.  A refused request takes nothing.
 *     token_offsets[b + 1] = min(n_0 + ... + n_b, T), token_offsets[0] = 0
 *     total_lens[b]        = L_b + n_b, of a refused request L_b
 *     slot_mapping[t]      = block * block_size + position % block_size (int64 [T]),
 *                            -1 for a refused request's tokens, for padding, and
 *                            where the block's id is outside [0, num_blocks)
 *     token_positions[t]   = L_b + index of the token in its request (int32 [T]), 0
 *                            for a refused request's tokens and padding
 * Calls that share a free_state must not overlap.  No two outputs may overlap,
 * nor an output and an input.  B == 0 and T == 0 are no no-ops here: what
 * remains is written (arrays of no elements may be NULL).
 */
int apex_steps_extend(const int32_t* context_lens, const int32_t* new_lens, int32_t* block_table,
                      int64_t block_table_stride, const int32_t* free_blocks, int32_t* free_state,
                      int32_t* token_offsets, int32_t* total_lens, int64_t* slot_mapping, int32_t* token_positions,
                      int B, int T, int block_size, int64_t num_blocks, void* stream);

/*
 * Gives back the blocks of dropped tokens: of request b, which has context_lens[b]
 * tokens, those that keep_lens[b] tokens (0: all go) do not need.  Their ids go on
 * top of free_blocks, for the requests in their order and a row's entries upwards;
 * the entries become -1.  Entries outside [0, num_blocks) are passed over.  A push
 * past num_blocks ids (a block given back twice) is dropped.
 */
int apex_steps_release(const int32_t* context_lens, const int32_t* keep_lens, int32_t* block_table,
                       int64_t block_table_stride, int32_t* free_blocks, int32_t* free_state, int B, int block_size,
                       int64_t num_blocks, void* stream);

/*
 * Causal attention of packed prompts over themselves:
 *     out[t][h] = sum_u softmax_u(scale * q[t][h] . k[u]) * v[u],  u from the request's first row to t
 * with out fp16 [T][Hq][d].
 */
int apex_steps_prompt_attention(const void* q, int64_t q_token_stride, const void* k, const void* v,
                                int64_t kv_token_stride, const int32_t* token_offsets, void* out, float* lse_out,
                                int B, int T, int Hq, int Hkv, int d, float scale, void* stream);

/*
 * Attention of drafted tokens: request b has L_b = context_lens[b] tokens in the
 * cache (as in apex_decode.h; L_b <= 0: none) and n_b drafted ones, whose rows are
 * packed and not in the cache yet.  Drafted token i attends the L_b cached tokens
 * and those drafted tokens j of its request that bit j of its tree_mask word
 * names (uint64 [T]; a token's own bit is up to the caller, bits from n_b on
 * count for nothing), so any tree, chain or set of branches will do:
 *     out[i][h] = sum_u softmax_u(scale * q[i][h] . K_u) * V_u
 * Once it is known which tokens are accepted, apex_kv_append stores their rows
 * (the others' slots -1).
 *
 * max_nodes (1 to APEX_STEPS_MAX_NODES) is the most drafted tokens of a request;
 * rows of a request behind its first max_nodes are taken as padding.  A context
 * longer than its table row is cut to the row; block ids outside [0, num_blocks)
 * are skipped: their tokens take no part.  num_blocks and block_table_stride < 2^27,
 * B * Hkv * (block_table_stride + 64) * ceil(max_nodes * Hq / Hkv / 128) < 2^31.
 * workspace: device memory of apex_steps_tree_workspace_bytes bytes, 256-byte
 * aligned, any content, or NULL for the library's own, one per device, grown on
 * demand (growing waits for the device).  Calls that can overlap need a
 * workspace each, and so do a captured graph's calls: under stream capture NULL is
 * refused.
 */
int apex_steps_tree_attention(const void* q, int64_t q_token_stride, const void* k_new, const void* v_new,
                              int64_t new_token_stride, const int32_t* token_offsets, const uint64_t* tree_mask,
                              const void* k_cache, const void* v_cache, const int32_t* block_table,
                              int64_t block_table_stride, const int32_t* context_lens, void* out, float* lse_out,
                              int B, int T, int max_nodes, int Hq, int Hkv, int d, int block_size,
                              int64_t num_blocks, float scale, void* workspace, size_t workspace_bytes, void* stream);

/* For the current device; 0 on bad shapes. */
size_t apex_steps_tree_workspace_bytes(int max_nodes, int Hq, int Hkv);

/* Message for the last failed call on this thread ("" if none). */
const char* apex_steps_last_error(void);

/* Frees the library's workspaces (waits for the devices first). */
int apex_steps_release_workspace(void);

#ifdef __cplusplus
}
#endif

#endif /* APEX_STEPS_H */
