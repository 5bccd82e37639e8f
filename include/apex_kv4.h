/*
 * apex_kv4.h -- C ABI of the 4-bit paged KV cache (MI355X, gfx950).
 *
 * GPU memory for KV pairs is what bounds the requests that a GPU attends in
 * the decode phase (APEX, Sec. 2.2 and Sec. 3.1); this cache holds 3.76 times
 * the tokens of an fp16 one, and its decode attention reads that much less.
 * Five calls: rows appended (quantised), rows read back as fp16, the decode
 * attention, the accumulation of its attention weights per cached token, and
 * the eviction of the lightest tokens down to a budget.
 *
 * Format.  A row of 128 values (one token's K or V of one kv-head) is four
 * groups of 32.  A group has one scale byte s, standing for 2^(s - 127), and
 * 32 codes of 4 bits, standing for 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 to 7)
 * and their negatives (8 to 15); a value is code x scale.  apex_kv4_append
 * takes the least power of two that keeps the group's largest value within 6
 * (an all-zero group: s = 127) and the nearest code, ties to the even code;
 * all of it is exact, so a row has one representation.  A group with a NaN
 * or an infinity gets s = 255 and stands for 32 NaNs.
 *
 * Layout.  kv_cache is [num_blocks][Hkv][APEX_KV4_SLAB_BYTES] bytes.  The slab
 * of a block of 16 tokens and one kv-head, for token t and dim i (j = i / 32):
 *   K codes   byte  t * 64 + i / 2                                     (even i: low 4 bits)
 *   V codes   byte  1024 + (t / 4) * 256 + (i / 8) * 16 + (t % 4) * 4 + (i % 8) / 2
 *   K scales  byte  2048 + t * 4 + j
 *   V scales  byte  2112 + j * 16 + t
 * weights (fp32) and positions (int32) of the cached tokens, where a caller
 * keeps them, are paged alike: [num_blocks][Hkv][16].
 *
 * All buffers are device memory, row-major and contiguous unless a stride is
 * given; q, k_new, v_new, out, k_out, v_out, kv_cache and weights are 16-byte
 * aligned, the other arrays to their element.  block_table is int32
 * [B][block_table_stride]; a context longer than its table row is cut to the
 * row; entries past ceil(L_b / 16) are never read.  Block ids outside [0,
 * num_blocks) are skipped: their tokens take no part.  Supported: d = 128,
 * block_size = 16, Hq / Hkv in {1, 2, 4, 8}, num_blocks < 2^31, block_table_stride < 2^27 - 1,
 * B * Hkv * (block_table_stride + 64) < 2^31, ceil(T / 16) * Hkv < 2^24, and in an
 * eviction B * Hkv < 2^22 and block_table_stride < 2^24; anything else returns
 * APEX_ERR_UNSUPPORTED.
 *
 * Ownership and errors as in apex_decode.h: the caller owns every buffer, a
 * call validates on the host, enqueues its kernels on `stream` (NULL = the
 * legacy default stream) of the current device, which must be the buffers'
 * device, and returns without synchronising; on failure it enqueues nothing
 * and apex_kv4_last_error() says why.  B == 0 or T == 0 is a successful no-op.
 */
#ifndef APEX_KV4_H
#define APEX_KV4_H

#include <stddef.h>
#include <stdint.h>

#include "apex_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

#define APEX_KV4_SLAB_BYTES 2176

/*
 * Appends rows: for every t in [0, T) with 0 <= slot_mapping[t] < num_blocks *
 * block_size and every kv-head, quantises k_new[t][g][:] and v_new[t][g][:]
 * (fp16, new_token_stride elements between tokens; 0 = Hkv * d, otherwise a
 * multiple of 8 and >= Hkv * d) into the slot.  Other slots, a padding token's
 * (negative) among them, are left as they are.  The slots of one call must be
 * distinct; of a slot given twice the content is unspecified.
 * positions and weights (either may be NULL): positions[slot][g] =
 * token_positions[t] (int32 [T], needed with positions), weights[slot][g] = 0.
 */
int apex_kv4_append(const void* k_new, const void* v_new, int64_t new_token_stride, void* kv_cache,
                    const int64_t* slot_mapping, const int32_t* token_positions, int32_t* positions,
                    float* weights, int T, int Hkv, int d, int block_size, int64_t num_blocks, void* stream);

/*
 * Reads rows back: k_out[t][g][:] and v_out[t][g][:] (fp16 [T][Hkv][d]) are the
 * values that slot_mapping[t] holds, rounded to fp16 (exact for every appended
 * value but the one that an append rounded up past 65504, which comes back as
 * 65504); zeros where the slot is outside the pool.  A slot may be given
 * several times.
 */
int apex_kv4_gather(const void* kv_cache, const int64_t* slot_mapping, void* k_out, void* v_out, int T,
                    int Hkv, int d, int block_size, int64_t num_blocks, void* stream);

/*
 * Decode attention of one layer-step:
 *     out[b][h] = sum_t softmax_t(scale * q[b][h] . K_t) * V_t,  t in [0, L_b)
 * with q and out fp16 [B][Hq][d], q-head h on kv-head h / (Hq / Hkv), and
 * lse_out (fp32 [B][Hq], may be NULL) the natural-log log-sum-exp of the scaled
 * logits.  L_b <= 0 gives zeros and -inf.  Scores, softmax and sums are fp32;
 * a row of q that holds a NaN or an infinity gives NaNs, a result past 65504
 * (of values that an append rounded up) is 65504.
 * workspace: device memory of apex_kv4_attention_workspace_bytes bytes, 256-byte
 * aligned, all zero before its first call (calls of any shapes that it is large
 * enough for may follow; what they need zero they leave zero, which an eviction
 * does not), or NULL for the library's own, one per device, grown on demand (growing
 * waits for the device).
 * Calls that can overlap need a workspace each, and so do a captured graph's
 * calls: under stream capture NULL is refused.
 */
int apex_kv4_attention(const void* q, const void* kv_cache, const int32_t* block_table,
                       int64_t block_table_stride, const int32_t* context_lens, void* out, float* lse_out,
                       int B, int Hq, int Hkv, int d, int block_size, int64_t num_blocks, float scale,
                       void* workspace, size_t workspace_bytes, void* stream);

/* 0 on bad shapes. */
size_t apex_kv4_attention_workspace_bytes(int B, int Hq, int Hkv);

/*
 * Accumulates the attention weights of a step whose log-sum-exp is lse:
 *     weights[slot of t][g] += sum over h of kv-head g of exp(scale * q[b][h] . K_t - lse[b][h]),  t in [0, L_b)
 * (the weights that the step's softmax gave the token, over the q-heads of its
 * kv-head).  A block may occur only once in the call's table rows.
 */
int apex_kv4_accumulate_weights(const void* q, const void* kv_cache, const int32_t* block_table,
                                int64_t block_table_stride, const int32_t* context_lens, const float* lse,
                                float* weights, int B, int Hq, int Hkv, int d, int block_size,
                                int64_t num_blocks, float scale, void* stream);

/*
 * Evicts tokens: of every request with more than `keep` tokens, each kv-head
 * keeps `keep` of them, in the first `keep` slots of its table row, and the
 * request's new length is keep (the caller's to set; its further blocks are
 * free).  Other requests are left as they are.  Only tokens and slots of the pool
 * count: in a row with ids outside it, the request's new length is up to the
 * keep-th slot of the pool, the slots outside before that included, and a request
 * with no more than `keep` tokens in the pool stays as long as it is.
 * Kept are, of each (request, kv-head): first the protected tokens, all alike,
 * those with a position below `sinks` or among the `recent` highest (position >
 * highest - recent), then the heaviest by weights; equal ones in the order of
 * their slots.  A NaN weighs as -infinity.  sinks + recent <= keep.
 * Tokens kept in the first `keep` slots stay where they are; the i-th evicted
 * slot there takes the i-th kept token from behind them, both counted upwards: its
 * K and V row, weight and position.  The slots behind are left as they are.  (The
 * attention does not depend on the order of the cached tokens; positions keeps
 * track of it.)  A block may occur only once in the call's table rows.
 * workspace: apex_kv4_evict_workspace_bytes bytes, 256-byte aligned, any content,
 * or NULL as above.
 */
int apex_kv4_evict(void* kv_cache, const int32_t* block_table, int64_t block_table_stride,
                   const int32_t* context_lens, float* weights, int32_t* positions, int B, int Hkv, int d,
                   int block_size, int64_t num_blocks, int keep, int sinks, int recent, void* workspace,
                   size_t workspace_bytes, void* stream);

/* 0 on bad shapes. */
size_t apex_kv4_evict_workspace_bytes(int B, int Hkv, int64_t block_table_stride);

/* Message for the last failed call on this thread ("" if none). */
const char* apex_kv4_last_error(void);

/* Frees the library's workspaces (waits for the devices first). */
int apex_kv4_release_workspace(void);

#ifdef __cplusplus
}
#endif

#endif /* APEX_KV4_H */
