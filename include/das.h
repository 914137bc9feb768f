/*
 * das.h -- C ABI of the GB300 (sm_103a) library for the data-parallel hot path
 * of DAS-Wave decoding ("Shallow Queries, Mature Values: Depth-Asynchronous
 * Self-Speculation for Looped Transformers").
 *
 * The library computes, on one GPU:
 *   das_mature_v_attention  depth-asynchronous draft attention, Eqs. 2-3
 *                           (Sec. 3.2), with explicit read depths (Eq. 4):
 *                           Mature-V is (key_depth, value_depth) = (r, R);
 *   das_verify_attention    the full-depth verify attention of Sec. 3.4
 *                           (Eq. 7): the same with key and value depth equal;
 *   das_greedy_accept       greedy acceptance of Sec. 3.4;
 *   das_kv_append           the commit of Sec. 3.4 / App. B.1.
 *
 * Conventions shared by every entry point
 *   - Every pointer argument marked "device" is device memory owned by the
 *     caller; the library never allocates or frees device memory.  Host
 *     pointers are read during the call only.
 *   - Calls are asynchronous on `stream` (a cudaStream_t; 0 = legacy default
 *     stream) and never synchronise the host.  Errors found on the host
 *     (arguments) are returned before anything is launched and nothing is
 *     written.  Errors found on the device are reported through flags
 *     described at each call.
 *   - bf16 tensors are IEEE bfloat16, row-major in the stated index order,
 *     densely packed, with base addresses aligned to 16 bytes.
 *   - Recurrent depths are numbered as in the paper: 1..R, R = full depth.
 *     Depth d is stored in slab d-1 of the cache.
 *   - Query head h reads kv head h / G, G = num_q_heads / kv_heads
 *     (contiguous grouping; the paper does not fix one).
 */
#ifndef DAS_H
#define DAS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DAS_OK = 0,
    DAS_ERR_INVALID_ARG = 1, /* a null pointer, bad size, depth or alignment */
    DAS_ERR_UNSUPPORTED = 2, /* a shape outside what the kernels implement  */
    DAS_ERR_WORKSPACE = 3,   /* workspace missing or smaller than required  */
    DAS_ERR_CUDA = 4         /* a CUDA runtime call failed                  */
} das_status;

/*
 * Depth-indexed KV cache of the verified prefix (Sec. 2: the cache holds
 * K_C^{r,l} and V_C^{r,l} for every recurrent depth r and core layer l; only
 * target-materialized positions are stored, App. B.1).
 *   k, v   device bf16 [depths][layers][batch][capacity][kv_heads][head_dim]
 * Slab (d, l, b) is contiguous, so the keys of one depth and the values of
 * another stream independently.  Positions >= prefix_len[b] may hold anything.
 */
typedef struct {
    void *k;
    void *v;
    int depths;   /* R, number of stored recurrent depths, 1..63        */
    int layers;   /* core layers                                        */
    int batch;    /* sequences                                          */
    int capacity; /* positions per sequence                             */
    int kv_heads; /* Hkv                                                */
    int head_dim; /* D: 64 or 128                                       */
} das_kv_cache;

/*
 * Bytes of device workspace that das_mature_v_attention and
 * das_verify_attention need for this cache shape, num_q_heads and max_block
 * on the current device.  Returns 0 for shapes the kernels do not support.
 * The first 256 bytes of a workspace are a header; its first int32 is a
 * status word that the kernels OR with 1 if an internal wait ran out (a bug
 * guard; it stays set until the caller clears it).  Zero a new workspace once
 * before its first use.
 */
size_t das_workspace_size(const das_kv_cache *cache, int num_q_heads, int max_block);

/*
 * Depth-asynchronous attention, Eqs. 2-3 (Sec. 3.2).  For each sequence b,
 * query head h and block row i < block_len[b]:
 *   keys   = [ K[key_depth][layer][b][j][h/G]   for j < prefix_len[b] ]
 *            ++ [ k_blk[b][j][h/G] for j <= i ]      (causal mask M)
 *   values = [ V[value_depth][layer][b][j][h/G] for j < prefix_len[b] ]
 *            ++ [ v_blk[b][j][h/G] for j <= i ]
 *   s_j = softmax_scale * <q[b][i][h], keys_j>,  one softmax over all j,
 *   out[b][i][h] = sum_j softmax(s)_j values_j,
 *   lse[b][h][i] = ln sum_j exp(s_j).
 * Mature-V for a draft at depth r is (key_depth, value_depth) = (r, R);
 * Aligned (r, r), Deep K (R, r) and Deep K/V (R, R) are the other policies
 * of Eq. 4.  The block's own K/V (k_blk, v_blk) are produced by the current
 * draft and are never written to the cache by this call (Sec. 3.2, 3.3).
 *
 *   cache          the depth-indexed cache (read only)
 *   layer          core layer, 0 <= layer < cache->layers
 *   key_depth      kappa, 1..cache->depths
 *   value_depth    nu, 1..cache->depths
 *   prefix_len     device int32 [batch]: verified prefix length per sequence,
 *                  0..capacity
 *   block_len      device int32 [batch]: draft rows per sequence, 0..max_block
 *   max_block      rows allocated per sequence in q/k_blk/v_blk/out/lse;
 *                  (num_q_heads / kv_heads) * max_block <= 64, max_block <= 64
 *   q              device bf16 [batch][max_block][num_q_heads][head_dim]
 *   k_blk, v_blk   device bf16 [batch][max_block][kv_heads][head_dim]
 *   num_q_heads    Hq, a multiple of kv_heads
 *   softmax_scale  scale of Eq. 2; <= 0 selects 1/sqrt(head_dim)
 *   out            device bf16 [batch][max_block][num_q_heads][head_dim];
 *                  rows i >= block_len[b] are written as 0
 *   lse            device fp32 [batch][num_q_heads][max_block]; -inf for rows
 *                  i >= block_len[b]
 *   workspace      device scratch of at least das_workspace_size() bytes,
 *                  aligned to 256 bytes; calls sharing a workspace must not
 *                  overlap in time
 * Device-side: prefix_len or block_len outside their ranges are clamped and
 * bit 1 of the workspace status word is set.
 */
das_status das_mature_v_attention(const das_kv_cache *cache, int layer, int key_depth,
                                  int value_depth, const int32_t *prefix_len,
                                  const int32_t *block_len, int max_block, const void *q,
                                  const void *k_blk, const void *v_blk, int num_q_heads,
                                  float softmax_scale, void *out, float *lse, void *workspace,
                                  size_t workspace_bytes, void *stream);

/*
 * Independent full-depth verify attention (Sec. 3.4, Eq. 7): the verifier
 * input [x_t, y_1 .. y_{w-1}] is the block (block_len[b] = w rows), it
 * attends to the verified prefix at one depth for keys and values alike
 * (depth = R for the target's last recurrence; every depth d of the verify
 * pass uses the same call) and to itself under the causal mask.  Arguments
 * and results as das_mature_v_attention with key_depth = value_depth = depth.
 */
das_status das_verify_attention(const das_kv_cache *cache, int layer, int depth,
                                const int32_t *prefix_len, const int32_t *block_len,
                                int max_block, const void *q, const void *k_blk,
                                const void *v_blk, int num_q_heads, float softmax_scale,
                                void *out, float *lse, void *workspace, size_t workspace_bytes,
                                void *stream);

/*
 * Greedy acceptance (Sec. 3.4).  logits[b][i] stands for the verifier's
 * conditional p_{i+1} of proposal y_{i+1} = draft_ids[b][i]:
 *   target_ids[b][i] = argmax_v logits[b][i][v]   (smallest index on ties;
 *                      binary32 comparisons; NaN logits are out of contract)
 *   accepted[b]      = number of leading i with draft_ids[b][i] == target_ids[b][i]
 *   next_token[b]    = target_ids[b][accepted[b]] if accepted[b] < W (the target
 *                      prediction emitted at the first mismatch), otherwise
 *                      draft_ids[b][W-1] (every proposal accepted: no further
 *                      conditional exists, and the last accepted token becomes
 *                      the next anchor).
 *   logits      device fp32 [B][W][vocab]
 *   draft_ids   device int32 [B][W]
 *   accepted    device int32 [B];  target_ids device int32 [B][W];
 *   next_token  device int32 [B]
 * Requires 1 <= W <= 1024, 1 <= vocab < 2^31.
 */
das_status das_greedy_accept(const float *logits, const int32_t *draft_ids, int B, int W,
                             int vocab, int32_t *accepted, int32_t *target_ids,
                             int32_t *next_token, void *stream);

/*
 * Shifted token readout of a DAS-Wave refinement round (Sec. 3.3, Eq. 6).
 * After the k recurrent draft updates of round j over the W = W_j active
 * positions [x_t, z_1 .. z_{W-1}] (W_j = min(gamma, W_init + j), Eq. 5), the
 * readout of position i updates the guess of the following position:
 *   tokens[b][i + 1] = argmax_v logits[b][i][v]   for 0 <= i < W
 * (smallest index on ties, binary32 comparisons, as das_greedy_accept).
 * tokens[b][0] (the anchor) and tokens[b][i] for i > W are not written; the
 * readout of the last active position is the candidate that enters the
 * window in the next round.
 *   logits   device fp32 [B][W][vocab]
 *   tokens   device int32 [B][stride], stride >= W + 1
 * Requires 1 <= W <= 1024, 1 <= vocab < 2^31.
 */
das_status das_wave_readout(const float *logits, int B, int W, int vocab, int32_t *tokens,
                            int stride, void *stream);

/*
 * Commit (Sec. 3.4; App. B.1): the verifier consumed W inputs
 * [x_t, y_1 .. y_{W-1}] and produced their K/V at every depth and layer.
 * With accepted[b] = a proposals accepted, the first n = min(a + 1, W) inputs
 * (the anchor and the accepted proposals that were verifier inputs) are
 * materialized: their staged K/V are copied byte for byte to cache positions
 * prefix_len[b] .. prefix_len[b] + n - 1 at every depth and layer, and
 * prefix_len[b] += n.  Rejected candidates' K/V are discarded.
 *   k_new, v_new  device bf16 [depths][layers][batch][W][kv_heads][head_dim]
 *   accepted      device int32 [batch] (as written by das_greedy_accept)
 *   prefix_len    device int32 [batch], updated in place
 *   error_flag    device int32: set to 1 (never cleared) if a sequence would
 *                 exceed the capacity; that sequence's cache and prefix_len
 *                 are left untouched
 * Requires 1 <= W <= capacity.
 */
das_status das_kv_append(const das_kv_cache *cache, const void *k_new, const void *v_new,
                         const int32_t *accepted, int W, int32_t *prefix_len,
                         int32_t *error_flag, void *stream);

/*
 * Bytes of device scratch built into the library for
 * das_mature_v_attention_noalloc (32 MiB on every device that loads it).
 */
#define DAS_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)

/*
 * das_mature_v_attention without a caller-provided workspace.  The paper has
 * no counterpart: this is for callers that cannot allocate device memory when
 * they call (a fixed memory plan in a serving loop, a plugin that only
 * receives the tensors it works on, a host that forbids cudaMalloc after
 * start-up).  The split-K scratch is a fixed array of
 * DAS_NOALLOC_SCRATCH_BYTES inside the library's device image, present on
 * every device that loads the library until the process exits; this call
 * allocates nothing and calls no allocating routine.
 *   - Arguments and results as das_mature_v_attention, minus the workspace.
 *   - Returns DAS_ERR_WORKSPACE if the shape needs more scratch than
 *     DAS_NOALLOC_SCRATCH_BYTES (das_workspace_size() tells how much), with
 *     nothing launched.
 *   - The first call on a device looks up the array's device address (set-up
 *     done once per device, then kept); make that first call before any CUDA
 *     graph capture on that device.  After cudaDeviceReset on a device, later
 *     calls in that process are invalid.
 *   - All calls share the array and it keeps the last call's contents: calls
 *     that overlap in time on the GPU race and must be ordered by the caller.
 *     A call that passes its argument checks clears the status word at the
 *     array's head (on `stream`, just before its kernels); its bits, as for
 *     the workspace status word of das_mature_v_attention, are read with
 *     das_noalloc_status until the next call.  A call that returns an error
 *     enqueues nothing.
 */
das_status das_mature_v_attention_noalloc(const das_kv_cache *cache, int layer, int key_depth,
                                          int value_depth, const int32_t *prefix_len,
                                          const int32_t *block_len, int max_block, const void *q,
                                          const void *k_blk, const void *v_blk, int num_q_heads,
                                          float softmax_scale, void *out, float *lse,
                                          void *stream);

/*
 * Copies the status word of das_mature_v_attention_noalloc's scratch on the
 * current device (bit 0: an internal wait timed out; bit 1: a prefix or block
 * length was out of range and clamped) to `dst` (host or device memory,
 * 4 bytes) on `stream`, after the work enqueued there before it.  Allocates
 * nothing.  The paper has no counterpart.
 */
das_status das_noalloc_status(int32_t *dst, void *stream);

/*
 * A depth-indexed cache whose depths below R are stored as 8-bit floats.
 * The paper has no counterpart: it keeps every depth in the model's precision.
 * This variant halves the bytes of the shallow-depth stream that Mature-V
 * reads (keys at depth r < R) while the mature depth R that carries the
 * values and the verifier's reads at R stays bf16.
 *   k_top, v_top  device bf16 [layers][batch][capacity][kv_heads][head_dim]:
 *                 depth R
 *   k_low, v_low  device e4m3 (OCP FP8 E4M3: 1 sign, 4 exponent bits with
 *                 bias 7, 3 mantissa bits; no infinities, S.1111.111 is NaN;
 *                 largest finite 448)
 *                 [depths - 1][layers][batch][capacity][kv_heads][head_dim]:
 *                 depth d < R at slab d - 1; may be NULL when depths == 1
 * All pointers 16-byte aligned; the caller owns the memory.
 */
typedef struct {
    void *k_top;
    void *v_top;
    void *k_low;
    void *v_low;
    int depths, layers, batch, capacity, kv_heads, head_dim;
} das_kv_cache_f8;

/* Workspace bytes for das_mature_v_attention_f8 (as das_workspace_size). */
size_t das_workspace_size_f8(const das_kv_cache_f8 *cache, int num_q_heads, int max_block);

/*
 * das_mature_v_attention over a das_kv_cache_f8: keys are read at key_depth
 * and values at value_depth from k_top / v_top (depth R) or from k_low / v_low
 * (depths below R, e4m3), so Eqs. 2-3 are evaluated on the stored values.
 * key_depth = value_depth = d is the verify attention of depth d (Sec. 3.4).
 * All other arguments, results and limits as das_mature_v_attention.
 * e4m3 operands are widened exactly to bf16 before the products, except for
 * e4m3 keys with bf16 values at head_dim 128 (Mature-V, key_depth < R =
 * value_depth): there the scores are e4m3 products of the stored keys with
 * each query row split exactly into two e4m3 parts under a power of two per
 * row (exact for elements down to about 2^-9 of the row's largest magnitude,
 * fp32 accumulation), and the queries must be finite.
 */
das_status das_mature_v_attention_f8(const das_kv_cache_f8 *cache, int layer, int key_depth,
                                     int value_depth, const int32_t *prefix_len,
                                     const int32_t *block_len, int max_block, const void *q,
                                     const void *k_blk, const void *v_blk, int num_q_heads,
                                     float softmax_scale, void *out, float *lse, void *workspace,
                                     size_t workspace_bytes, void *stream);

/*
 * das_kv_append into a das_kv_cache_f8: the staged bf16 K/V of depth R are
 * copied byte for byte; those of depths below R are rounded to e4m3 (round to
 * nearest, ties to even; magnitudes above 448 saturate to 448; NaN stays NaN).
 * Arguments and errors as das_kv_append.
 */
das_status das_kv_append_f8(const das_kv_cache_f8 *cache, const void *k_new, const void *v_new,
                            const int32_t *accepted, int W, int32_t *prefix_len,
                            int32_t *error_flag, void *stream);

/*
 * ---- Paged cache with block scales, and sampling ----------------------------
 * The paper has no counterpart for what follows: its experiments decode one
 * sequence greedily out of one contiguous cache.
 */

/* Tokens of one page, and of one block of a scale. */
#define DAS_PAGE_TOKENS 64

/*
 * A depth-indexed cache in pages of 64 tokens, every depth held in 8 bits with
 * a scale per (page, kv head):
 *   k, v              device e4m3 (as in das_kv_cache_f8)
 *                     [depths][layers][pages][kv_heads][64][head_dim]
 *   k_scale, v_scale  device fp32 [depths][layers][pages][kv_heads], positive;
 *                     the key (value) is its code times its page's scale
 * A sequence's tokens 64 t .. 64 t + 63 are in page block_table[b][t]; the
 * tables, of as many sequences as the caller has, are arguments of the calls.
 * Places of a page past its sequence's length may hold anything.  k and v are
 * 16-byte aligned; the caller owns the memory.
 */
typedef struct {
    void *k;
    void *v;
    float *k_scale;
    float *v_scale;
    int depths, layers, pages, kv_heads, head_dim; /* head_dim: 64 or 128 */
} das_kv_cache_paged;

/*
 * Block tables and slot maps from request lengths.  Request b holds
 * seq_len[b] tokens in pages(seq_len[b]) pages, pages(n) = ceil(n / 64), the
 * first entries of row b of block_table; grow[b] > 0 asks for that many tokens
 * more, grow[b] < 0 gives the last -grow[b] back (all of them if fewer are
 * held: the request has ended).  In request order
 *   - the pages of table entries pages(new) .. pages(old) - 1 of every
 *     request that shrinks are pushed on the stack of free pages;
 *   - then every request that grows takes what it needs from the stack's top
 *     into its next table entries.
 * A request that asks for more is refused (keeps its length and pages; bit 0
 * of error_flag is set) if its row is too short, if the pages that it and the
 * growing requests before it need (those of too short a row aside) are more
 * than there are and it needs any, or if their tokens are more than max_slots.
 *   seq_len         device int32 [batch]
 *   grow            device int32 [batch]
 *   block_table     device int32 [batch][max_pages], changed in place; entries
 *                   past a request's pages may hold anything
 *   free_pages      device int32 [pages], changed in place: the stack
 *   free_count      device int32 [1]: pages on the stack
 *   slots           device int32 [max_slots]: the place page * 64 + i of every
 *                   new token, request after request; -1 past the last
 *   slot_start      device int32 [batch + 1]: where each request's begin
 *   new_len         device int32 [batch]: the length after the call (may be
 *                   seq_len itself)
 *   new_free_count  device int32 [1] (may be free_count itself)
 *   error_flag      device int32 [1]: bits are set, never cleared; bit 1: a
 *                   length or a count was out of range and clamped
 * With outputs apart from their inputs the call can be repeated and gives the
 * same result: it changes only stack entries from free_count on, and table
 * entries past the pages of old lengths.
 * Requires 0 <= batch <= 2^24, max_pages and pages in 1..2^25 - 1, and
 * 0 <= max_slots <= 2^30.
 */
das_status das_page_assign(const int32_t *seq_len, const int32_t *grow, int batch,
                           int32_t *block_table, int max_pages, int32_t *free_pages, int pages,
                           const int32_t *free_count, int32_t *slots, int max_slots,
                           int32_t *slot_start, int32_t *new_len, int32_t *new_free_count,
                           int32_t *error_flag, void *stream);

/*
 * Commit into a paged cache: the first n_b = slot_start[b + 1] - slot_start[b]
 * of each sequence's W staged tokens are stored at slots[slot_start[b] ..] at
 * every depth and layer (das_page_assign makes both; a sequence's slots run on
 * within a page and start the next page at its first place).
 * For each page, kv head, and keys and values apart: the scale is 2^e with the
 * least e in [-40, 120] such that every finite new element is at most
 * 448 * 2^e in size.  If the page already holds tokens before the first new
 * one, it is the larger of that and its present scale, and the older codes
 * are rounded again where the scale grew (exact unless a code becomes
 * subnormal).  A code is the element / scale rounded to e4m3 (nearest, ties to
 * even, +-448 at most; NaN stays NaN).
 *   k_new, v_new  device bf16 [depths][layers][batch][W][kv_heads][head_dim]
 *   slots         device int32 [max_slots]
 *   slot_start    device int32 [batch + 1]
 *   error_flag    device int32 [1]: bit 1 is set (never cleared) and the page
 *                 left alone where a slot lies outside the cache, a page does
 *                 not start at its first place, or n_b is not in 0..W
 * Sequences do not share the pages that they write.  Requires W >= 1 and
 * batch >= 0 (with 0, k_new and v_new may be NULL; with max_slots 0, slots).
 */
das_status das_kv_append_paged(const das_kv_cache_paged *cache, const void *k_new,
                               const void *v_new, int batch, int W, const int32_t *slots,
                               int max_slots, const int32_t *slot_start, int32_t *error_flag,
                               void *stream);

/* Workspace bytes for das_mature_v_attention_paged (as das_workspace_size). */
size_t das_workspace_size_paged(const das_kv_cache_paged *cache, int batch, int num_q_heads,
                                int max_block);

/*
 * das_mature_v_attention over a paged cache (Eqs. 2-3 on the values that its
 * codes and scales stand for): keys of key_depth, values of value_depth;
 * key_depth = value_depth is the verify attention.  max_block = 1 with
 * block_len 1 is the call for single tokens.
 *   block_table  device int32 [batch][max_pages]; entries past a sequence's
 *                ceil(prefix_len / 64) pages are not read.  The host, which does
 *                not know the lengths, chooses how to split the work by max_pages:
 *                a table much wider than the prefixes can cost some
 *                microseconds, with hundreds of short sequences half as much again
 *   prefix_len   device int32 [batch], 0..64 max_pages
 *   k_blk, v_blk device bf16 [batch][max_block][kv_heads][head_dim]
 * All other arguments, results and limits as das_mature_v_attention.  Bit 2
 * of the workspace's status word is set where a table entry is no page of the
 * cache; its 64 tokens are then taken as masked.
 * The products run on the codes: a query row is split into two e4m3 parts,
 * exactly for elements down to about 2^-13 of the row's largest (queries must
 * be finite), a softmax weight into three e5m2 parts: to 2^-9 of itself, as a
 * bf16 weight is, where weight times value scale is above 2^-21 of the row's
 * largest sum of these over a page, below to 2^-6 of itself or 2^-30 of that sum.
 * Scores, sums and outputs are accumulated in fp32.  The value scales that one
 * sequence reads are to be within a factor of 2^100 of each other and of 1 (a
 * scale of 0 counts as 2^-60).
 */
das_status das_mature_v_attention_paged(const das_kv_cache_paged *cache, int layer, int key_depth,
                                        int value_depth, const int32_t *block_table, int max_pages,
                                        const int32_t *prefix_len, const int32_t *block_len,
                                        int batch, int max_block, const void *q, const void *k_blk,
                                        const void *v_blk, int num_q_heads, float softmax_scale,
                                        void *out, float *lse, void *workspace,
                                        size_t workspace_bytes, void *stream);

typedef enum { DAS_LOGITS_F32 = 0, DAS_LOGITS_BF16 = 1 } das_logits_type;

/* Sampling parameters, each device memory of one value per sequence, or NULL. */
typedef struct {
    const float *temperature; /* NULL: 1; <= 0 or NaN: greedy (the first maximum) */
    const int32_t *top_k;     /* NULL or <= 0: all tokens                         */
    const float *top_p;       /* NULL, >= 1 or NaN: all tokens                    */
    const float *min_p;       /* NULL, <= 0 or NaN: all tokens; 1 at most         */
} das_sampling;

/*
 * One token drawn from every row of logits with the row's random number.
 * With m the row's largest logit l_v (NaN counts as -inf) and T the
 * temperature,
 *   e_v = 1 if l_v = m, 0 if l_v = -inf, else exp((l_v - m) / T) in binary32,
 *   w_v = e_v * 2^32 rounded to a whole number,
 * tokens ordered by logit, largest first, equal ones by index:
 *   top-k keeps the first top_k tokens,
 *   top-p keeps the least number of those (one at least) whose w sum to at
 *         least ceil(top_p * S), S the sum over what top-k kept,
 *   min-p keeps those of them with e_v >= min_p.
 * With R the sum of the kept w, the token is the least index v for which the
 * kept w up to and including v sum to more than floor(u R) (products in
 * binary64; u is clamped to [0, 1)), and its logprob (l_v - m) / T -
 * ln(R / 2^32).  Greedy rows keep the first token alone.  All sums are of
 * whole numbers, so the result does not depend on their order.  A row with no
 * logit above -inf gives token -1 and logprob -inf.
 *   logits    device fp32 or bf16, row (b, i) at element
 *             (b * W + i) * row_stride, row_stride >= vocab
 *   uniforms  device fp32 [B][W], in [0, 1)
 *   tokens    device int32 [B][W]
 *   logprobs  device fp32 [B][W], or NULL
 * Requires B >= 0 (with 0 the tensors may be NULL), 1 <= W <= 1024,
 * 1 <= vocab < 2^31.
 */
das_status das_sample(const void *logits, das_logits_type type, int B, int W, int vocab,
                      long long row_stride, const das_sampling *sampling, const float *uniforms,
                      int32_t *tokens, float *logprobs, void *stream);

/*
 * Sampled acceptance of proposals that a drafter made without chance (as
 * DAS drafting does): target_ids[b][i] is drawn from logits[b][i] as
 * das_sample draws it, and proposals are accepted while they equal it, so
 * that every emitted token is a draw from the target's own (truncated)
 * distribution.  accepted, target_ids and next_token as das_greedy_accept;
 *   committed  device int32 [B], or NULL: min(accepted + 1, W), the verifier
 *              inputs to commit (grow of das_page_assign)
 * At temperature 0 it is das_greedy_accept, except that a row with no logit
 * above -inf gives -1, which no proposal equals.
 */
das_status das_sample_accept(const void *logits, das_logits_type type, const int32_t *draft_ids,
                             int B, int W, int vocab, long long row_stride,
                             const das_sampling *sampling, const float *uniforms,
                             int32_t *accepted, int32_t *target_ids, int32_t *next_token,
                             int32_t *committed, float *logprobs, void *stream);

/* Static text for a status code. */
const char *das_status_string(das_status s);

#ifdef __cplusplus
}
#endif

#endif /* DAS_H */
