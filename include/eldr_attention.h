/*
 * eldr_attention.h -- the attention half of a decode step over the paged KV
 * cache, for MI355X (gfx950): what a decode worker runs beside the MoE layer
 * of eldr_moe.h.
 *
 *   moe_kv_append     rotary positions of the new tokens' queries and keys
 *                     (one position axis or several), and the write of their
 *                     keys and values into the cache's pages
 *   moe_attn_decode   attention of one query token a request over its cached
 *                     tokens; a prefix that requests share is read once for
 *                     all of them
 *   moe_attn_weights  the attention weight each cached token received, added
 *                     to what it has accumulated
 *   moe_kv_evict      the tokens of largest accumulated weight stay, the rest
 *                     leave, and the cache is compacted in place
 *
 * Requests that a locality router places together share their domain's prompt
 * prefix, and with prefix caching they share its pages as well (Design,
 * Prefix Cache Coherence); a request's pages are listed in the same int32
 * block table that moe_sig_request_counts reads.
 *
 * Same conventions as eldr_moe.h: plain device pointers, sizes and a
 * hipStream_t passed as void*; the caller owns every buffer; calls are
 * asynchronous on `stream`, allocate nothing, keep no state, never
 * synchronise and can be captured in a graph; they return MOE_OK or a
 * negative MOE_ERR_* code (eldr_moe.h) before any launch.  Queries, keys,
 * values, outputs of attention, caches, rotation tables and the workspace are
 * 16-byte aligned; every other array (lse, sinks, scales, accumulated weights,
 * int32) 4-byte.
 *
 * The cache
 * ---------
 * k_cache and v_cache each hold, for page b < num_blocks, kv head h < Hkv and
 * offset o < block_size, one row of D values, at element
 *
 *   b * block_stride + (h * block_size + o) * D
 *
 * (block_stride 0 stands for the dense Hkv * block_size * D; a larger one, a
 * multiple of 16, lets keys and values, or layers, interleave in one allocation).  Offsets are
 * computed in 64 bits.  kv_type MOE_KV_BF16: values are bf16.  MOE_KV_FP8:
 * values are OCP e4m3 codes that stand for code * scale[h], with k_scale and
 * v_scale [Hkv] fp32 device arrays (NULL: all 1); ignored for bf16.
 *
 * Token slot j of request r lies in page block_table[r, j / block_size] at
 * offset j % block_size.  A slot whose page is outside [0, num_blocks) is
 * absent: it is not read, and counts as masked.  lens[r] tokens are cached;
 * it is taken as clamped to [0, N], N = max_blocks * block_size, and as 0 where
 * num_blocks is 0.  What pages hold past lens[r] is never used, whatever its
 * bits are.
 *
 * Groups that share a prefix
 * --------------------------
 * group_start [n_groups + 1] and prefix_len [n_groups] (int32, on the device):
 * requests group_start[g] .. group_start[g + 1] - 1 hold the same tokens in
 * slots [0, prefix_len[g]), and those are read through the block table row of
 * the group's first request that holds anything (lens > 0), once for the group.
 * (The slots are shared as far as the shortest non-empty member reaches; past
 * that, and in a group of one, each request reads its own row.  An empty
 * member's row is not read.)  group_start must not descend; it is taken
 * as clamped to [0, R], and requests outside every group share nothing.
 * n_groups = 0: nothing is shared and both pointers may be NULL; more than
 * MOE_ATTN_MAX_R is MOE_ERR_INVALID.
 */
#ifndef ELDR_ATTENTION_H_
#define ELDR_ATTENTION_H_

#include <stddef.h>
#include <stdint.h>

#include "eldr_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What the caches hold. */
#define MOE_KV_BF16 0
#define MOE_KV_FP8 1

/* What moe_kv_append's q, k and v are. */
#define MOE_IN_BF16 0
#define MOE_IN_FP32 1

/* Limits.  D is 64, 128 or 256; Hkv divides Hq; block_size is a power of two. */
#define MOE_ATTN_MAX_R 1024 /* requests, and groups */
#define MOE_ATTN_MAX_HEADS 256
#define MOE_ATTN_MIN_BLOCK 16
#define MOE_ATTN_MAX_BLOCK 1024
#define MOE_ATTN_MAX_TOKENS (1 << 19) /* max_blocks * block_size */
#define MOE_ATTN_MAX_APPEND (1 << 20)
#define MOE_ATTN_MAX_AXES 8

/* One attention layer's shape: R requests, Hq query heads over Hkv kv heads
 * of D values, and the paged cache. */
typedef struct moe_attn_dims {
  int32_t R, Hq, Hkv, D;
  int32_t block_size, max_blocks, num_blocks, kv_type;
  int64_t block_stride;
} moe_attn_dims;

/*
 * moe_kv_append -- rotate the T new tokens' queries and keys by their
 * positions and store keys and values (d.R and d.max_blocks are checked as for
 * the other calls, and not used).
 *
 *   for pair i < rot / 2 of token t, with a = pair_axis[i]:
 *     C = cos_table[positions[a, t], i], S = sin_table[positions[a, t], i]
 *     x'[lo] = x[lo] C - x[hi] S,  x'[hi] = x[hi] C + x[lo] S
 *     (lo, hi) = (i, i + rot / 2), or (2 i, 2 i + 1) if interleaved != 0
 *   values from rot on are copied; q_out[t, h] = bf16(q'), and with
 *   s = slots[t] >= 0 the cache's slot s (page s / block_size, offset
 *   s % block_size) becomes k' and v, as bf16 or as e4m3 of value / scale[h],
 *   clamped to +-448 (round to nearest even).
 *
 * The products and the sum are each rounded to fp32, in that order.
 * q [T, Hq, D], k, v [T, Hkv, D]: bf16 or fp32 (in_type), each with its own
 * token stride in elements (a multiple of 8), heads and values contiguous, so
 * that the rows of one fused projection can be passed as they are.
 * positions [n_axes, T] int32; pair_axis [rot / 2] int32 (text: one axis, all
 * zeros; images and video: the axis, of time, height and width, whose position
 * turns the pair, in any order); cos_table, sin_table [max_pos, rot / 2] fp32.
 * A position outside [0, max_pos), or an axis outside [0, n_axes), makes the
 * pair's values NaN.  A slot that is negative is not stored (the token's k and
 * v are dropped), nor is one in a page past num_blocks.  Slots of one call are
 * distinct.  rot is a multiple of 16, 0 <= rot <= D (0: nothing is rotated).
 * q_out [T, Hq, D] bf16, dense; it may be NULL (with q) where only keys and
 * values are wanted.
 */
int moe_kv_append(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride,
                  int64_t v_stride, int32_t in_type, int32_t T, const int32_t* positions,
                  int32_t n_axes, const int32_t* pair_axis, const float* cos_table,
                  const float* sin_table, int32_t max_pos, int32_t rot, int32_t interleaved,
                  const int32_t* slots, moe_attn_dims d, const float* k_scale,
                  const float* v_scale, uint16_t* q_out, void* k_cache, void* v_cache,
                  void* stream);

/*
 * moe_attn_decode -- attention of each request's one query token.
 *
 *   s_j = scale * q[r, h] . k_j,  over the cached slots j of r that are
 *         visible: j < lens[r], and j >= lens[r] - window if window > 0
 *   lse[r, h] = log(sum_j exp(s_j) + exp(sinks[h]))     (no sink: sinks NULL)
 *   out[r, h] = sum_j exp(s_j - lse) v_j
 *
 * Query head h reads kv head h / (Hq / Hkv).  q, out [R, Hq, D] bf16; lse
 * [R, Hq] fp32 (NULL: not wanted); sinks [Hq] fp32 or NULL.  A request with no
 * visible slot, or none whose score is above -inf, gets out = 0 and lse = -inf,
 * or the sink's value; a sink of -inf weighs nothing.  A NaN that counts (in a
 * query, a visible row or a sink) gives NaN.  Where window > 0 no prefix is
 * shared.  Scores, statistics and sums are fp32; a weight enters the product with
 * v in two bf16 parts, 16 bits of it, so that out's error is that of its own
 * rounding.  The result does not depend on anything but the arguments' values (no
 * atomics on floats); how a long request is split depends on the whole batch's
 * lengths, so a request's last bits may differ between batches.
 * ws: moe_attn_workspace_bytes(d) bytes, 16-byte aligned, whose contents mean
 * nothing between calls: one workspace serves every layer on a stream.
 */
size_t moe_attn_workspace_bytes(moe_attn_dims d);
int moe_attn_decode(const uint16_t* q, const void* k_cache, const void* v_cache,
                    const int32_t* block_table, const int32_t* lens, const int32_t* group_start,
                    const int32_t* prefix_len, int32_t n_groups, const float* k_scale,
                    const float* v_scale, const float* sinks, int32_t window, float scale,
                    moe_attn_dims d, uint16_t* out, float* lse, void* ws, size_t ws_bytes,
                    void* stream);

/*
 * moe_attn_weights -- the attention weight of every cached token, summed over
 * the query heads that read its kv head:
 *
 *   weights_out[r, h, j] = weights_in[r, h, j]
 *                        + sum over query heads i of kv head h of
 *                          exp(scale * q[r, i] . k_j - lse[r, i])
 *
 * for the slots j < lens[r]; other slots are not written (an absent one gets
 * weights_in).  lse as moe_attn_decode wrote it, for the same arguments and no
 * window.  weights_in, weights_out [R, Hkv, N] fp32; weights_in may be NULL
 * (zeros) or weights_out itself.
 */
int moe_attn_weights(const uint16_t* q, const void* k_cache, const int32_t* block_table,
                     const int32_t* lens, const int32_t* group_start, const int32_t* prefix_len,
                     int32_t n_groups, const float* k_scale, float scale, const float* lse,
                     moe_attn_dims d, const float* weights_in, float* weights_out, void* stream);

/*
 * moe_kv_evict -- cut every request with more than `budget` cached tokens to
 * `budget`, kv head by kv head.  For request r and kv head h, n = lens[r]:
 *
 *   slot j is protected if j < protect[r] (NULL: 0), or if its token is one of
 *   the last: pos[r, h, j] >= seen[r] - recent (seen[r]: tokens the request
 *   has had so far; pos: the position of the token in each slot)
 *   the budget slots that come first stay, in the order: protected before
 *   others, larger weight first, lower slot first (a weight that is NaN comes
 *   last; protected slots rank by slot alone)
 *   slots >= budget that stay move, in ascending order, into the slots below
 *   budget that leave, in ascending order; every other slot keeps its place
 *
 * Requests are expected to own the pages of slots >= protect[r]: a shared
 * prefix is protected, and protected slots below budget never move.
 * weights [R, Hkv, N] fp32, pos [R, Hkv, N] int32, lens, seen, protect [R]
 * int32 (inputs).  Outputs:
 *   k_cache, v_cache  the moved rows, in place
 *   src [R, Hkv, budget]  the slot that each slot's token was in (itself where
 *                     it stayed), -1 from n on
 *   new_lens [R]      min(lens, budget); not lens itself
 *   weights_out, pos_out [R, Hkv, N]  as moved; 0 and -1 in [new_lens, n);
 *                     slots from n on are not written.  They may be weights
 *                     and pos themselves.
 * Order does not matter to attention without a window, whose keys carry their
 * positions, so nothing else has to move: one token over the budget costs one
 * row.  A row whose page is absent is not moved.  d.Hq and block_table as
 * above; 1 <= budget <= MOE_ATTN_MAX_TOKENS and R * Hkv <= 65535 (else
 * MOE_ERR_UNSUPPORTED).
 */
int moe_kv_evict(const float* weights, const int32_t* pos, const int32_t* lens,
                 const int32_t* seen, const int32_t* protect, const int32_t* block_table,
                 moe_attn_dims d, int32_t budget, int32_t recent, void* k_cache, void* v_cache,
                 int32_t* src, int32_t* new_lens, float* weights_out, int32_t* pos_out,
                 void* stream);

#ifdef __cplusplus
}
#endif

#endif  /* ELDR_ATTENTION_H_ */
