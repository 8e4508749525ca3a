/*
 * eldr_kv_cache.h -- more of the paged KV cache of eldr_attention.h, for
 * MI355X (gfx950).
 *
 *   moe_kv_append_norm  moe_kv_append with queries and keys normed head by head
 *                       before they are turned
 *   moe_kv_append_int8  the same, norms or none, into a cache of 8-bit integers
 *                       with a scale for each page and kv head
 *   moe_kv_fork         copies of requests: they share the full pages and get
 *                       the last, partly filled one for themselves
 *   moe_kv_compact      live pages move into free ones, block tables follow
 *
 * Same conventions as eldr_attention.h.
 *
 * The cache of 8-bit integers (kv_type MOE_KV_INT8)
 * --------------------------------------------------
 * Values are signed codes, laid out as in the other caches, that stand for
 * code * scale[page, h]: k_scale and v_scale are [num_blocks, Hkv] fp32 device
 * arrays, which moe_kv_append_int8 writes and moe_attn_decode reads.  They are
 * not optional for this type.  A page's scale holds for all of its slots, so a
 * page that receives tokens belongs to one request (moe_kv_fork sees to that).
 * moe_kv_append and moe_kv_append_norm (which know slots, not pages),
 * moe_attn_weights and moe_kv_evict (a row would move under another page's
 * scale) return MOE_ERR_UNSUPPORTED for it.
 */
#ifndef ELDR_KV_CACHE_H_
#define ELDR_KV_CACHE_H_

#include <stddef.h>
#include <stdint.h>

#include "eldr_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits. */
#define MOE_KV_MAX_FORKS 65535
#define MOE_KV_MAX_LAYERS 1024

/*
 * moe_kv_append_norm -- moe_kv_append, with x the values of one head of a query
 * or a key first replaced by
 *
 *   (x * i) * w,   i = 1 / sqrt(mean of x^2 over the head's D values + eps)
 *
 * The mean and i are computed in 64 bits; i, and each of the two products, is
 * rounded to fp32.  w: q_norm for queries, k_norm for keys, [D] fp32, 16-byte
 * aligned; NULL: that side is not normed.  eps: finite, >= 0.  All other
 * arguments as for moe_kv_append, whose results it gives where both are NULL.
 */
int moe_kv_append_norm(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride,
                       int64_t v_stride, int32_t in_type, int32_t T, const int32_t* positions,
                       int32_t n_axes, const int32_t* pair_axis, const float* cos_table,
                       const float* sin_table, int32_t max_pos, int32_t rot, int32_t interleaved,
                       const int32_t* slots, moe_attn_dims d, const float* q_norm, const float* k_norm,
                       float eps, const float* k_scale, const float* v_scale, uint16_t* q_out,
                       void* k_cache, void* v_cache, void* stream);

/*
 * moe_kv_append_int8 -- the new tokens of R requests: norms (or none) and
 * rotation as above, queries to bf16, keys and values into pages of 8-bit
 * integers.
 *
 * Tokens query_start[r] .. query_start[r + 1] - 1 (int32 [R + 1], on the device,
 * not descending, taken as clamped to [0, T]) are request r's; they go to its
 * cache slots lens[r], lens[r] + 1, ... (lens: what it holds before, taken as
 * clamped to [0, N]; the call does not change it).  For each page that receives
 * tokens and each kv head, of keys and of values apart, with a the largest
 * absolute value of the new tokens' rows:
 *
 *   no slot of the page is held (its first new slot is at offset 0), or its
 *   scale is 0:   scale' = a * (1 / 127)   (both rounded to fp32)
 *   else:         scale' = scale * 2^n, n >= 0 the smallest with
 *                 127 * scale' >= a; the held slots' codes become
 *                 round(code * 2^-n)
 *   new codes:    round(x / scale'), clamped to +-127; 0 where scale' is 0
 *
 * (Round to nearest even.  A scale grows by powers of two so that a held value
 * never ends up more than one step of the page's last scale off, however often
 * it grew.  127 scale is compared exactly: rounding may leave it below the value
 * that set the scale, and a later row as large then doubles it.)  Where a, or a
 * held page's scale, is not finite, scale' is NaN: the page and head stand for NaN,
 * as a NaN stored in the other caches would.
 * Held slots of a page whose scale was 0 become codes of 0.
 *
 * What is not stored: tokens past slot N, and those whose page is absent.  Tokens
 * of no request (padding behind query_start[R]) are dropped, and their rows of
 * q_out are left as they are.  Pages that receive tokens are distinct: for
 * distinct requests, and for distinct places of a request's row.  Slots past the new
 * tokens are left as they are.
 */
int moe_kv_append_int8(const void* q, const void* k, const void* v, int64_t q_stride, int64_t k_stride,
                       int64_t v_stride, int32_t in_type, int32_t T, const int32_t* positions,
                       int32_t n_axes, const int32_t* pair_axis, const float* cos_table,
                       const float* sin_table, int32_t max_pos, int32_t rot, int32_t interleaved,
                       const int32_t* query_start, const int32_t* block_table, const int32_t* lens,
                       moe_attn_dims d, const float* q_norm, const float* k_norm, float eps,
                       uint16_t* q_out, void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                       void* stream);

/*
 * moe_kv_fork -- request child[i] becomes a copy of request parent[i], i < F.
 * With n = lens[parent] (clamped to [0, N]), full = n / block_size and
 * rest = n % block_size:
 *
 *   block_table[child, j] = block_table[parent, j] for j < full, -1 behind
 *   rest > 0: block_table[child, full] = page[i], and slots [0, rest) of that
 *   page become those of the parent's page, keys and values of every kv head,
 *   in every layer (with the page's scales for MOE_KV_INT8)
 *   lens[child] = n
 *
 * parent, child, page: int32 [F], on the device.  A fork whose parent or child
 * is outside [0, R), or whose child is its parent, does nothing.  Where page[i],
 * or the parent's last page, is absent, the entry becomes -1 and the slots
 * absent.  Children are distinct and no parents of the same call; pages are
 * distinct and held by no request.  A parent may have several children.
 *
 * layers: caches of all layers, layer l's keys at element l * layer_stride of
 * k_cache, values of v_cache (layer_stride a multiple of 16, at least what a
 * layer's pages take up unless layers interleave in the block stride; 0: dense,
 * num_blocks * block stride); its scales, [num_blocks, Hkv], at l * num_blocks *
 * Hkv of k_scale and v_scale (NULL, and ignored, but for MOE_KV_INT8).  The
 * block table is the same for all layers.
 */
int moe_kv_fork(const int32_t* parent, const int32_t* child, const int32_t* page, int32_t F,
                int32_t* block_table, int32_t* lens, moe_attn_dims d, int32_t layers,
                int64_t layer_stride, void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                void* stream);

/*
 * moe_kv_compact -- page b moves to page remap[b], and block tables follow.
 *
 *   remap[b] == b:                      the page stays
 *   remap[b] outside [0, num_blocks):   the page is free (no longer held)
 *   else, to = remap[b], a free page:   keys, values and scales of page b, in
 *                                       every layer, are copied to page `to`
 *   else (`to` is not free):            the page stays
 *   table_out[r, j] = where page block_table[r, j] is now; -1 where it is free,
 *   or absent
 *
 * remap int32 [num_blocks], on the device.  Distinct pages move to distinct
 * pages.  table_out [R, max_blocks] may be block_table itself.  Layers and
 * scales as for moe_kv_fork.  What moved pages hold afterwards is what they held
 * before.
 */
int moe_kv_compact(const int32_t* remap, const int32_t* block_table, int32_t* table_out,
                   moe_attn_dims d, int32_t layers, int64_t layer_stride, void* k_cache,
                   void* v_cache, float* k_scale, float* v_scale, void* stream);

#ifdef __cplusplus
}
#endif

#endif  /* ELDR_KV_CACHE_H_ */
