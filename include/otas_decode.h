/*
 * otas_decode.h -- C ABI of the operators with which a decoder reads the encoder's output on AMD MI355X (gfx950):
 * rotary positions, masked attention over packed rows, a key/value cache of fixed capacity, attention of drafted
 * tokens over it, and eviction from it by accumulated attention weight.
 *
 * The conventions are those of otas.h: contexts, streams, errors, host and dev pointers.  In addition:
 *   - H, d_h = D / H and the element type are the context's; its layers' weights are not read.  d_h is any multiple of 4 up
 *     to 128.  kv_heads divides H: head h reads key / value head h / (H / kv_heads).
 *   - Packed rows: qkv dev [T, (H + 2 kv_heads) d_h], a row's query heads, then its key heads, then its value heads
 *     (with kv_heads = H the rows of otas_attention).  Query q owns rows offsets[q] .. offsets[q+1]-1; it may own none.
 *   - Every dev pointer must be aligned to 16 bytes (EINVAL), arrays of 4-byte elements to 4.
 *   - The device that was current stays current.
 *   - Host numbers travel in the kernels' arguments while they are at most OTAS_DECODE_ARGUMENTS 4-byte entries (each
 *     entry point says how many it has), else through the context's plan buffer.  Calls of the first kind may be captured into a
 *     HIP graph (their host numbers are part of it); of the second kind they are refused under capture (EUNSUPPORTED), and
 *     limited to 1048576 entries (ENOMEM).
 *   - A call whose launch would have 2^24 workgroups or more is refused (EUNSUPPORTED): 2^27 rows of otas_rotary, 2^24 of
 *     otas_cache_append, attention over very many queries of which one is very long (all are given as many workgroups as the longest).
 *     otas_cache_evict has a limit of its own.
 *   - Results do not depend on the order in which the device happens to run anything.
 */
#ifndef OTAS_DECODE_H_
#define OTAS_DECODE_H_

#include "otas.h"

#ifdef __cplusplus
extern "C" {
#endif

#define OTAS_DECODE_ARGUMENTS 960
#define OTAS_MAX_LONG_SEQ 1048576  /* rows of a query, entries of a cache slot */
#define OTAS_MAX_TREE_NODES 64

/* Rotary positions: the first rot_dim elements of every query and key head are turned in pairs, pair i of a row at position
 * p by the angle p f_i (inverse != 0: by -p f_i, which undoes it and is its gradient), times magnitude:
 *   (a, b) -> magnitude (a cos - b sin, a sin + b cos),   f_i = base^(-2 i / rot_dim), i < rot_dim / 2, and by scaling
 *   OTAS_ROTARY_PLAIN     f_i
 *   OTAS_ROTARY_LINEAR    f_i / factor
 *   OTAS_ROTARY_BASE      base base factor^(rot_dim / (rot_dim - 2)) in place of base (rot_dim >= 4)
 *   OTAS_ROTARY_BY_PARTS  w f_i + (1 - w) f_i / factor,  w = (original_length f_i / (2 pi) - slow_turns) / (fast_turns - slow_turns)
 *                         held to [0, 1]: pairs that turn often within the original length keep their pace
 *   layout  OTAS_ROTARY_HALF pair i = elements (i, i + rot_dim / 2), OTAS_ROTARY_INTERLEAVED (2 i, 2 i + 1)
 * Angles are formed in 64 bits and reduced there, so that far positions lose nothing.  A description whose base or angles do not fit
 * 64 bits is refused (EINVAL).
 *   positions dev int32 [T], any value;  out dev [T, (H + 2 kv_heads) d_h], may be qkv (then only what turns is written), else no
 *   overlap.  rot_dim even, 0 .. d_h (0: a copy).  No host numbers. */
enum { OTAS_ROTARY_HALF = 0, OTAS_ROTARY_INTERLEAVED = 1 };
enum { OTAS_ROTARY_PLAIN = 0, OTAS_ROTARY_LINEAR = 1, OTAS_ROTARY_BASE = 2, OTAS_ROTARY_BY_PARTS = 3 };
typedef struct {
  int32_t rot_dim, layout, scaling, inverse;
  double base;             /* > 0 */
  double factor;           /* > 0; not read by PLAIN */
  double original_length;  /* > 0, BY_PARTS only, as the next two: fast_turns > slow_turns */
  double fast_turns, slow_turns;
  double magnitude;        /* finite, not 0 */
} otas_rotary_desc;
otas_status otas_rotary(otas_ctx *ctx, const void *qkv, int64_t T, int32_t kv_heads, const int32_t *positions,
                        const otas_rotary_desc *rope, void *out);

/* How products become logits, for both attentions below.  s = scale (q . k); where cap > 0, s = cap tanh(s / cap); then, where
 * slopes are given, s - slopes[h] |position_i - position_j|. */
typedef struct {
  float scale;          /* finite; 0 = 1 / sqrt(d_h) */
  float cap;            /* finite, >= 0; 0 = none.  For the cap a bf16 logit is off by up to 1e-6 cap, or 4e-6 of itself where cap > 256.
                         * scale / cap up to 1e38 (EINVAL) */
  const float *slopes;  /* dev [H] or NULL */
} otas_score_desc;

/* Attention over packed rows: o[i] = sum over the keys j that row i sees of softmax(s)_j v_j, heads concatenated.
 * Row i sees row j of its query if neither is padding and
 *   j < prefix[q], or document_i == document_j and (not causal or j <= i)          (i, j counted within the query).
 *   prefix    host [B], 0 <= prefix[q] <= the query's rows, or NULL (none)
 *   documents dev int32 [T] or NULL (a query is one document); a negative number marks padding
 *   positions dev int32 [T] or NULL (i, j themselves): for the distance only; within +- 2^29
 *   score     NULL = all defaults
 *   o         dev [T, D], no overlap with any other array.  A row that sees nothing, or no key of weight, is zero.
 *   Logits, weights and sums are float.  bf16 models with d_h of 64, 80, 96 or 128 round each weight to bf16 (by 2^-8 of itself at most)
 *   before it meets its value; the weights' sum takes them unrounded.  The same goes for otas_attention_tree.
 * Keys and values that a row does not see do not reach it, infinities and NaN included.
 * Lengths up to OTAS_MAX_LONG_SEQ (EUNSUPPORTED).  Host numbers: 2 B + 1. */
otas_status otas_attention_masked(otas_ctx *ctx, const void *qkv, int32_t kv_heads, const int32_t *offsets, int32_t B,
                                  int32_t causal, const int32_t *prefix, const int32_t *documents, const int32_t *positions,
                                  const otas_score_desc *score, void *o);

/* A cache: `slots` places for one query each, of `capacity` entries.  An entry is a token's key and value heads, its position
 * and the attention weight that it has gathered.  The caller owns the memory and knows which query has which slot and how many
 * entries of it are filled (they are entries 0 .. length - 1; those behind are neither read nor written, except where a call
 * says so).  The four arrays overlap neither each other nor any other array of a call (EINVAL where k and v are one, or the call's
 * qkv, o or workspace has a byte in common with k or v; the others are not looked at). */
typedef struct {
  void *k, *v;         /* dev [slots, kv_heads, capacity, d_h], model dtype */
  int32_t *positions;  /* dev [slots, capacity] */
  float *mass;         /* dev [slots, capacity] or NULL */
  int32_t slots, kv_heads, capacity;
} otas_kv_cache;

/* Puts rows behind the entries of their query: the key and value heads of row rows[i] (NULL: of row i), i = row_offsets[q] ..
 * row_offsets[q+1] - 1, become entries length[q], length[q] + 1, .. of slot[q], with positions[rows[i]] and mass 0.
 *   qkv dev [T, ..], positions dev int32 [T]; rows host [row_offsets[B]] or NULL, 0 <= rows[i] < T (EINVAL)
 *   slot, length host [B]; the slots of a call differ from each other, and the rows fit in behind the entries (EINVAL)
 *   length_out host [B], filled on return.   Host numbers: 3 B + 1, and with rows row_offsets[B] more. */
otas_status otas_cache_append(otas_ctx *ctx, const otas_kv_cache *cache, const void *qkv, int64_t T, const int32_t *row_offsets,
                              const int32_t *rows, const int32_t *positions, const int32_t *slot, const int32_t *length,
                              int32_t B, int32_t *length_out);

/* Attention of drafted tokens, nodes of a tree, over their query's cache: node i of query q sees every entry of the cache,
 * itself, its parent, its parent's parent and so on, and no other node.  One token after the cache is a tree of one node; a
 * run of tokens is a chain.  The nodes' keys and values are taken from qkv (otas_cache_append puts those that are accepted into
 * the cache afterwards).
 *   qkv dev [T, (H + 2 kv_heads) d_h], kv_heads the cache's;  offsets host [B+1]: at most OTAS_MAX_TREE_NODES rows a query
 *   (EUNSUPPORTED)
 *   parents host [T]: for every node the parent's index within the query, smaller than its own (EINVAL), or -1; NULL = chains
 *   positions dev int32 [T] or NULL, read where score has slopes (then required); within +- 2^29, as the cache's
 *   slot, length host [B].  With add_mass the slots of a call differ from each other (EINVAL)
 *   add_mass != 0: entry j's mass grows by the weights it got, summed over the query's nodes and all heads (cache->mass required)
 *   workspace dev >= otas_attention_tree_workspace_bytes for the same offsets, length and add_mass, 256-byte aligned.  The bytes
 *   grow with the lengths; with add_mass there may be 4 for every row, head and entry among them
 *   o dev [T, D]; o and the workspace overlap no other array.  A node without a key of weight is zero.   Host numbers: 3 B + 1, with parents T / 4 more.
 * The split of a long cache between workgroups, and with it the last bits of o, depends on the whole call's lengths. */
size_t otas_attention_tree_workspace_bytes(const otas_ctx *ctx, int32_t kv_heads, const int32_t *offsets, const int32_t *length,
                                           int32_t B, int32_t add_mass);
otas_status otas_attention_tree(otas_ctx *ctx, const otas_kv_cache *cache, const void *qkv, const int32_t *offsets,
                                const int32_t *parents, const int32_t *positions, const int32_t *slot, const int32_t *length,
                                int32_t B, const otas_score_desc *score, int32_t add_mass, void *workspace,
                                size_t workspace_bytes, void *o);

/* Cuts caches down to keep[q] entries.  Entries are ranked: first those that are protected (entry < lead, or position >=
 * recent_from[q]), which are alike whatever their mass, then the others by mass, largest first (NaN counts as least); ties go to the
 * lower entry.  (So where more are protected than keep[q], the lowest of them stay.)  The first keep[q] stay: an entry
 * below keep[q] that stays does not move, and the j-th that stays from above takes, with position and mass, the place of
 * the j-th below that goes (so no more is moved than has to be, and entries are in no order afterwards).  Entries from keep[q]
 * on are left as they were.
 *   slot, length, keep host [B], slots differ from each other, keep >= 0 (keep >= length: nothing happens)
 *   recent_from host [B] or NULL (none protected by position);  lead >= 0
 *   workspace dev >= otas_cache_evict_workspace_bytes for the same numbers, 256-byte aligned; cache->mass required
 *   length_out host [B] = min(length, keep), filled on return.   Host numbers: 5 B.
 *   Up to 65535 queries, whose min(keep, length - keep) add up to less than 2^30 - B / 2 (EUNSUPPORTED). */
size_t otas_cache_evict_workspace_bytes(const otas_ctx *ctx, const int32_t *length, const int32_t *keep, int32_t B);
otas_status otas_cache_evict(otas_ctx *ctx, const otas_kv_cache *cache, const int32_t *slot, const int32_t *length,
                             const int32_t *keep, int32_t B, int32_t lead, const int32_t *recent_from, void *workspace,
                             size_t workspace_bytes, int32_t *length_out);

#ifdef __cplusplus
}
#endif
#endif /* OTAS_DECODE_H_ */
