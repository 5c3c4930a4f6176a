/*
 * otas_decode.h -- C ABI of the operators with which a decoder reads the encoder's output on AMD MI355X (gfx950):
 * rotary positions, also with norms of the heads, masked and windowed attention over packed rows, a key/value cache of fixed
 * capacity, attention of drafted tokens over it, eviction from it by accumulated attention weight, attention of its last tokens
 * through a window, and all of the latter with the cache held in 4 bits.
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
 *   - A call whose launch would have 2^24 workgroups or more is refused (EUNSUPPORTED): 2^27 rows of otas_rotary, 2^26 of otas_norm_rotary,
 *     attention over very many queries of which one is very long.  (otas_attention_masked and otas_attention_tree give all queries as many
 *     workgroups as the longest; the attentions with a window do so where three quarters of those have rows, or where their host
 *     numbers leave no room for B + 1 more, with which they count the queries' workgroups one by one.)  2^24 rows of otas_cache_append, otas_cache4_append or otas_cache4_read are
 *     refused too, and otas_cache_evict has a limit of its own.
 *   - Attention adds up weighted values in float before it divides by the weights' sum, and weights may be up to 2^8 there.  Finite
 *     values of a row's keys beyond 1e30 are not for these entry points: up to there no sum of 2^20 of them passes the largest
 *     float, beyond it o may be infinite or NaN although the mean is a float.  (A cache in 4 bits holds, and reads, up to 6 2^125.)
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
                         * Which of two forms of that accuracy a row's logits take hangs on those of the rows that are worked on with it, and in
                         * otas_attention_masked also on keys of theirs that no row sees.
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

/* Norms of query and key heads with rotary positions in the same pass: every query head x of d_h elements becomes
 *   y = (x - c) r gain,   r = 1 / sqrt(mean((x - c)^2) + eps),   c = mean(x) where center != 0, else 0,
 * every key head the same with its own gain, and y is turned as otas_rotary turns it (rot_dim 0: not at all).  Values stay as they are.
 *   q_gain, k_gain dev, model dtype, [d_h], with per_head != 0 [H, d_h] and [kv_heads, d_h], or NULL (ones)
 *   eps finite, > 0 (EINVAL).  Means, norms and rotation are float, rounded once; heads of elements beyond 1e18, whose squares' sum
 *   is no float, are not for this entry point.
 *   positions may be NULL where rot_dim is 0.  out may be qkv (then only query and key heads are written), else no overlap; the gains overlap
 *   no part of out (EINVAL).  No host numbers. */
typedef struct {
  const void *q_gain, *k_gain;
  float eps;
  int32_t center, per_head;
} otas_head_norm_desc;
otas_status otas_norm_rotary(otas_ctx *ctx, const void *qkv, int64_t T, int32_t kv_heads, const otas_head_norm_desc *norm,
                             const int32_t *positions, const otas_rotary_desc *rope, void *out);

/* Attention over packed rows through a sliding window, with first tokens that stay visible: row i of a query sees row j of it where
 *   j <= i  and  (i - j < window or j < sinks)                                         (i, j counted within the query),
 * so at least itself.  window >= 1 (EINVAL), INT32_MAX or anything past the longest query: all rows before it (for which
 * otas_attention_masked with its defaults is the faster call in bf16 at d_h = 64, by a tenth);  sinks >= 0.
 * score, o, what infinities and NaN in rows that are not seen do (nothing), lengths as in otas_attention_masked; the distance for slopes is
 * i - j.  Keys that no row of a workgroup sees are read only where they share a tile, of 32 or 64 keys, with one that some row does.
 * rows of a query (H / kv_heads) < 2^30 (EUNSUPPORTED).  Host numbers: B + 1. */
otas_status otas_attention_window(otas_ctx *ctx, const void *qkv, int32_t kv_heads, const int32_t *offsets, int32_t B,
                                  int32_t window, int32_t sinks, const otas_score_desc *score, void *o);

/* The same for the last tokens of a cache whose entries lie in the order of their tokens (as otas_cache_append leaves them; not after
 * otas_cache_evict): a query's n rows are its last n entries, which are in the cache already, and row i is entry
 * t = length[q] - n + i, which sees the entries j of its slot with j <= t and (t - j < window or j < sinks).
 *   qkv dev [T, (H + 2 kv_heads) d_h], kv_heads the cache's: only the query heads are read.  One row is a token that was just appended, many
 *   are a run of drafts or a prompt taken in pieces.
 *   offsets, slot, length host: 0 <= rows of a query <= length[q] (EINVAL); slots may repeat
 *   score NULL = all defaults; the distance for slopes is t - j.  Neither the cache's positions nor its mass are touched.
 *   workspace dev >= otas_attention_recent_workspace_bytes for the same kv_heads, offsets, length, window and sinks, 256-byte aligned;
 *   the bytes grow with the lengths
 *   o dev [T, D]; o and the workspace overlap no other array.   Host numbers: 3 B + 1.
 * d_h a multiple of 8 up to 128, length[q] (H / kv_heads) < 2^30 (EUNSUPPORTED).  Keys and values that a row does not see do not reach it.  A row that sees a key or value
 * that is not finite is not finite where it counts, or all NaN.  f32 models form products from operands cut into three
 * bf16 pieces each, without loss but for the product of the two last (2^-30 of the product): sums are float.  bf16 models round
 * weights as otas_attention_masked does.  The split of a long window between workgroups, and with it the last bits of o, depends on the whole
 * call's lengths. */
size_t otas_attention_recent_workspace_bytes(const otas_ctx *ctx, int32_t kv_heads, const int32_t *offsets, const int32_t *length,
                                             int32_t B, int32_t window, int32_t sinks);
otas_status otas_attention_recent(otas_ctx *ctx, const otas_kv_cache *cache, const void *qkv, const int32_t *offsets,
                                  const int32_t *slot, const int32_t *length, int32_t B, int32_t window, int32_t sinks,
                                  const otas_score_desc *score, void *workspace, size_t workspace_bytes, void *o);

/* A cache in 4 bits an element (the E2M1 elements and E8M0 scales of the OCP Microscaling formats, blocks of 32).  The elements of a head
 * of an entry form groups of OTAS_CACHE4_GROUP, the last one of the rest.  A group has one scale 2^e: e is the smallest
 * exponent with max |x| <= 7 2^e, held to [-125, 125], so that no element is off by more than half a step of its place in
 *   0, 1/2, 1, 3/2, 2, 3, 4, 6   (times 2^e)
 * (but beyond 7 2^125, which becomes 6 2^125).  An element is held as the nearest of these, of two as near the one whose code (its
 * place in the list) is even, with the sign in bit 3; an element at an even place lies in the low half of its byte.  The scale is held as
 * e + 127.  A group with an element that is not finite is held as scale 255, codes 0: all of it reads as NaN.
 *   k, v              dev [slots, kv_heads, capacity, d_h / 2] bytes, aligned to 16
 *   k_scales, v_scales dev [slots, kv_heads, ceil(d_h / 32), capacity] bytes, aligned to 16
 * capacity a multiple of 32 (EINVAL);  d_h a multiple of 8 (EUNSUPPORTED from every call).  The four arrays overlap neither each
 * other nor any other array of a call (EINVAL where they do).  Entries are tokens in order: there is no position and no mass.
 * What lies behind a slot's entries is not used, whatever it holds, and not written. */
#define OTAS_CACHE4_GROUP 32
typedef struct {
  void *k, *v;
  void *k_scales, *v_scales;
  int32_t slots, kv_heads, capacity;
} otas_kv_cache4;

/* otas_cache_append for it: rows[i] (NULL: row i), i = row_offsets[q] .. row_offsets[q+1] - 1, become entries length[q],
 * length[q] + 1, .. of slot[q].  Arguments and limits as there.   Host numbers: 3 B + 1, and with rows row_offsets[B] more. */
otas_status otas_cache4_append(otas_ctx *ctx, const otas_kv_cache4 *cache, const void *qkv, int64_t T, const int32_t *row_offsets,
                               const int32_t *rows, const int32_t *slot, const int32_t *length, int32_t B, int32_t *length_out);

/* Entries first[q] .. first[q] + (row_offsets[q+1] - row_offsets[q]) - 1 of slot[q] as rows row_offsets[q] .. of kv, in the model's dtype
 * (which holds them exactly): the key heads, then the value heads.   kv dev [row_offsets[B], 2 kv_heads d_h]; slots may repeat;
 * what is asked for lies within the capacity (EINVAL).   Host numbers: 3 B + 1. */
otas_status otas_cache4_read(otas_ctx *ctx, const otas_kv_cache4 *cache, const int32_t *slot, const int32_t *first,
                             const int32_t *row_offsets, int32_t B, void *kv);

/* otas_attention_recent over it, with the same arguments and workspace.  Products are of the held values, exactly; nothing
 * is rounded to fewer bits than there. */
otas_status otas_attention_cache4(otas_ctx *ctx, const otas_kv_cache4 *cache, const void *qkv, const int32_t *offsets,
                                  const int32_t *slot, const int32_t *length, int32_t B, int32_t window, int32_t sinks,
                                  const otas_score_desc *score, void *workspace, size_t workspace_bytes, void *o);

#ifdef __cplusplus
}
#endif
#endif /* OTAS_DECODE_H_ */
