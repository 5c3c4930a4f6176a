// Host-side launchers of the decoder's operators (include/otas_decode.h).  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "kernels.h"

namespace otas {

// Workgroups of 256 threads that one launch may have (its threads are counted in 32 bits), and what a launcher returns, with nothing
// launched, for a call of more.
constexpr int64_t kMostGroups = UINT32_MAX / 256;
constexpr hipError_t kTooManyGroups = hipErrorInvalidConfiguration;

struct RotaryArgs {
  double turns[64];   // full turns per position of every pair (negative: the inverse)
  float magnitude;
  int rot, interleaved;
};
hipError_t launch_rotary(int dtype, const void* qkv, void* out, const int32_t* positions, int64_t T, int H, int KV, int dh,
                         const RotaryArgs& r, hipStream_t s);

struct CacheRef {
  void *k, *v;
  int32_t* positions;
  float* mass;
  int64_t capacity;
  int KV, dh;
};
// plan: row_off [B+1] | slot [B] | length [B] | rows [N] (has_rows); N = row_off[B]
hipError_t launch_cache_append(int dtype, const CacheRef& c, const void* qkv, int H, const int32_t* positions, const int32_t* plan,
                               size_t count, const int32_t* d_plan, int B, int64_t N, bool has_rows, hipStream_t s);

// What every attention of these operators does to its products.
struct ScoreArgs {
  float scale, cap;
  const float* slopes;
};
struct MaskArgs {
  const int32_t *documents, *positions;
  int causal;
};
// plan: off [B+1] | prefix [B]
hipError_t launch_attention_masked(int dtype, const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B,
                                   int max_n, int H, int KV, int dh, const ScoreArgs& sc, const MaskArgs& mk, void* o, hipStream_t s);
// Head widths of the bf16 kernels.
inline bool bf16_width(int dh) { return dh == 64 || dh == 80 || dh == 96 || dh == 128; }
hipError_t launch_attention_masked_bf16(const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int max_n, int H,
                                        int KV, int dh, const ScoreArgs& sc, const MaskArgs& mk, void* o, hipStream_t s);

// How a call of the tree attention is cut up (pure host).  A workgroup has up to `rows` of the nodes x (H / KV) rows of a key
// head, and `chunk` of the cache's entries; `parts` = most chunks of a query.
//   A chunk costs its workgroup some 6 us before the first product and a share of the join afterwards, and too few leave CUs without
// work.  Rows of 64 and 128 and fp32: as many parts as bring the call to 512 and 1024 workgroups (8 x 48 nodes over 4000: 42 us, 54 with
// 1024).  bf16 and 32 rows or fewer: one part up to 384 entries (no join: 24 queries over 300 17.7 -> 14.2 us); blocks of 128
// entries while that makes no more workgroups than CUs; a workgroup per CU where
// that leaves 512 entries or fewer to each (8 queries over 6000, 2 key heads: 19 us; 27 with blocks of 128); else 384 entries or more and up to
// 768 workgroups, which are counted from every query's own length: the longest query's many parts leave nothing to do for those of
// shorter queries (24 queries of 400 .. 8000: 105 -> 96 us; with weights added up 125 -> 115).
//   The nodes themselves follow a query's first chunk, which makes its workgroup the last by 3 us; or they are a part of their own
// (`apart`), behind the chunks, where there are several: one token over 1537 entries 14.6 -> 12.6 us, 8 x 48 nodes over 4000 42 -> 39, fp32 6 x 40 over
// 5000 105 -> 85.  bf16 rows of 32 have them apart while all workgroups find a CU: one fits a CU there at width 128, and
// more of them cost a full chip more than they save (32 tokens over 8192 205 -> 238 us).
struct TreeShape {
  int rows, groups, chunk, parts;   // parts: of the longest query, the nodes' among them
  int apart;                        // 1: the nodes have a part of their own
  int room;                         // parts that the workspace has place for; >= parts, and grows with the lengths
  __host__ __device__ int chunks(int length) const { return (length + chunk - 1) / chunk; }
  __host__ __device__ int parts_of(int length) const { return chunks(length) > 1 ? chunks(length) + apart : 1; }
};
inline TreeShape tree_shape(int dtype, int dh, int H, int KV, const int32_t* off, const int32_t* length, int B) {
  TreeShape t{32, 1, 128, 1, 0, 1};
  int64_t most = 0, longest = 0;
  for (int q = 0; q < B; ++q) {
    most = std::max<int64_t>(most, off[q + 1] - off[q]);
    longest = std::max<int64_t>(longest, length[q]);
  }
  const bool bf16 = dtype != 0 && bf16_width(dh);
  const int64_t rows = most * (H / KV);
  if (bf16) t.rows = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  t.groups = (int)std::max<int64_t>(1, (rows + t.rows - 1) / t.rows);
  const bool few = bf16 && t.rows == 32;
  const int64_t wgs = (int64_t)B * KV * t.groups, target = few ? 768 : t.rows > 32 ? 512 : 1024;
  auto pieces = [](int64_t n, int64_t of) { return std::max<int64_t>(1, (n + of - 1) / of); };
  auto whole = [](int64_t n) { return std::max<int64_t>(128, (n + 127) & ~127); };
  int64_t least = 128;
  if (few && longest <= 384) {
    least = 384;
  } else if (few && wgs * pieces(longest, 128) > 256) {
    const int64_t each = pieces(longest, std::max<int64_t>(1, 256 / wgs));
    least = wgs <= 256 && each <= 512 ? whole(each) : 384;
  }
  const int64_t wanted = std::max<int64_t>(1, std::min(target / wgs, pieces(longest, least)));
  int64_t chunk = whole(pieces(longest, wanted));
  if (few && wanted > 1) {   // the smallest chunk, down to half of that, that keeps to the target
    for (int64_t c = std::max(least, whole(pieces(longest, 2 * wanted))); c < chunk; c += std::max<int64_t>(128, c / 8 & ~127)) {
      int64_t used = 0;
      for (int q = 0; q < B; ++q) used += pieces(length[q], c);
      if (used * KV <= target) chunk = c;   // ends the loop
    }
  }
  t.chunk = (int)chunk;
  t.apart = !few || wgs * (t.chunks((int)longest) + 1) <= 256;
  t.parts = t.parts_of((int)longest);
  const int64_t most_chunks = std::min((few ? 2 : 1) * (target / wgs), pieces(longest, 128));
  t.room = most_chunks > 1 ? (int)most_chunks + 1 : 1;
  return t;
}
// Floats of workspace: ends [T H][2]; where there is room for more than one part, for each largest logits and weight sums [T H][2]
// and sums [T H][dh]; where weights are added up over few rows (bf16), logits [T H][stride].  Sums and logits are accessed four at a
// time and begin at multiples of four (dh is one, so that the sums end before the logits whatever the parts).
inline int64_t tree_logit_stride(int max_len) { return (max_len + 3) / 4 * 4; }
inline size_t tree_sums_at(const TreeShape& t, int64_t T, int H) { return ((size_t)T * H * 2 * (1 + (size_t)t.parts) + 3) / 4 * 4; }
inline size_t tree_logits_at(const TreeShape& t, int64_t T, int H, int dh) {
  return ((size_t)T * H * ((t.room > 1 ? (size_t)t.room * (dh + 2) : 0) + 2) + 3) / 4 * 4;
}
inline size_t tree_workspace_floats(const TreeShape& t, int dtype, int64_t T, int H, int dh, int max_len, bool add_mass) {
  const bool logits = add_mass && dtype != 0 && bf16_width(dh) && t.rows == 32;
  return tree_logits_at(t, T, H, dh) + (logits ? (size_t)T * H * tree_logit_stride(max_len) : 0);
}
struct TreeBuffers {
  float *sums, *tops, *ends, *logits;   // ends, logits: or NULL
  int64_t TH, stride;
};
// plan: off [B+1] | slot [B] | length [B] | parents, a byte each (has_parents)
hipError_t launch_attention_tree(int dtype, const CacheRef& c, const void* qkv, int H, const int32_t* positions, const int32_t* plan,
                                 size_t count, const int32_t* d_plan, int B, int64_t T, int max_len, bool has_parents, const ScoreArgs& sc,
                                 bool add_mass, const TreeShape& shape, float* workspace, void* o, hipStream_t s);
hipError_t launch_attention_tree_bf16(const CacheRef& c, const void* qkv, int H, const int32_t* positions, const int32_t* plan, size_t count,
                                      const int32_t* d_plan, int B, int64_t T, int max_len, bool has_parents, const ScoreArgs& sc, bool add_mass,
                                      const TreeShape& shape, float* workspace, void* o, hipStream_t s);

// plan: slot [B] | length [B] | keep [B] | recent_from [B] | list offset [B].  lists: counts [B], then per query its places
// and sources (2 x the bound of its moves).
inline int evict_moves_bound(int length, int keep) { return keep >= length ? 0 : std::min(keep, length - keep); }
hipError_t launch_cache_evict(int dtype, const CacheRef& c, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int max_len,
                              int max_moves, int lead, bool has_recent, int32_t* lists, hipStream_t s);

}  // namespace otas
