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
struct TreeShape {
  int rows, groups, chunk, parts, room;   // room: what the workspace has place for; >= parts, and grows with the lengths
};
inline TreeShape tree_shape(int dtype, int dh, int H, int KV, const int32_t* off, const int32_t* length, int B) {
  TreeShape t{32, 1, 0, 1, 1};
  int most = 0, longest = 0;
  for (int q = 0; q < B; ++q) {
    most = std::max(most, off[q + 1] - off[q]);
    longest = std::max(longest, (int)length[q]);
  }
  const int rows = most * (H / KV);
  if (dtype != 0 && bf16_width(dh)) t.rows = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  t.groups = std::max(1, (rows + t.rows - 1) / t.rows);
  const int64_t wgs = (int64_t)B * KV * t.groups;
  const int target = t.rows > 32 ? 512 : 1024;
  const int wanted = (int)std::max<int64_t>(1, std::min<int64_t>(target / wgs, (longest + 127) / 128));
  t.chunk = std::max(128, ((longest + wanted - 1) / wanted + 127) & ~127);
  t.parts = std::max(1, (longest + t.chunk - 1) / t.chunk);
  t.room = wanted;
  return t;
}
// Floats of workspace: ends [T H][2]; where there is room for more than one part, for each largest logits and weight sums [T H][2]
// and sums [T H][dh]; where weights are added up over few rows (bf16), logits [T H][stride].
inline int64_t tree_logit_stride(int max_len) { return (max_len + 3) / 4 * 4; }
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
