// C ABI of the decoder's operators (include/otas_decode.h): argument validation and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "../../include/otas_decode.h"
#include "context.h"
#include "decode_kernels.h"

using namespace otas;

namespace {

static_assert(OTAS_DECODE_ARGUMENTS == kArgInts && (size_t)OTAS_MAX_LONG_SEQ <= kPlanInts, "documented limits");

// The context's device for the length of a call.
struct OnDevice {
  int before = -1;
  bool ok;
  explicit OnDevice(const otas_ctx* c) {
    ok = hipGetDevice(&before) == hipSuccess && (before == c->device || hipSetDevice(c->device) == hipSuccess);
    if (before == c->device) before = -1;
  }
  ~OnDevice() {
    if (ok && before >= 0) (void)hipSetDevice(before);
  }
};

// The host numbers of a call: in the kernels' arguments, or uploaded; the latter not into a graph, whose replays would read the
// staging slot after later calls have filled it.
otas_status place_plan(otas_ctx* c, const std::vector<int32_t>& plan) {
  if (plan_in_args(plan.size())) return OTAS_OK;
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(c->stream, &cap) != hipSuccess) return OTAS_EDEVICE;
  if (cap != hipStreamCaptureStatusNone) return OTAS_EUNSUPPORTED;
  return upload_plan(c, plan);
}

// A launch of an operator; one of more workgroups than a launch may have is refused.
#define OTAS_LAUNCH_FITTING(kind, expr)                      \
  do {                                                       \
    hipError_t _e;                                           \
    {                                                        \
      LaunchTimer _t(c, kind, c->stream);                    \
      _e = (expr);                                           \
    }                                                        \
    if (_e == kTooManyGroups) return OTAS_EUNSUPPORTED;      \
    OTAS_HIP(_e);                                            \
  } while (0)

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

// Whether [a, a + bytes) and [b, b + more) have a byte in common.
bool overlap(const void* a, size_t bytes, const void* b, size_t more) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + more && y < x + bytes;
}

size_t qkv_bytes(const otas_ctx* c, int64_t T, int kv) {
  const int dh = c->desc.D / c->desc.H;
  return (size_t)T * (c->desc.H + 2 * kv) * dh * elem_size(c->desc.dtype);
}
size_t rows_bytes(const otas_ctx* c, int64_t T) { return (size_t)T * c->desc.D * elem_size(c->desc.dtype); }

bool kv_heads_ok(const otas_ctx* c, int kv) { return kv > 0 && kv <= c->desc.H && c->desc.H % kv == 0; }

// The cache's description, and that every query's slot is one of its own and holds its entries.
otas_status cache_ok(const otas_ctx* c, const otas_kv_cache* cache) {
  if (!cache || !cache->k || !cache->v || !cache->positions) return OTAS_EINVAL;
  if (cache->slots <= 0 || cache->capacity <= 0 || !kv_heads_ok(c, cache->kv_heads)) return OTAS_EINVAL;
  if (cache->capacity > OTAS_MAX_LONG_SEQ) return OTAS_EUNSUPPORTED;
  if (cache->k == cache->v) return OTAS_EINVAL;
  if (!aligned16(cache->k) || !aligned16(cache->v) || !aligned4(cache->positions) || !aligned4(cache->mass)) return OTAS_EINVAL;
  return OTAS_OK;
}
otas_status slots_ok(const otas_kv_cache* cache, const int32_t* slot, const int32_t* length, int B, bool distinct) {
  for (int q = 0; q < B; ++q)
    if (slot[q] < 0 || slot[q] >= cache->slots || length[q] < 0 || length[q] > cache->capacity) return OTAS_EINVAL;
  if (distinct) {
    std::vector<int32_t> seen(slot, slot + B);
    std::sort(seen.begin(), seen.end());
    if (std::adjacent_find(seen.begin(), seen.end()) != seen.end()) return OTAS_EINVAL;
  }
  return OTAS_OK;
}
// Whether an array has a byte in common with the cache's keys or values.  (Sizes past 64 bits are everything.)
bool in_cache(const otas_ctx* c, const otas_kv_cache* cache, const void* p, size_t bytes) {
  const double d = (double)cache->slots * cache->kv_heads * cache->capacity * (c->desc.D / c->desc.H) * elem_size(c->desc.dtype);
  const size_t limit = SIZE_MAX - std::max((uintptr_t)cache->k, (uintptr_t)cache->v), all = d < (double)limit ? (size_t)d : limit;
  return overlap(p, bytes, cache->k, all) || overlap(p, bytes, cache->v, all);
}
CacheRef cache_ref(const otas_ctx* c, const otas_kv_cache* cache) {
  return CacheRef{cache->k, cache->v, cache->positions, cache->mass, cache->capacity, cache->kv_heads, c->desc.D / c->desc.H};
}

otas_status score_ok(const otas_ctx* c, const otas_score_desc* score, ScoreArgs* out) {
  *out = ScoreArgs{1.f / std::sqrt((float)(c->desc.D / c->desc.H)), 0.f, nullptr};
  if (!score) return OTAS_OK;
  if (!std::isfinite(score->scale) || !std::isfinite(score->cap) || score->cap < 0.f || !aligned4(score->slopes)) return OTAS_EINVAL;
  if (score->scale != 0.f) out->scale = score->scale;
  out->cap = score->cap;
  // The kernels' factors, exp2 in place of exp and tanh by it, have to be finite too.
  const double scale = std::fabs((double)out->scale), most = 3.4e38;
  if (scale * 1.5 > most || (score->cap > 0.f && (score->cap * 1.5 > most || scale / score->cap * 3.0 > most))) return OTAS_EINVAL;
  // A cap that the scale is no float's part of: products of up to 2^115 are off by 2^-23 of themselves without it.
  if (score->cap > 0.f && scale / score->cap < 1.17549435e-38) out->cap = 0.f;
  out->slopes = score->slopes;
  return OTAS_OK;
}

// No C++ exception leaves the library: the only ones are failed allocations of host arrays.
template <typename F> otas_status guarded(F f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return OTAS_ENOMEM;
  } catch (...) {
    return OTAS_EDEVICE;
  }
}
template <typename F> size_t guarded_size(F f) noexcept {
  try {
    return f();
  } catch (...) {
    return 0;
  }
}

// The rotation's turns per position of every pair.
bool rotary_args(const otas_rotary_desc& d, RotaryArgs* r) {
  const int pairs = d.rot_dim / 2;
  double base = d.base;
  if (d.scaling == OTAS_ROTARY_BASE) base *= std::pow(d.factor, (double)d.rot_dim / (d.rot_dim - 2));
  if (!std::isfinite(base) || base <= 0.0) return false;
  for (int i = 0; i < pairs; ++i) {
    double turns = std::pow(base, -2.0 * i / d.rot_dim) / (2.0 * 3.14159265358979323846);
    if (d.scaling == OTAS_ROTARY_LINEAR) turns /= d.factor;
    if (d.scaling == OTAS_ROTARY_BY_PARTS) {
      const double w = std::min(1.0, std::max(0.0, (d.original_length * turns - d.slow_turns) / (d.fast_turns - d.slow_turns)));
      turns = w * turns + (1.0 - w) * turns / d.factor;
    }
    if (!std::isfinite(turns * 2147483648.0)) return false;   // the farthest position's
    r->turns[i] = d.inverse ? -turns : turns;
  }
  for (int i = pairs; i < 64; ++i) r->turns[i] = 0.0;
  r->magnitude = (float)d.magnitude;
  r->rot = d.rot_dim;
  r->interleaved = d.layout == OTAS_ROTARY_INTERLEAVED;
  return true;
}

}  // namespace

extern "C" {

otas_status otas_rotary(otas_ctx* c, const void* qkv, int64_t T, int32_t kv_heads, const int32_t* positions,
                        const otas_rotary_desc* rope, void* out) {
  return guarded([&]() -> otas_status {
    if (!c || !rope || T < 0 || !kv_heads_ok(c, kv_heads)) return OTAS_EINVAL;
    if (T > 0 && (!qkv || !positions || !out)) return OTAS_EINVAL;   // no rows, no arrays
    const int dh = c->desc.D / c->desc.H;
    const otas_rotary_desc& d = *rope;
    if (d.rot_dim < 0 || d.rot_dim > dh || d.rot_dim % 2 != 0) return OTAS_EINVAL;
    if (d.layout != OTAS_ROTARY_HALF && d.layout != OTAS_ROTARY_INTERLEAVED) return OTAS_EINVAL;
    if (d.scaling < OTAS_ROTARY_PLAIN || d.scaling > OTAS_ROTARY_BY_PARTS) return OTAS_EINVAL;
    if (!std::isfinite(d.base) || d.base <= 0.0 || !std::isfinite((float)d.magnitude) || d.magnitude == 0.0) return OTAS_EINVAL;
    if (d.scaling != OTAS_ROTARY_PLAIN && (!std::isfinite(d.factor) || d.factor <= 0.0)) return OTAS_EINVAL;
    if (d.scaling == OTAS_ROTARY_BASE && d.rot_dim < 4) return OTAS_EINVAL;
    if (d.scaling == OTAS_ROTARY_BY_PARTS &&
        (!std::isfinite(d.original_length) || d.original_length <= 0.0 || !std::isfinite(d.fast_turns) ||
         !std::isfinite(d.slow_turns) || d.fast_turns <= d.slow_turns))
      return OTAS_EINVAL;
    if (!aligned16(qkv) || !aligned16(out) || !aligned4(positions)) return OTAS_EINVAL;
    if (T > INT32_MAX) return OTAS_EUNSUPPORTED;
    const size_t bytes = qkv_bytes(c, T, kv_heads);
    if (out != qkv && overlap(qkv, bytes, out, bytes)) return OTAS_EINVAL;
    RotaryArgs r;
    if (!rotary_args(d, &r)) return OTAS_EINVAL;
    if (T == 0 || (out == qkv && d.rot_dim == 0)) return OTAS_OK;
    OnDevice on(c);
    if (!on.ok) return OTAS_EDEVICE;
    OTAS_LAUNCH_FITTING(K_MISC, launch_rotary(c->desc.dtype, qkv, out, positions, T, c->desc.H, kv_heads, dh, r, c->stream));
    return OTAS_OK;
  });
}

otas_status otas_attention_masked(otas_ctx* c, const void* qkv, int32_t kv_heads, const int32_t* offsets, int32_t B,
                                  int32_t causal, const int32_t* prefix, const int32_t* documents, const int32_t* positions,
                                  const otas_score_desc* score, void* o) {
  return guarded([&]() -> otas_status {
    if (!c || !offsets || B <= 0 || !kv_heads_ok(c, kv_heads) || !offsets_ok(offsets, B)) return OTAS_EINVAL;
    if (offsets[B] > 0 && (!qkv || !o)) return OTAS_EINVAL;
    ScoreArgs sc;
    const otas_status st = score_ok(c, score, &sc);
    if (st != OTAS_OK) return st;
    if (!aligned16(qkv) || !aligned16(o) || !aligned4(documents) || !aligned4(positions)) return OTAS_EINVAL;
    const int64_t T = offsets[B];
    if (overlap(qkv, qkv_bytes(c, T, kv_heads), o, rows_bytes(c, T))) return OTAS_EINVAL;
    int max_n = 0;
    for (int q = 0; q < B; ++q) {
      const int n = offsets[q + 1] - offsets[q];
      if (prefix && (prefix[q] < 0 || prefix[q] > n)) return OTAS_EINVAL;
      max_n = std::max(max_n, n);
    }
    if (max_n > OTAS_MAX_LONG_SEQ) return OTAS_EUNSUPPORTED;
    std::vector<int32_t> plan(2 * (size_t)B + 1, 0);   // offsets [B+1] | prefix [B]
    std::copy(offsets, offsets + B + 1, plan.begin());
    if (prefix) std::copy(prefix, prefix + B, plan.begin() + B + 1);
    if (T == 0) return OTAS_OK;
    OnDevice on(c);
    if (!on.ok) return OTAS_EDEVICE;
    const otas_status placed = place_plan(c, plan);
    if (placed != OTAS_OK) return placed;
    OTAS_LAUNCH_FITTING(K_ATTN, launch_attention_masked(c->desc.dtype, qkv, plan.data(), plan.size(), c->d_plan, B, max_n, c->desc.H, kv_heads,
                                                c->desc.D / c->desc.H, sc, MaskArgs{documents, positions, causal != 0}, o, c->stream));
    return OTAS_OK;
  });
}

otas_status otas_cache_append(otas_ctx* c, const otas_kv_cache* cache, const void* qkv, int64_t T, const int32_t* row_offsets,
                              const int32_t* rows, const int32_t* positions, const int32_t* slot, const int32_t* length,
                              int32_t B, int32_t* length_out) {
  return guarded([&]() -> otas_status {
    if (!c || !row_offsets || !slot || !length || !length_out || B <= 0 || T < 0) return OTAS_EINVAL;
    otas_status st = cache_ok(c, cache);
    if (st != OTAS_OK) return st;
    if (!aligned16(qkv) || !aligned4(positions) || !offsets_ok(row_offsets, B)) return OTAS_EINVAL;
    if (row_offsets[B] > 0 && (!qkv || !positions || in_cache(c, cache, qkv, qkv_bytes(c, T, cache->kv_heads)))) return OTAS_EINVAL;
    st = slots_ok(cache, slot, length, B, true);
    if (st != OTAS_OK) return st;
    const int64_t N = row_offsets[B];
    for (int q = 0; q < B; ++q)
      if (row_offsets[q + 1] - row_offsets[q] > cache->capacity - length[q]) return OTAS_EINVAL;
    if (rows) {
      for (int64_t i = 0; i < N; ++i)
        if (rows[i] < 0 || rows[i] >= T) return OTAS_EINVAL;
    } else if (N > T) {
      return OTAS_EINVAL;
    }
    if (N > kMostGroups) return OTAS_EUNSUPPORTED;   // a workgroup a row
    const size_t count = 3 * (size_t)B + 1 + (rows ? (size_t)N : 0);
    if (count > kPlanInts) return OTAS_ENOMEM;
    std::vector<int32_t> plan(count);   // row offsets [B+1] | slot [B] | length [B] | rows [N]
    std::copy(row_offsets, row_offsets + B + 1, plan.begin());
    std::copy(slot, slot + B, plan.begin() + B + 1);
    std::copy(length, length + B, plan.begin() + 2 * B + 1);
    if (rows) std::copy(rows, rows + N, plan.begin() + 3 * B + 1);
    if (N > 0) {
      OnDevice on(c);
      if (!on.ok) return OTAS_EDEVICE;
      st = place_plan(c, plan);
      if (st != OTAS_OK) return st;
      OTAS_LAUNCH(K_MISC, launch_cache_append(c->desc.dtype, cache_ref(c, cache), qkv, c->desc.H, positions, plan.data(), plan.size(),
                                              c->d_plan, B, N, rows != nullptr, c->stream));
    }
    for (int q = 0; q < B; ++q) length_out[q] = length[q] + (row_offsets[q + 1] - row_offsets[q]);
    return OTAS_OK;
  });
}

size_t otas_attention_tree_workspace_bytes(const otas_ctx* c, int32_t kv_heads, const int32_t* offsets, const int32_t* length, int32_t B,
                                           int32_t add_mass) {
  return guarded_size([&]() -> size_t {
    if (!c || !offsets || !length || B <= 0 || !kv_heads_ok(c, kv_heads) || !offsets_ok(offsets, B)) return 0;
    int max_len = 0;
    for (int q = 0; q < B; ++q) {
      if (length[q] < 0 || length[q] > OTAS_MAX_LONG_SEQ || offsets[q + 1] - offsets[q] > OTAS_MAX_TREE_NODES) return 0;
      max_len = std::max(max_len, (int)length[q]);
    }
    const int dh = c->desc.D / c->desc.H;
    const TreeShape t = tree_shape(c->desc.dtype, dh, c->desc.H, kv_heads, offsets, length, B);
    const size_t floats = tree_workspace_floats(t, c->desc.dtype, offsets[B], c->desc.H, dh, max_len, add_mass != 0);
    return align_up(std::max<size_t>(1, floats) * sizeof(float), kAlign);
  });
}

otas_status otas_attention_tree(otas_ctx* c, const otas_kv_cache* cache, const void* qkv, const int32_t* offsets,
                                const int32_t* parents, const int32_t* positions, const int32_t* slot, const int32_t* length,
                                int32_t B, const otas_score_desc* score, int32_t add_mass, void* workspace,
                                size_t workspace_bytes, void* o) {
  return guarded([&]() -> otas_status {
    if (!c || !offsets || !slot || !length || B <= 0 || !offsets_ok(offsets, B)) return OTAS_EINVAL;
    if (offsets[B] > 0 && (!qkv || !workspace || !o)) return OTAS_EINVAL;
    otas_status st = cache_ok(c, cache);
    if (st != OTAS_OK) return st;
    ScoreArgs sc;
    st = score_ok(c, score, &sc);
    if (st != OTAS_OK) return st;
    if ((sc.slopes && !positions) || (add_mass && !cache->mass)) return OTAS_EINVAL;
    if (!aligned16(qkv) || !aligned16(o) || !aligned4(positions) || (uintptr_t)workspace % kAlign != 0) return OTAS_EINVAL;
    st = slots_ok(cache, slot, length, B, add_mass != 0);
    if (st != OTAS_OK) return st;
    const int64_t T = offsets[B];
    bool chains = true;
    int max_len = 0;
    for (int q = 0; q < B; ++q) {
      const int n = offsets[q + 1] - offsets[q];
      if (n > OTAS_MAX_TREE_NODES) return OTAS_EUNSUPPORTED;
      max_len = std::max(max_len, (int)length[q]);
      for (int i = 0; parents && i < n; ++i) {
        const int p = parents[offsets[q] + i];
        if (p < -1 || p >= i) return OTAS_EINVAL;
        chains = chains && p == i - 1;
      }
    }
    const int dh = c->desc.D / c->desc.H;
    const TreeShape shape = tree_shape(c->desc.dtype, dh, c->desc.H, cache->kv_heads, offsets, length, B);
    const size_t floats = tree_workspace_floats(shape, c->desc.dtype, T, c->desc.H, dh, max_len, add_mass != 0);
    if (T > 0 && workspace_bytes < floats * sizeof(float)) return OTAS_ENOMEM;
    const size_t in_bytes = qkv_bytes(c, T, cache->kv_heads), out_bytes = rows_bytes(c, T);
    if (overlap(qkv, in_bytes, o, out_bytes) || overlap(workspace, floats * sizeof(float), o, out_bytes) ||
        overlap(workspace, floats * sizeof(float), qkv, in_bytes) || in_cache(c, cache, o, out_bytes) ||
        in_cache(c, cache, workspace, floats * sizeof(float)))
      return OTAS_EINVAL;
    std::vector<int32_t> plan(3 * (size_t)B + 1 + (chains ? 0 : (size_t)(T + 3) / 4), 0);
    std::copy(offsets, offsets + B + 1, plan.begin());
    std::copy(slot, slot + B, plan.begin() + B + 1);
    std::copy(length, length + B, plan.begin() + 2 * B + 1);
    if (!chains)
      for (int64_t i = 0; i < T; ++i)
        plan[3 * (size_t)B + 1 + i / 4] = (int32_t)((uint32_t)plan[3 * (size_t)B + 1 + i / 4] | (uint32_t)(parents[i] & 255) << (8 * (i & 3)));
    if (T == 0) return OTAS_OK;
    OnDevice on(c);
    if (!on.ok) return OTAS_EDEVICE;
    st = place_plan(c, plan);
    if (st != OTAS_OK) return st;
    OTAS_LAUNCH_FITTING(K_ATTN, launch_attention_tree(c->desc.dtype, cache_ref(c, cache), qkv, c->desc.H, positions, plan.data(), plan.size(), c->d_plan,
                                              B, T, max_len, !chains, sc, add_mass != 0, shape, (float*)workspace, o, c->stream));
    return OTAS_OK;
  });
}

size_t otas_cache_evict_workspace_bytes(const otas_ctx* c, const int32_t* length, const int32_t* keep, int32_t B) {
  if (!c || !length || !keep || B <= 0) return 0;
  size_t ints = (size_t)B;
  for (int q = 0; q < B; ++q) {
    if (length[q] < 0 || length[q] > OTAS_MAX_LONG_SEQ || keep[q] < 0) return 0;
    ints += 2 * (size_t)evict_moves_bound(length[q], keep[q]);
  }
  return align_up(ints * sizeof(int32_t), kAlign);
}

otas_status otas_cache_evict(otas_ctx* c, const otas_kv_cache* cache, const int32_t* slot, const int32_t* length,
                             const int32_t* keep, int32_t B, int32_t lead, const int32_t* recent_from, void* workspace,
                             size_t workspace_bytes, int32_t* length_out) {
  return guarded([&]() -> otas_status {
    if (!c || !slot || !length || !keep || !workspace || !length_out || B <= 0 || lead < 0) return OTAS_EINVAL;
    otas_status st = cache_ok(c, cache);
    if (st != OTAS_OK) return st;
    if (!cache->mass || (uintptr_t)workspace % kAlign != 0) return OTAS_EINVAL;
    st = slots_ok(cache, slot, length, B, true);
    if (st != OTAS_OK) return st;
    if (B > 65535) return OTAS_EUNSUPPORTED;   // grid
    std::vector<int32_t> plan(5 * (size_t)B, 0);   // slot | length | keep | recent_from | first entry of the query's lists
    int64_t at = 0;
    int max_len = 0, max_moves = 0;
    for (int q = 0; q < B; ++q) {
      if (keep[q] < 0) return OTAS_EINVAL;
      const int moves = evict_moves_bound(length[q], keep[q]);
      plan[q] = slot[q];
      plan[B + q] = length[q];
      plan[2 * (size_t)B + q] = keep[q];
      plan[3 * (size_t)B + q] = recent_from ? recent_from[q] : 0;
      plan[4 * (size_t)B + q] = (int32_t)at;
      at += 2 * (int64_t)moves;
      if (at > INT32_MAX - B) return OTAS_EUNSUPPORTED;
      max_len = std::max(max_len, (int)length[q]);
      max_moves = std::max(max_moves, moves);
    }
    if (workspace_bytes < ((size_t)B + at) * sizeof(int32_t)) return OTAS_ENOMEM;
    if (in_cache(c, cache, workspace, ((size_t)B + at) * sizeof(int32_t))) return OTAS_EINVAL;
    if (max_moves > 0) {
      OnDevice on(c);
      if (!on.ok) return OTAS_EDEVICE;
      st = place_plan(c, plan);
      if (st != OTAS_OK) return st;
      OTAS_LAUNCH(K_MISC, launch_cache_evict(c->desc.dtype, cache_ref(c, cache), plan.data(), plan.size(), c->d_plan, B, max_len, max_moves,
                                             lead, recent_from != nullptr, (int32_t*)workspace, c->stream));
    }
    for (int q = 0; q < B; ++q) length_out[q] = std::min(length[q], keep[q]);
    return OTAS_OK;
  });
}

}  // extern "C"
