// What the entry points of the decoder's operators share: checks of arguments, the context's device, host numbers, launches.
// Internal to the library.
#ifndef OTAS_DECODE_CHECKS_H_
#define OTAS_DECODE_CHECKS_H_

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "../../include/otas_decode.h"
#include "context.h"
#include "decode_kernels.h"

namespace otas {

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
inline otas_status place_plan(otas_ctx* c, const std::vector<int32_t>& plan) {
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

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

// Whether [a, a + bytes) and [b, b + more) have a byte in common.
inline bool overlap(const void* a, size_t bytes, const void* b, size_t more) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return bytes > 0 && more > 0 && x < y + more && y < x + bytes;
}

inline size_t qkv_bytes(const otas_ctx* c, int64_t T, int kv) {
  const int dh = c->desc.D / c->desc.H;
  return (size_t)T * (c->desc.H + 2 * kv) * dh * elem_size(c->desc.dtype);
}
inline size_t rows_bytes(const otas_ctx* c, int64_t T) { return (size_t)T * c->desc.D * elem_size(c->desc.dtype); }

inline bool kv_heads_ok(const otas_ctx* c, int kv) { return kv > 0 && kv <= c->desc.H && c->desc.H % kv == 0; }

// The cache's description, and that every query's slot is one of its own and holds its entries.
inline otas_status cache_ok(const otas_ctx* c, const otas_kv_cache* cache) {
  if (!cache || !cache->k || !cache->v || !cache->positions) return OTAS_EINVAL;
  if (cache->slots <= 0 || cache->capacity <= 0 || !kv_heads_ok(c, cache->kv_heads)) return OTAS_EINVAL;
  if (cache->capacity > OTAS_MAX_LONG_SEQ) return OTAS_EUNSUPPORTED;
  if (cache->k == cache->v) return OTAS_EINVAL;
  if (!aligned16(cache->k) || !aligned16(cache->v) || !aligned4(cache->positions) || !aligned4(cache->mass)) return OTAS_EINVAL;
  return OTAS_OK;
}
inline otas_status slots_ok(int slots, int capacity, const int32_t* slot, const int32_t* length, int B, bool distinct) {
  for (int q = 0; q < B; ++q)
    if (slot[q] < 0 || slot[q] >= slots || length[q] < 0 || length[q] > capacity) return OTAS_EINVAL;
  if (distinct) {
    std::vector<int32_t> seen(slot, slot + B);
    std::sort(seen.begin(), seen.end());
    if (std::adjacent_find(seen.begin(), seen.end()) != seen.end()) return OTAS_EINVAL;
  }
  return OTAS_OK;
}
inline otas_status slots_ok(const otas_kv_cache* cache, const int32_t* slot, const int32_t* length, int B, bool distinct) {
  return slots_ok(cache->slots, cache->capacity, slot, length, B, distinct);
}
// Whether an array has a byte in common with the cache's keys or values.  (Sizes past 64 bits are everything.)
inline bool in_cache(const otas_ctx* c, const otas_kv_cache* cache, const void* p, size_t bytes) {
  const double d = (double)cache->slots * cache->kv_heads * cache->capacity * (c->desc.D / c->desc.H) * elem_size(c->desc.dtype);
  const size_t limit = SIZE_MAX - std::max((uintptr_t)cache->k, (uintptr_t)cache->v), all = d < (double)limit ? (size_t)d : limit;
  return overlap(p, bytes, cache->k, all) || overlap(p, bytes, cache->v, all);
}
inline CacheRef cache_ref(const otas_ctx* c, const otas_kv_cache* cache) {
  return CacheRef{cache->k, cache->v, cache->positions, cache->mass, cache->capacity, cache->kv_heads, c->desc.D / c->desc.H};
}

inline otas_status score_ok(const otas_ctx* c, const otas_score_desc* score, ScoreArgs* out) {
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
template <typename F> inline otas_status guarded(F f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return OTAS_ENOMEM;
  } catch (...) {
    return OTAS_EDEVICE;
  }
}
template <typename F> inline size_t guarded_size(F f) noexcept {
  try {
    return f();
  } catch (...) {
    return 0;
  }
}

// What of a rotation can be said without its factors.
inline bool rotary_desc_ok(const otas_rotary_desc& d, int dh) {
  if (d.rot_dim < 0 || d.rot_dim > dh || d.rot_dim % 2 != 0) return false;
  if (d.layout != OTAS_ROTARY_HALF && d.layout != OTAS_ROTARY_INTERLEAVED) return false;
  if (d.scaling < OTAS_ROTARY_PLAIN || d.scaling > OTAS_ROTARY_BY_PARTS) return false;
  if (!std::isfinite(d.base) || d.base <= 0.0 || !std::isfinite((float)d.magnitude) || d.magnitude == 0.0) return false;
  if (d.scaling != OTAS_ROTARY_PLAIN && (!std::isfinite(d.factor) || d.factor <= 0.0)) return false;
  if (d.scaling == OTAS_ROTARY_BASE && d.rot_dim < 4) return false;
  return d.scaling != OTAS_ROTARY_BY_PARTS ||
         (std::isfinite(d.original_length) && d.original_length > 0.0 && std::isfinite(d.fast_turns) && std::isfinite(d.slow_turns) &&
          d.fast_turns > d.slow_turns);
}
// The rotation's turns per position of every pair.
inline bool rotary_args(const otas_rotary_desc& d, RotaryArgs* r) {
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

}  // namespace otas
#endif  // OTAS_DECODE_CHECKS_H_
