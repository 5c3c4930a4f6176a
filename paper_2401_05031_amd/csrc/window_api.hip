// C ABI of the operators of include/otas_decode.h with norms of heads, windows and the cache in 4 bits: argument validation and launches.
#include <hip/hip_runtime.h>

#include "decode_checks.h"
#include "window_kernels.h"

using namespace otas;

static_assert(OTAS_MAX_LONG_SEQ % (1 << kRowsShift) == 0, "the last tile of a full cache");

namespace {

bool window_ok(int window, int sinks) { return window >= 1 && sinks >= 0; }

// [a, a + bytes) ends within 64 bits for sizes of this many bytes, and whether two of a list of arrays have a byte in common.
struct Range {
  const void* p;
  double bytes;
};
bool meet(const Range& a, const Range& b) {
  auto held = [](const Range& r) { return r.bytes < (double)(SIZE_MAX / 4) ? (size_t)r.bytes : SIZE_MAX / 4; };
  return overlap(a.p, held(a), b.p, held(b));
}

// The arrays of a cache in 4 bits.
void cache4_ranges(const otas_ctx* c, const otas_kv_cache4* cache, Range (&r)[4]) {
  const int dh = c->desc.D / c->desc.H, groups = (dh + OTAS_CACHE4_GROUP - 1) / OTAS_CACHE4_GROUP;
  const double entries = (double)cache->slots * cache->kv_heads * cache->capacity;
  r[0] = Range{cache->k, entries * (dh / 2)};
  r[1] = Range{cache->v, entries * (dh / 2)};
  r[2] = Range{cache->k_scales, entries * groups};
  r[3] = Range{cache->v_scales, entries * groups};
}
otas_status cache4_ok(const otas_ctx* c, const otas_kv_cache4* cache) {
  if (!cache || !cache->k || !cache->v || !cache->k_scales || !cache->v_scales) return OTAS_EINVAL;
  if (cache->slots <= 0 || cache->capacity <= 0 || cache->capacity % 32 != 0 || !kv_heads_ok(c, cache->kv_heads)) return OTAS_EINVAL;
  if (!aligned16(cache->k) || !aligned16(cache->v) || !aligned16(cache->k_scales) || !aligned16(cache->v_scales)) return OTAS_EINVAL;
  if (cache->capacity > OTAS_MAX_LONG_SEQ || c->desc.D / c->desc.H % 8 != 0) return OTAS_EUNSUPPORTED;
  Range r[4];
  cache4_ranges(c, cache, r);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (meet(r[i], r[j])) return OTAS_EINVAL;
  return OTAS_OK;
}
bool in_cache4(const otas_ctx* c, const otas_kv_cache4* cache, const void* p, size_t bytes) {
  Range r[4];
  cache4_ranges(c, cache, r);
  return std::any_of(r, r + 4, [&](const Range& x) { return meet(x, Range{p, (double)bytes}); });
}
Cache4Ref cache4_ref(const otas_ctx* c, const otas_kv_cache4* cache) {
  const int dh = c->desc.D / c->desc.H;
  return Cache4Ref{(char*)cache->k, (char*)cache->v, (char*)cache->k_scales, (char*)cache->v_scales, cache->capacity, cache->kv_heads, dh,
                   (dh + OTAS_CACHE4_GROUP - 1) / OTAS_CACHE4_GROUP};
}

// Rows that are the last entries of their slots.
otas_status recent_ok(const int32_t* offsets, const int32_t* length, int B) {
  for (int q = 0; q < B; ++q)
    if (offsets[q + 1] - offsets[q] > length[q]) return OTAS_EINVAL;
  return OTAS_OK;
}
// Rows of a query x heads that share a key head are counted in 32 bits.
bool rows_fit(const otas_ctx* c, int kv, int64_t n) { return n * (c->desc.H / kv) <= INT32_MAX / 2; }

// Either attention of the last tokens; apart(array, bytes): whether it is clear of the cache.
template <typename Apart>
otas_status attention_last(otas_ctx* c, const Cache4Ref& cache, bool four, int slots, const void* qkv, const int32_t* offsets, const int32_t* slot,
                           const int32_t* length, int B, int window, int sinks, const otas_score_desc* score, void* workspace,
                           size_t workspace_bytes, void* o, Apart apart) {
  ScoreArgs sc;
  otas_status st = score_ok(c, score, &sc);
  if (st != OTAS_OK) return st;
  if (!window_ok(window, sinks) || !aligned16(qkv) || !aligned16(o) || (uintptr_t)workspace % kAlign != 0) return OTAS_EINVAL;
  st = slots_ok(slots, (int)cache.capacity, slot, length, B, false);
  if (st == OTAS_OK) st = recent_ok(offsets, length, B);
  if (st != OTAS_OK) return st;
  if (cache.dh % 8 != 0) return OTAS_EUNSUPPORTED;
  for (int q = 0; q < B; ++q)
    if (!rows_fit(c, cache.KV, length[q])) return OTAS_EUNSUPPORTED;
  const int64_t T = offsets[B];
  WindowShape shape = recent_shape(c->desc.dtype, four, cache.dh, c->desc.H, cache.KV, offsets, length, B, window, sinks);
  const size_t need = recent_workspace_floats(shape, T * c->desc.H, cache.dh) * sizeof(float);
  if (T > 0 && workspace_bytes < need) return OTAS_ENOMEM;
  const size_t in_bytes = qkv_bytes(c, T, cache.KV), out_bytes = rows_bytes(c, T);
  if (overlap(qkv, in_bytes, o, out_bytes) || overlap(workspace, need, o, out_bytes) || overlap(workspace, need, qkv, in_bytes) ||
      !apart(o, out_bytes) || !apart(workspace, need))
    return OTAS_EINVAL;
  std::vector<int32_t> plan(3 * (size_t)B + 1);   // offsets [B+1] | slot [B] | length [B]
  std::copy(offsets, offsets + B + 1, plan.begin());
  std::copy(slot, slot + B, plan.begin() + B + 1);
  std::copy(length, length + B, plan.begin() + 2 * B + 1);
  if (T == 0) return OTAS_OK;
  shape.count_groups(plan, offsets, B, c->desc.H / cache.KV, kArgInts, kPlanInts);
  OnDevice on(c);
  if (!on.ok) return OTAS_EDEVICE;
  st = place_plan(c, plan);
  if (st != OTAS_OK) return st;
  OTAS_LAUNCH_FITTING(K_ATTN, launch_attention_recent(c->desc.dtype, four, cache, qkv, c->desc.H, plan.data(), plan.size(), c->d_plan, B, T, sc,
                                              shape, (float*)workspace, o, c->stream));
  return OTAS_OK;
}

}  // namespace

extern "C" {

otas_status otas_norm_rotary(otas_ctx* c, const void* qkv, int64_t T, int32_t kv_heads, const otas_head_norm_desc* norm,
                             const int32_t* positions, const otas_rotary_desc* rope, void* out) {
  return guarded([&]() -> otas_status {
    if (!c || !norm || !rope || T < 0 || !kv_heads_ok(c, kv_heads)) return OTAS_EINVAL;
    const int dh = c->desc.D / c->desc.H;
    if (!rotary_desc_ok(*rope, dh)) return OTAS_EINVAL;
    if (T > 0 && (!qkv || !out || (!positions && rope->rot_dim > 0))) return OTAS_EINVAL;   // no rows, no arrays
    if (!std::isfinite(norm->eps) || norm->eps <= 0.f) return OTAS_EINVAL;
    if (!aligned16(qkv) || !aligned16(out) || !aligned4(positions) || !aligned16(norm->q_gain) || !aligned16(norm->k_gain)) return OTAS_EINVAL;
    if (T > INT32_MAX) return OTAS_EUNSUPPORTED;
    const size_t bytes = qkv_bytes(c, T, kv_heads), head = dh * elem_size(c->desc.dtype);
    if (out != qkv && overlap(qkv, bytes, out, bytes)) return OTAS_EINVAL;
    if (norm->q_gain && overlap(norm->q_gain, head * (norm->per_head ? c->desc.H : 1), out, bytes)) return OTAS_EINVAL;
    if (norm->k_gain && overlap(norm->k_gain, head * (norm->per_head ? kv_heads : 1), out, bytes)) return OTAS_EINVAL;
    RotaryArgs r;
    if (!rotary_args(*rope, &r)) return OTAS_EINVAL;
    if (T == 0) return OTAS_OK;
    OnDevice on(c);
    if (!on.ok) return OTAS_EDEVICE;
    const HeadNormArgs n{norm->q_gain, norm->k_gain, norm->eps, norm->center != 0, norm->per_head != 0};
    OTAS_LAUNCH_FITTING(K_MISC, launch_norm_rotary(c->desc.dtype, qkv, out, positions, T, c->desc.H, kv_heads, dh, n, r, c->stream));
    return OTAS_OK;
  });
}

otas_status otas_attention_window(otas_ctx* c, const void* qkv, int32_t kv_heads, const int32_t* offsets, int32_t B,
                                  int32_t window, int32_t sinks, const otas_score_desc* score, void* o) {
  return guarded([&]() -> otas_status {
    if (!c || !offsets || B <= 0 || !kv_heads_ok(c, kv_heads) || !offsets_ok(offsets, B) || !window_ok(window, sinks)) return OTAS_EINVAL;
    if (offsets[B] > 0 && (!qkv || !o)) return OTAS_EINVAL;
    ScoreArgs sc;
    const otas_status st = score_ok(c, score, &sc);
    if (st != OTAS_OK) return st;
    if (!aligned16(qkv) || !aligned16(o)) return OTAS_EINVAL;
    const int64_t T = offsets[B];
    if (overlap(qkv, qkv_bytes(c, T, kv_heads), o, rows_bytes(c, T))) return OTAS_EINVAL;
    int max_n = 0;
    for (int q = 0; q < B; ++q) max_n = std::max(max_n, offsets[q + 1] - offsets[q]);
    if (max_n > OTAS_MAX_LONG_SEQ || !rows_fit(c, kv_heads, max_n)) return OTAS_EUNSUPPORTED;
    if (T == 0) return OTAS_OK;
    const int dh = c->desc.D / c->desc.H;
    WindowShape shape = packed_shape(c->desc.dtype, dh, c->desc.H, kv_heads, max_n, window, sinks);
    std::vector<int32_t> plan(offsets, offsets + B + 1);
    shape.count_groups(plan, offsets, B, shape.rows == kManyRows ? c->desc.H / kv_heads : 1, kArgInts, kPlanInts);
    OnDevice on(c);
    if (!on.ok) return OTAS_EDEVICE;
    const otas_status placed = place_plan(c, plan);
    if (placed != OTAS_OK) return placed;
    OTAS_LAUNCH_FITTING(K_ATTN, launch_attention_window(c->desc.dtype, qkv, plan.data(), plan.size(), c->d_plan, B, c->desc.H, kv_heads, dh,
                                                        sc, shape, o, c->stream));
    return OTAS_OK;
  });
}

size_t otas_attention_recent_workspace_bytes(const otas_ctx* c, int32_t kv_heads, const int32_t* offsets, const int32_t* length, int32_t B,
                                             int32_t window, int32_t sinks) {
  return guarded_size([&]() -> size_t {
    if (!c || !offsets || !length || B <= 0 || !kv_heads_ok(c, kv_heads) || !offsets_ok(offsets, B) || !window_ok(window, sinks)) return 0;
    for (int q = 0; q < B; ++q)
      if (length[q] < 0 || length[q] > OTAS_MAX_LONG_SEQ || !rows_fit(c, kv_heads, length[q])) return 0;
    if (recent_ok(offsets, length, B) != OTAS_OK) return 0;
    size_t floats = 1;
    for (bool four : {false, true}) {
      const WindowShape shape = recent_shape(c->desc.dtype, four, c->desc.D / c->desc.H, c->desc.H, kv_heads, offsets, length, B, window, sinks);
      floats = std::max(floats, recent_room_floats(shape, (int64_t)offsets[B] * c->desc.H, c->desc.D / c->desc.H));
    }
    return align_up(floats * sizeof(float), kAlign);
  });
}

otas_status otas_attention_recent(otas_ctx* c, const otas_kv_cache* cache, const void* qkv, const int32_t* offsets, const int32_t* slot,
                                  const int32_t* length, int32_t B, int32_t window, int32_t sinks, const otas_score_desc* score,
                                  void* workspace, size_t workspace_bytes, void* o) {
  return guarded([&]() -> otas_status {
    if (!c || !offsets || !slot || !length || B <= 0 || !offsets_ok(offsets, B)) return OTAS_EINVAL;
    if (offsets[B] > 0 && (!qkv || !workspace || !o)) return OTAS_EINVAL;
    const otas_status st = cache_ok(c, cache);
    if (st != OTAS_OK) return st;
    if (in_cache(c, cache, qkv, qkv_bytes(c, offsets[B], cache->kv_heads))) return OTAS_EINVAL;
    const Cache4Ref ref{(char*)cache->k, (char*)cache->v, nullptr, nullptr, cache->capacity, cache->kv_heads, c->desc.D / c->desc.H, 0};
    return attention_last(c, ref, false, cache->slots, qkv, offsets, slot, length, B, window, sinks, score, workspace, workspace_bytes, o,
                          [&](const void* p, size_t bytes) { return !in_cache(c, cache, p, bytes); });
  });
}

otas_status otas_cache4_append(otas_ctx* c, const otas_kv_cache4* cache, const void* qkv, int64_t T, const int32_t* row_offsets,
                               const int32_t* rows, const int32_t* slot, const int32_t* length, int32_t B, int32_t* length_out) {
  return guarded([&]() -> otas_status {
    if (!c || !row_offsets || !slot || !length || !length_out || B <= 0 || T < 0) return OTAS_EINVAL;
    otas_status st = cache4_ok(c, cache);
    if (st != OTAS_OK) return st;
    if (!aligned16(qkv) || !offsets_ok(row_offsets, B)) return OTAS_EINVAL;
    if (row_offsets[B] > 0 && (!qkv || in_cache4(c, cache, qkv, qkv_bytes(c, T, cache->kv_heads)))) return OTAS_EINVAL;
    st = slots_ok(cache->slots, cache->capacity, slot, length, B, true);
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
    if (N > kMostGroups) return OTAS_EUNSUPPORTED;   // as otas_cache_append
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
      OTAS_LAUNCH(K_MISC, launch_cache4_append(c->desc.dtype, cache4_ref(c, cache), qkv, c->desc.H, plan.data(), plan.size(), c->d_plan, B, N,
                                               rows != nullptr, c->stream));
    }
    for (int q = 0; q < B; ++q) length_out[q] = length[q] + (row_offsets[q + 1] - row_offsets[q]);
    return OTAS_OK;
  });
}

otas_status otas_cache4_read(otas_ctx* c, const otas_kv_cache4* cache, const int32_t* slot, const int32_t* first, const int32_t* row_offsets,
                             int32_t B, void* kv) {
  return guarded([&]() -> otas_status {
    if (!c || !slot || !first || !row_offsets || B <= 0 || !offsets_ok(row_offsets, B)) return OTAS_EINVAL;
    otas_status st = cache4_ok(c, cache);
    if (st != OTAS_OK) return st;
    const int64_t N = row_offsets[B];
    const size_t bytes = (size_t)N * 2 * cache->kv_heads * (c->desc.D / c->desc.H) * elem_size(c->desc.dtype);
    if (!aligned16(kv) || (N > 0 && (!kv || in_cache4(c, cache, kv, bytes)))) return OTAS_EINVAL;
    st = slots_ok(cache->slots, cache->capacity, slot, first, B, false);
    if (st != OTAS_OK) return st;
    for (int q = 0; q < B; ++q)
      if (row_offsets[q + 1] - row_offsets[q] > cache->capacity - first[q]) return OTAS_EINVAL;
    if (N > kMostGroups) return OTAS_EUNSUPPORTED;   // as otas_cache_append
    if (N == 0) return OTAS_OK;
    std::vector<int32_t> plan(3 * (size_t)B + 1);   // row offsets [B+1] | slot [B] | first [B]
    std::copy(row_offsets, row_offsets + B + 1, plan.begin());
    std::copy(slot, slot + B, plan.begin() + B + 1);
    std::copy(first, first + B, plan.begin() + 2 * B + 1);
    OnDevice on(c);
    if (!on.ok) return OTAS_EDEVICE;
    st = place_plan(c, plan);
    if (st != OTAS_OK) return st;
    OTAS_LAUNCH(K_MISC, launch_cache4_read(c->desc.dtype, cache4_ref(c, cache), plan.data(), plan.size(), c->d_plan, B, N, kv, c->stream));
    return OTAS_OK;
  });
}

otas_status otas_attention_cache4(otas_ctx* c, const otas_kv_cache4* cache, const void* qkv, const int32_t* offsets, const int32_t* slot,
                                  const int32_t* length, int32_t B, int32_t window, int32_t sinks, const otas_score_desc* score,
                                  void* workspace, size_t workspace_bytes, void* o) {
  return guarded([&]() -> otas_status {
    if (!c || !offsets || !slot || !length || B <= 0 || !offsets_ok(offsets, B)) return OTAS_EINVAL;
    if (offsets[B] > 0 && (!qkv || !workspace || !o)) return OTAS_EINVAL;
    const otas_status st = cache4_ok(c, cache);
    if (st != OTAS_OK) return st;
    if (in_cache4(c, cache, qkv, qkv_bytes(c, offsets[B], cache->kv_heads))) return OTAS_EINVAL;
    return attention_last(c, cache4_ref(c, cache), true, cache->slots, qkv, offsets, slot, length, B, window, sinks, score, workspace,
                          workspace_bytes, o, [&](const void* p, size_t bytes) { return !in_cache4(c, cache, p, bytes); });
  });
}

}  // extern "C"
