// C ABI of the decoder's operators (include/otas_decode.h): argument validation and launches.
#include <hip/hip_runtime.h>

#include "decode_checks.h"

using namespace otas;

static_assert(OTAS_DECODE_ARGUMENTS == kArgInts && (size_t)OTAS_MAX_LONG_SEQ <= kPlanInts, "documented limits");

extern "C" {

otas_status otas_rotary(otas_ctx* c, const void* qkv, int64_t T, int32_t kv_heads, const int32_t* positions,
                        const otas_rotary_desc* rope, void* out) {
  return guarded([&]() -> otas_status {
    if (!c || !rope || T < 0 || !kv_heads_ok(c, kv_heads)) return OTAS_EINVAL;
    if (T > 0 && (!qkv || !positions || !out)) return OTAS_EINVAL;   // no rows, no arrays
    const int dh = c->desc.D / c->desc.H;
    const otas_rotary_desc& d = *rope;
    if (!rotary_desc_ok(d, dh)) return OTAS_EINVAL;
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
        overlap(workspace, floats * sizeof(float), qkv, in_bytes) || in_cache(c, cache, qkv, in_bytes) || in_cache(c, cache, o, out_bytes) ||
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
