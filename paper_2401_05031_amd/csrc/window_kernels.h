// Host-side launchers of the operators of include/otas_decode.h that came with windows and the cache in 4 bits.  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <vector>

#include "decode_kernels.h"

namespace otas {

struct HeadNormArgs {
  const void *q_gain, *k_gain;   // or NULL
  float eps;
  int center, per_head;
};
hipError_t launch_norm_rotary(int dtype, const void* qkv, void* out, const int32_t* positions, int64_t T, int H, int KV, int dh,
                              const HeadNormArgs& n, const RotaryArgs& r, hipStream_t s);

// Which tiles of 2^shift keys rows at places p0 .. p1 see through a window, counted through: those of the sinks that lie before the
// window of the first row, then the window's.
struct WindowTiles {
  int sinks, first, count;   // tiles 0 .. sinks - 1, then first .. first + count - sinks - 1
  __host__ __device__ int tile(int i) const { return i < sinks ? i : i - sinks + first; }
};
__host__ __device__ inline WindowTiles window_tiles(int shift, int p0, int p1, int window, int sinks) {
  const int far = p0 - window + 1 > 0 ? p0 - window + 1 : 0;
  const int s = ((sinks < far ? sinks : far) + (1 << shift) - 1) >> shift;
  const int first = s > far >> shift ? s : far >> shift;
  return WindowTiles{s, first, s + (p1 >> shift) + 1 - first};
}

// A cache in 4 bits; a cache of the model's dtype has no scales.
struct Cache4Ref {
  char *k, *v, *ks, *vs;
  int64_t capacity;
  int KV, dh, groups;   // groups of elements a head
};
// plan: row_off [B+1] | slot [B] | length [B] | rows [N] (has_rows); N = row_off[B]
hipError_t launch_cache4_append(int dtype, const Cache4Ref& c, const void* qkv, int H, const int32_t* plan, size_t count, const int32_t* d_plan, int B,
                                int64_t N, bool has_rows, hipStream_t s);
// plan: row_off [B+1] | slot [B] | first [B]
hipError_t launch_cache4_read(int dtype, const Cache4Ref& c, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int64_t N, void* kv,
                              hipStream_t s);

// How a call through a window is cut up (pure host).  A workgroup has `rows` of a query's n (H / KV) rows of a key head, and `each` of
// the tiles of 2^shift keys that they see; `parts` = most such shares of a group of rows.
constexpr int kRecentShift = 5, kRowsShift = 6;   // of attention_recent.hip, of attention_rows_bf16.hip
constexpr int kManyRows = 128;                    // rows of a workgroup of the latter
struct WorkPlace { int unit, group, part; };      // unit: the query's and its key head's
struct WindowShape {
  int window, sinks, shift, rows, groups, each, parts;
  int room;   // parts that the workspace has place for; >= parts, and grows with the lengths
  int firsts; // where the plan has the groups of rows before every query and of all [B+1]; 0: nowhere, every query has `groups` workgroups' places
  __host__ __device__ WindowTiles tiles(int group, int n, int G, int length) const {
    const int last = (group + 1) * rows < n * G ? (group + 1) * rows - 1 : n * G - 1, at = length - n;
    return window_tiles(shift, at + group * rows / G, at + last / G, window, sinks);
  }
  // Tiles that go side by side: one for each wave, or one that all waves have in LDS.
  __host__ __device__ int at_once() const { return rows == kManyRows ? 1 : 4; }
  // Tiles of a part of these: as many parts as shares of `each` would be, or fewer, but alike.
  __host__ __device__ int each_of(const WindowTiles& t) const {
    const int unit = at_once(), steps = (t.count + unit - 1) / unit, p = (t.count + each - 1) / each;
    return (steps + p - 1) / p * unit;
  }
  __host__ __device__ int parts_of(const WindowTiles& t) const {
    const int e = each_of(t);
    return (t.count + e - 1) / e;
  }
  // The row groups of a share run side by side on one XCD, whose L2 then has the share once.
  __host__ __device__ WorkPlace place(int id, int units) const { return place(id, units, groups); }
  __host__ __device__ WorkPlace place(int id, int units, int groups) const {
    const int shares = units * parts, eights = shares & ~7, span = 8 * groups;
    int group, share;
    if (id < eights * groups) {
      group = id % span / 8;
      share = id / span * 8 + id % 8;
    } else {
      id -= eights * groups;
      group = id / (shares - eights);
      share = eights + id % (shares - eights);
    }
    return WorkPlace{share / parts, groups - 1 - group, share % parts};   // later rows see more keys: first (8192 rows that see all before them, 16 heads of 128: 358 -> 312 us)
  }
  // Workgroup `id` of a call's B queries of KV key heads.
  template <typename P> __host__ __device__ WorkPlace work(const P& plan, int id, int B, int KV) const {
    if (firsts == 0) return place(id, B * KV);
    const int shares = KV * parts, g = id / shares;
    int lo = 0, hi = B;   // the last query that begins at or before group g
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.at(firsts + mid) <= g) lo = mid; else hi = mid;
    }
    const int first = plan.at(firsts + lo);
    WorkPlace w = place(id - first * shares, KV, plan.at(firsts + lo + 1) - first);
    w.unit += lo * KV;
    return w;
  }
  // All workgroups: where queries are counted one by one their own, else as many for each as the longest has.
  int64_t workgroups(const int32_t* plan, int B, int KV) const {
    return (firsts == 0 ? (int64_t)B * groups : plan[firsts + B]) * KV * parts;
  }
  // Counts the queries' groups one by one, at the end of the plan, where more than a quarter of the workgroups would otherwise find no rows and
  // the plan stays where it was (in the kernel's arguments, of `args` numbers, or in memory, of `most`).  A prompt of 4000 rows with 200
  // single tokens (32 heads of 64 on 8, window 1024): 224 us without, 68 with (first launches).
  void count_groups(std::vector<int32_t>& plan, const int32_t* off, int B, int G, size_t args, size_t most) {
    auto of = [&](int q) { return (int)(((int64_t)(off[q + 1] - off[q]) * G + rows - 1) / rows); };
    int64_t all = 0;
    for (int q = 0; q < B; ++q) all += of(q);
    if (all * 4 >= (int64_t)B * groups * 3 || all > INT32_MAX || plan.size() + B + 1 > (plan.size() <= args ? args : most)) return;
    firsts = (int)plan.size();
    plan.push_back(0);
    for (int q = 0; q < B; ++q) plan.push_back(plan.back() + of(q));
  }
};
// rows of a workgroup of attention_recent.hip, or kManyRows
inline int window_rows(int dtype, int dh, int64_t most) {
  if (most <= 16) return 16;
  return most > 32 && dtype != 0 && bf16_width(dh) ? kManyRows : 32;
}
// Workgroups of these kernels that the chip holds at once: by their registers, of the many rows' by LDS (at width 64 it holds three a CU; shares
// for that many took 2 to 5 us longer: 64 rows of 8 queries over 2000 entries, 32 heads on 8, 35.5 and 38.5 us).
inline int window_slots(int dtype, bool four, int rows) {
  return 256 * (rows == 16 ? (four && dtype != 0 ? 3 : 2) : rows == kManyRows ? 2 : 1);
}
// The share of a workgroup is chosen by what a call should take: rounds of workgroups of so many steps (four tiles at once, one a wave; of many
// rows one tile), a launch more and its join where there are several parts.  A step is latency, or the bytes of all workgroups at
// once.  In us, measured: 6 before the first step, 3.5 and a tenth for each part for the join; 1 a step (f32 1.5 at width 64, 3 at 128), 1.3 a tile of many rows (4 bits 2.3) and 1.7 times that
// where two workgroups share a CU; 6.5 TB/s.  Shares counted from every query's own length: one token of 32 queries over 5700 .. 8192 entries of 8 key heads of 128
// in 4 bits 48 us, where shares of the longest query's length in 768 / 256 parts had every third query's last part empty.
inline WindowShape recent_shape(int dtype, bool four, int dh, int H, int KV, const int32_t* off, const int32_t* length, int B, int window, int sinks) {
  const int G = H / KV;
  int64_t most = 0;
  for (int q = 0; q < B; ++q) most = std::max<int64_t>(most, off[q + 1] - off[q]);
  WindowShape t{window, sinks, kRecentShift, 16, 1, 1, 1, 1, 0};
  if (most == 0) return t;
  t.rows = window_rows(dtype, dh, most * G);
  const bool many = t.rows == kManyRows;
  if (many) t.shift = kRowsShift;
  t.groups = (int)((most * G + t.rows - 1) / t.rows);
  std::vector<int32_t> counts;   // tiles of every group of rows of a key head
  int64_t reach = 1;             // as many and more, whatever multiple a window begins at: grows with the lengths
  auto whole = [&](int64_t keys) { return (keys + (1 << t.shift) - 1) >> t.shift; };
  for (int q = 0; q < B; ++q) {
    const int n = off[q + 1] - off[q], mine = (int)(((int64_t)n * G + t.rows - 1) / t.rows);
    for (int g = 0; g < mine; ++g) counts.push_back(t.tiles(g, n, G, length[q]).count);
    if (n > 0)
      reach = std::max(reach, std::min(whole(length[q]), whole(std::min(sinks, length[q])) + whole((int64_t)std::min(window, length[q]) + t.rows / G + 1) + 1));
  }
  const int longest = *std::max_element(counts.begin(), counts.end()), slots = window_slots(dtype, four, t.rows), at_once = t.at_once();
  const double bytes = at_once * (2 << t.shift) * (four ? dh / 2 + (dh + 31) / 32 : dh * (dtype == 0 ? 4.0 : 2.0));
  const double latency = many ? (four ? 2.3 : 1.3) : dtype == 0 ? dh / 43.0 : 1.0;
  double best = 1e30;
  t.each = longest;
  for (int steps = (longest + at_once - 1) / at_once; steps > 0; steps -= std::max(1, steps / 12)) {
    const int each = steps * at_once;
    int64_t wgs = 0;
    for (const int32_t c : counts) wgs += (c + each - 1) / each;
    wgs *= KV;
    const int64_t active = std::min<int64_t>(wgs, slots), rounds = (wgs + slots - 1) / slots;
    if (each < longest && rounds > 2) break;   // more workgroups take longer from here on
    const double step = std::max(many && active > slots / 2 ? 1.7 * latency : latency, active * bytes / 6.5e6);
    const double us = rounds * (6 + steps * step) + (each < longest ? 3.5 + 0.1 * ((longest + each - 1) / each) : 0);
    if (us < best) {
      best = us;
      t.each = each;
    }
  }
  t.parts = t.parts_of(WindowTiles{0, 0, longest});
  for (const int32_t c : counts) t.parts = std::max(t.parts, t.parts_of(WindowTiles{0, 0, c}));
  // Every group of rows has a workgroup of each key head, and no more than two rounds are chosen.
  const int64_t most_parts = std::max<int64_t>(1, 2 * slots / KV - ((int64_t)counts.size() - 1));
  t.room = (int)std::min(most_parts, (reach + at_once - 1) / at_once);
  return t;
}
// Floats of workspace: of calls of several parts, for each largest logits and weight sums [T H][2] and sums [T H][dh], from a multiple
// of four on.
inline size_t recent_sums_at(const WindowShape& t, int64_t TH) { return ((size_t)TH * 2 * t.parts + 3) / 4 * 4; }
inline size_t recent_workspace_floats(const WindowShape& t, int64_t TH, int dh) {
  return t.parts > 1 ? recent_sums_at(t, TH) + (size_t)TH * t.parts * dh : 0;
}
inline size_t recent_room_floats(const WindowShape& t, int64_t TH, int dh) { return t.room > 1 ? (size_t)TH * t.room * (dh + 2) + 3 : 0; }
struct RecentBuffers {
  float *sums, *tops;
  int64_t TH;
};
// plan: off [B+1] | slot [B] | length [B], then what the shape has counted.  four: in 4 bits, else of the model's dtype.
hipError_t launch_attention_recent(int dtype, bool four, const Cache4Ref& c, const void* qkv, int H, const int32_t* plan, size_t count,
                                   const int32_t* d_plan, int B, int64_t T, const ScoreArgs& sc, const WindowShape& shape, float* workspace, void* o,
                                   hipStream_t s);
// Of several parts it leaves their sums in the buffers.  c.k NULL: packed rows' own keys, plan: off [B+1], then what the shape has counted.
hipError_t launch_attention_rows_bf16(bool four, const Cache4Ref& c, const void* qkv, int H, const int32_t* plan, size_t count, const int32_t* d_plan, int B,
                                      const ScoreArgs& sc, const WindowShape& shape, const RecentBuffers& buf, void* o, hipStream_t s);
// Packed rows: one share of all tiles.  Of fp32 products a workgroup has 32 rows of one head of `heads` H, else 128 of one of KV key heads.
inline WindowShape packed_shape(int dtype, int dh, int H, int KV, int max_n, int window, int sinks) {
  const bool many = dtype != 0 && bf16_width(dh);
  WindowShape t{window, sinks, many ? kRowsShift : kRecentShift, many ? kManyRows : 32, 0, 1, 1, 1, 0};   // `each` is not looked at
  t.groups = (int)(((int64_t)max_n * (many ? H / KV : 1) + t.rows - 1) / t.rows);
  return t;
}
// plan: off [B+1], then what the shape has counted
hipError_t launch_attention_window(int dtype, const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int H, int KV, int dh,
                                   const ScoreArgs& sc, const WindowShape& shape, void* o, hipStream_t s);

}  // namespace otas
