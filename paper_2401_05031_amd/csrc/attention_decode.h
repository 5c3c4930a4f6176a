// What the fp32 and the bf16 attention of the decoder's operators share: which keys a row sees, how products become logits, the
// lines of a tree of drafts.
#pragma once
#include <type_traits>

#include "common.h"
#include "decode_kernels.h"
#include "plan_args.h"

namespace otas {

// A call's host numbers in the kernel's arguments or, where they do not fit, on the device.
struct PlanAny {
  int32_t v[kArgInts];
  const int32_t* p;
  __device__ int32_t operator[](int i) const { return p ? p[i] : v[i]; }
  // For an index that the wave shares: the compiler cannot tell that what comes of either place is the same in all lanes, and without that
  // every address formed from it would be a vector's.
  __device__ int32_t at(int i) const { return __builtin_amdgcn_readfirstlane((*this)[i]); }
};
inline PlanAny plan_any(const int32_t* plan, size_t count, const int32_t* d_plan) {
  PlanAny a;
  a.p = plan_in_args(count) ? nullptr : d_plan;
  if (!a.p) std::memcpy(a.v, plan, count * sizeof(int32_t));
  return a;
}

// Head i of XCD x where the heads of all queries, counted through, divide among the eight.
__device__ inline int xcd_head(int x, int i, int H) {
  if (H % 8) return i * 8 + x;
  const int each = H >> 3, q = i / each;
  return q * H + x * each + i - q * each;
}

struct RowMask {
  int row, document, prefix, causal;
  __device__ bool sees(int j, int doc) const {
    return ((document | doc) >= 0) & ((j < prefix) | ((doc == document) & (!causal | (j <= row))));
  }
};

// Logits of the fp32 kernels, in units of ln 2: exp(s - m) is then one v_exp_f32 (good to a unit in the last place).
struct RowScore {
  float scale, cap, cap2, slope2;
  int position;
  bool sloped;
  static __device__ RowScore of(const ScoreArgs& sc, int head, int position) {
    constexpr float log2e = 1.44269504088896340736f;
    const bool capped = sc.cap > 0.f, sloped = sc.slopes != nullptr;
    return RowScore{capped ? sc.scale / sc.cap : sc.scale * log2e, sc.cap, sc.cap * log2e, sloped ? sc.slopes[head] * log2e : 0.f, position, sloped};
  }
  __device__ float scaled(float s) const { return cap > 0.f ? cap2 * tanhf(s * scale) : s * scale; }
  __device__ float with_distance(float s, int key_position) const { return s - slope2 * fabsf((float)(position - key_position)); }
  __device__ void capped(floatx16& s) const {
    if (cap > 0.f) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = cap2 * tanhf(s[e] * scale);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] *= scale;
    }
  }
};

// f(integral_constant<int, tiles of 32 columns>, bool_constant whether the tiles are whole): the checks of columns of a width that
// is no multiple of 32 take branches and registers that 32, 64, 96 and 128 do without.
template <typename F>
inline hipError_t with_tiles(int dh, F f) {
  auto tiles = [&](auto dt) { return dh % 32 ? f(dt, std::false_type{}) : f(dt, std::true_type{}); };
  switch ((dh + 31) / 32) {
    case 1: return tiles(std::integral_constant<int, 1>{});
    case 2: return tiles(std::integral_constant<int, 2>{});
    case 3: return tiles(std::integral_constant<int, 3>{});
    case 4: return tiles(std::integral_constant<int, 4>{});
  }
  return hipErrorInvalidValue;
}

// What sums relative to m count relative to top >= m.  Nothing of weight so far (m = -inf): they are 0, or NaN where a logit was, and stay.
__device__ __forceinline__ float to_top(float m, float top) { return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top); }

// A 64-bit value of lane `from`.
__device__ inline uint64_t lane_value(uint64_t v, int from) {
  const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)v, from), hi = (uint32_t)__shfl((int)(uint32_t)(v >> 32), from);
  return (uint64_t)hi << 32 | lo;
}

// Lane i: the set of nodes that node i sees, itself among them.  Every node knows its parent (a byte each from plan entry `at`
// on, 255 = none; without has_parents the node before it); in six steps every one adds what its ancestor knows and jumps to the
// ancestor's ancestor, which doubles the distance each time.  All lanes of the wave take part.
template <typename P>
__device__ inline uint64_t tree_lines(const P& plan, int at, int base, int n, bool has_parents, int lane) {
  if (!has_parents) return lane < 63 ? (2ull << lane) - 1 : ~0ull;
  int up = 255;
  if (lane < n) up = (int)((uint32_t)plan[at + ((base + lane) >> 2)] >> (8 * ((base + lane) & 3)) & 255);
  uint64_t line = 1ull << lane;
#pragma unroll
  for (int step = 0; step < 6; ++step) {
    const int from = up == 255 ? lane : up;
    const uint64_t theirs = lane_value(line, from);
    const int next = __shfl(up, from);
    if (up != 255) line |= theirs;
    up = up == 255 ? 255 : next;
  }
  return line;
}

}  // namespace otas
