// The parts of a tree's rows joined, for both types of attention_decode.hip and attention_tree_bf16.hip: maxima in units of ln 2.
// Bound by latency (3.8 us for one token of 14 parts: the launch and two round trips to L2) or, with weights added up from the logits, by
// their bytes (32 x 16 rows over 8192 entries: 8 us for 15 MB of logits, from L2).
#pragma once
#include "attention_decode.h"

namespace otas {

// Largest logit and weight sum of a row from its parts' (stride TH): four at a time, so that the loads overlap.
__device__ __forceinline__ float2 join_ends(const float* tops, int64_t TH, int64_t at, int parts) {
  float m = -INFINITY, l = 0.f;
  for (int p0 = 0; p0 < parts; p0 += 4) {
    float2 e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = *reinterpret_cast<const float2*>(tops + 2 * (min(p0 + i, parts - 1) * TH + at));
    float top = m;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, e[i].x);
    l *= to_top(m, top);
#pragma unroll
    for (int i = 0; i < 4; ++i) l += p0 + i < parts ? e[i].y * to_top(e[i].x, top) : 0.f;
    m = top;
  }
  return make_float2(m, l);
}

// The chunks of every row joined, a wave a row (the first join_wgs workgroups), and beside it, where the logits are at hand, the
// weights of 256 entries of a query added up over its rows (the others): mass_j += sum_i exp(s_ij - m_i) / l_i.  A lane has four
// entries and a wave every fourth row, in order; the waves are added in order.  With an entry a thread and all rows one after the
// other the loads were long chains (calls of 17 x 14 nodes and 16 heads over 2 entries 46 -> 26 us, 4 x 14 over 3000 92 -> 31 us).
template <typename T>
__global__ __launch_bounds__(256) void attention_tree_join_kernel(CacheRef c, PlanAny plan, int B, int H, int dh, TreeShape shape, TreeBuffers in,
                                                                       int join_wgs, int xblks, T* __restrict__ o) {
  extern __shared__ __attribute__((aligned(16))) float2 ends[];   // m, 1 / l of the query's rows
  __shared__ floatx4 shares[4][64];
  const int tid = (int)threadIdx.x;
  if ((int)blockIdx.x < join_wgs) {
    const int64_t at = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63;
    if (at >= in.TH) return;
    const int row = (int)(at / H);
    int lo = 0, hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.at(mid) <= row) lo = mid; else hi = mid;
    }
    const int parts = shape.parts_of(plan.at(2 * B + 1 + lo));
    if (parts <= 1) return;   // written already
    // lane d has columns 2 d and 2 d + 1; eight parts at a time, so that their loads overlap
    const bool mine = 2 * lane < dh;
    float2 acc = {0.f, 0.f}, e = {-INFINITY, 0.f};   // e: largest logit, weight sum
    for (int p0 = 0; p0 < parts; p0 += 8) {
      float2 t[8], v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t p = min(p0 + i, parts - 1) * in.TH + at;
        t[i] = *reinterpret_cast<const float2*>(in.tops + 2 * p);
        v[i] = *reinterpret_cast<const float2*>(in.sums + p * dh + (mine ? 2 * lane : 0));
      }
      float top = e.x;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, t[i].x);
      const float f = to_top(e.x, top);
      acc.x *= f; acc.y *= f; e.y *= f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (p0 + i < parts) {   // wave-uniform; also where the factor is 0: NaN stays
          const float k = to_top(t[i].x, top);
          e.y += k * t[i].y;
          acc.x += k * v[i].x;
          acc.y += k * v[i].y;
        }
      }
      e.x = top;
    }
    const float inv = e.y == 0.f ? 0.f : 1.f / e.y;
    if (mine) {
      struct alignas(2 * sizeof(T)) Pair { T x[2]; } out;
      out.x[0] = from_float<T>(e.y == 0.f ? 0.f : acc.x * inv);
      out.x[1] = from_float<T>(e.y == 0.f ? 0.f : acc.y * inv);
      *reinterpret_cast<Pair*>(o + at * dh + 2 * lane) = out;
    }
    if (in.ends && lane == 0) { in.ends[2 * at] = e.x; in.ends[2 * at + 1] = e.y; }
    return;
  }
  const int id = (int)blockIdx.x - join_wgs, q = id / xblks, e0 = (id % xblks) * 256;
  const int base = plan.at(q), n = plan.at(q + 1) - base, len = plan.at(2 * B + 1 + q), parts = shape.parts_of(len);
  const int64_t slot = plan.at(B + 1 + q);
  if (e0 >= len || n == 0) return;   // workgroup-uniform
  for (int r = tid; r < n * H; r += 256) {
    const int64_t at = (int64_t)base * H + r;
    const float2 e = parts <= 1 ? make_float2(in.ends[2 * at], in.ends[2 * at + 1]) : join_ends(in.tops, in.TH, at, parts);
    ends[r] = e.y == 0.f ? make_float2(0.f, 0.f) : make_float2(e.x, 1.f / e.y);
  }
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  floatx4 got = {0.f, 0.f, 0.f, 0.f};
  if (e0 + 4 * lane < len) {   // up to three past the end: within the stride
    const float* s = in.logits + (int64_t)base * H * in.stride + e0 + 4 * lane;
#pragma unroll 8
    for (int r = wave; r < n * H; r += 4) {
      const float2 e = ends[r];
      const floatx4 x = *reinterpret_cast<const floatx4*>(s + (int64_t)r * in.stride);
#pragma unroll
      for (int i = 0; i < 4; ++i) got[i] += e.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(x[i] - e.x) * e.y;
    }
  }
  shares[wave][lane] = got;
  __syncthreads();
  const int j = e0 + tid;
  if (j >= len) return;
  auto share = [&](int w) { return reinterpret_cast<const float*>(&shares[w][0])[tid]; };
  c.mass[slot * c.capacity + j] += (share(0) + share(1)) + (share(2) + share(3));
}

// mass_blocks: blocks of 256 entries a query whose weights are to be added up from logits, or 0.
template <typename T>
inline hipError_t launch_attention_tree_join(const CacheRef& c, const PlanAny& plan, int B, int H, const TreeShape& shape, const TreeBuffers& in,
                                             int64_t join_wgs, int mass_blocks, void* o, hipStream_t s) {
  const size_t lds = mass_blocks ? 32 * (size_t)c.KV * sizeof(float2) : 0;   // rows of 32 a key head at most
  attention_tree_join_kernel<T><<<dim3((unsigned)(join_wgs + (int64_t)B * mass_blocks)), dim3(256), lds, s>>>(c, plan, B, H, c.dh, shape, in, (int)join_wgs,
                                                                                                              mass_blocks, (T*)o);
  return hipGetLastError();
}

}  // namespace otas
