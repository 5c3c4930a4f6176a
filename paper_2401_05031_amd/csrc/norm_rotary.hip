// Norms of query and key heads with rotary positions in the same pass: y = (x - c) r gain, r = 1 / sqrt(mean (x - c)^2 + eps), then the
// pairs of y turned.  Every byte moves once: bound by HBM (16384 bf16 rows of 16 + 2 x 8 heads of 128, 268 MB: 51.6 us, 5.2 TB/s; asking for the next
// head ahead 64 -> 52 us); 9 float rows 4.4 us, a launch's latency.
//   A head has L lanes of a wave (a power of two), V elements each: sums over a head are exchanges within the wave, and so are
// the partners of pairs that lie in halves, which go through LDS as floats (a lane's V partners are one run there where the
// chunks divide the half).  The norm needs all of a head before any of it is stored, so that a call in place needs no more care.
#include "rotary_angles.h"
#include "window_kernels.h"

namespace otas {

template <int L> __device__ __forceinline__ float lanes_sum(float v) {   // over every L lanes; all 64 active
  static_assert(L <= 32, "128 elements, four and more a lane");
  if (L >= 32) v = xor16_sum(v);
  if (L >= 16) {   // a rotation by half of the period that the values have reached is the butterfly's partner
    v = dpp_sum<dpp_ror(8)>(v);
    v = dpp_sum<dpp_ror(4)>(v);
    v = dpp_sum<dpp_ror(2)>(v);
    return dpp_sum<dpp_ror(1)>(v);
  }
  if (L >= 2) v = dpp_sum<kDppXor1>(v);
  if (L >= 4) v = dpp_sum<kDppXor2>(v);
  if (L >= 8) v = dpp_sum<kDppHalfMirror>(v);
  return v;
}

template <typename T, int V, int L>
__global__ __launch_bounds__(256) void norm_rotary_kernel(const T* qkv, T* out, const int32_t* __restrict__ positions, int64_t rows, int H, int KV,
                                                          int dh, int tokens, HeadNormArgs n, RotaryArgs r) {
  __shared__ __attribute__((aligned(16))) float2 cs[4 * 64];
  __shared__ __attribute__((aligned(16))) float turned[256 * V];
  const int pairs = r.rot >> 1, all_heads = H + 2 * KV;
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int nt = (int)min((int64_t)tokens, rows - t0);
  if (r.rot) rotary_angles(cs, positions, t0, nt, r);
  const int lane_of = (int)threadIdx.x % L, own = (int)threadIdx.x / L, e = lane_of * V;
  const bool there = e < dh;
  const int heads = out != qkv ? all_heads : H + KV;   // values move only into another array
  typedef Chunk<T, V> C;
  float* mine = turned + own * (L * V);
  const float inv = 1.f / (float)dh;
  const bool whole_halves = pairs % V == 0;   // a chunk's partners are one run
  C gains[2];                                 // shared by all heads
  const bool shared = !n.per_head;
  if (shared && there) {
    if (n.q_gain) gains[0] = *reinterpret_cast<const C*>((const T*)n.q_gain + e);
    if (n.k_gain) gains[1] = *reinterpret_cast<const C*>((const T*)n.k_gain + e);
  }
  // Where head i of the workgroup's lies: its row and its place there move on by so many a round.
  const int step_t = 256 / L / heads, step_h = 256 / L % heads;
  int t = own / heads, h = own - t * heads;
  auto where = [&](int t, int h) { return ((t0 + t) * all_heads + h) * dh + e; };
  C next;
  if (there && t < nt) next = *reinterpret_cast<const C*>(qkv + where(t, h));
  for (int i0 = 0; i0 < nt * heads; i0 += 256 / L) {
    const bool active = there && t < nt;
    const int64_t at = where(t, h);
    C x = next;
    int t_next = t + step_t, h_next = h + step_h;
    if (h_next >= heads) { h_next -= heads; ++t_next; }
    if (there && t_next < nt) next = *reinterpret_cast<const C*>(qkv + where(t_next, h_next));
    float y[V];
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = active ? to_float(x.x[j]) : 0.f;
    if (n.center) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) s += y[j];
      const float mean = lanes_sum<L>(s) * inv;
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = there ? y[j] - mean : 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) s += y[j] * y[j];
    const float scale = 1.f / sqrtf(fmaf(lanes_sum<L>(s), inv, n.eps));
    const bool query = h < H, norm = active && h < H + KV;
    if (norm) {
      const T* g = (const T*)(query ? n.q_gain : n.k_gain);
      C gain = query ? gains[0] : gains[1];
      if (g && !shared) gain = *reinterpret_cast<const C*>(g + (int64_t)(query ? h : h - H) * dh + e);
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = y[j] * scale * (g ? to_float(gain.x[j]) : 1.f);
    }
    if (r.rot && !r.interleaved) {   // partners: elements pairs away.  A head's lanes are one wave's, whose LDS operations keep their order
#pragma unroll
      for (int j = 0; j < V; j += 4) *reinterpret_cast<floatx4*>(mine + e + j) = floatx4{y[j], y[j + 1], y[j + 2], y[j + 3]};
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (norm && e < r.rot) {
        const float2* a = cs + t * 64;
        float z[V];
        if (whole_halves) {
          const bool low = e < pairs;
          const float* other = mine + (low ? e + pairs : e - pairs);
          const float4* w = reinterpret_cast<const float4*>(a + (low ? e : e - pairs));   // cosine and sine of two pairs
          const float sign = low ? -1.f : 1.f;
#pragma unroll
          for (int j = 0; j < V; j += 4) {
            const floatx4 p = *reinterpret_cast<const floatx4*>(other + j);
            const float4 w0 = w[j / 2], w1 = w[j / 2 + 1];
            z[j] = y[j] * w0.x + p[0] * (sign * w0.y);
            z[j + 1] = y[j + 1] * w0.z + p[1] * (sign * w0.w);
            z[j + 2] = y[j + 2] * w1.x + p[2] * (sign * w1.y);
            z[j + 3] = y[j + 3] * w1.z + p[3] * (sign * w1.w);
          }
        } else
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int p = e + j;
          const bool low = p < pairs;
          const float2 w = a[low ? p : min(p - pairs, 63)];
          const float other = mine[low ? p + pairs : p - pairs];
          z[j] = p < r.rot ? y[j] * w.x + other * (low ? -w.y : w.y) : y[j];
        }
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = z[j];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else if (r.rot && norm) {
#pragma unroll
      for (int j = 0; j < V; j += 2)
        if (e + j < r.rot) {
          const float2 w = cs[t * 64 + ((e + j) >> 1)];
          const float lo = y[j], hi = y[j + 1];
          y[j] = lo * w.x - hi * w.y;
          y[j + 1] = lo * w.y + hi * w.x;
        }
    }
    if (norm) {
#pragma unroll
      for (int j = 0; j < V; ++j) x.x[j] = from_float<T>(y[j]);
    }
    if (active) *reinterpret_cast<C*>(out + at) = x;
    t = t_next;
    h = h_next;
  }
}

hipError_t launch_norm_rotary(int dtype, const void* qkv, void* out, const int32_t* positions, int64_t T, int H, int KV, int dh,
                              const HeadNormArgs& n, const RotaryArgs& r, hipStream_t s) {
  if (T <= 0) return hipSuccess;
  // Rows per workgroup: angles of several keep all threads busy (16384 rows: 2 55 us, 4 52, 8 55), but a small call wants its rows on many CUs.
  const int tokens = T >= 2048 ? 4 : T >= 1024 ? 2 : 1;
  const int64_t wgs = (T + tokens - 1) / tokens;
  if (wgs > kMostGroups) return kTooManyGroups;
  auto run = [&](auto zero, auto v, auto lanes) {
    typedef decltype(zero) E;
    norm_rotary_kernel<E, decltype(v)::value, decltype(lanes)::value>
        <<<dim3((unsigned)wgs), dim3(256), 0, s>>>((const E*)qkv, (E*)out, positions, T, H, KV, dh, tokens, n, r);
    return hipGetLastError();
  };
  auto by_lanes = [&](auto zero, auto v) {
    const int lanes = (dh + decltype(v)::value - 1) / decltype(v)::value;
    if (lanes <= 1) return run(zero, v, std::integral_constant<int, 1>{});
    if (lanes <= 2) return run(zero, v, std::integral_constant<int, 2>{});
    if (lanes <= 4) return run(zero, v, std::integral_constant<int, 4>{});
    if (lanes <= 8) return run(zero, v, std::integral_constant<int, 8>{});
    if (lanes <= 16) return run(zero, v, std::integral_constant<int, 16>{});
    return run(zero, v, std::integral_constant<int, 32>{});
  };
  if (dtype == 0) return by_lanes(0.f, std::integral_constant<int, 4>{});
  if (dh % 8) return by_lanes(bf16_t{}, std::integral_constant<int, 4>{});
  return by_lanes(bf16_t{}, std::integral_constant<int, 8>{});
}

}  // namespace otas
