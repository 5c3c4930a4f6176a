// Rotary positions on packed rows, and packed rows into the cache: both move every byte once and are bound by HBM.
#include "common.h"
#include "decode_kernels.h"
#include "plan_args.h"
#include "rotary_angles.h"

namespace otas {

// ------------------------------------------------------------------------------------------------ rotary positions
// A workgroup has `tokens` rows.  First its threads put the cosine and sine of every (row, pair) into LDS: one double
// product and a reduction to a fraction of a turn per angle (a float product at position 2^17 would be off by 2^17 2^-24
// turns), then sincospif, shared by all heads of the row.  Then they walk the rows in chunks of V elements (16 bytes where
// heads and pairs allow it).  A chunk of the first half of the pairs is turned together with its partner by one thread,
// so that a call in place has no other thread read what it writes.  Memory-bound: a row's bytes in and out once (16384 bf16 rows of
// 16 + 2 x 8 heads of 128, 268 MB: 50 us, 5.3 TB/s; as many float rows of 12 + 2 x 12 heads of 64, 302 MB: 51 us; 37 rows 3.9 us, a launch's latency).
template <typename T, int V>
__global__ __launch_bounds__(256) void rotary_kernel(const T* qkv, T* out, const int32_t* __restrict__ positions, int64_t rows, int heads,
                                                     int W, int dh, int tokens, RotaryArgs r) {
  __shared__ float2 cs[8 * 64];
  const int pairs = r.rot >> 1;
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int nt = (int)min((int64_t)tokens, rows - t0);
  rotary_angles(cs, positions, t0, nt, r);
  const bool copies = out != qkv;
  const int per_row = W / V, per_head = dh / V;
  typedef Chunk<T, V> C;
  for (int i = (int)threadIdx.x; i < nt * per_row; i += 256) {
    const int t = i / per_row, u = i - t * per_row, h = u / per_head, e = (u - h * per_head) * V;
    const int64_t at = (t0 + t) * W + (int64_t)u * V;
    const float2* a = cs + t * 64;
    if (h >= heads || e >= r.rot) {   // values, and what of a head does not turn
      if (copies) *reinterpret_cast<C*>(out + at) = *reinterpret_cast<const C*>(qkv + at);
    } else if (r.interleaved) {
      C x = *reinterpret_cast<const C*>(qkv + at);
#pragma unroll
      for (int j = 0; j < V; j += 2)
        if (e + j < r.rot) {   // a chunk can hold the last pair and what follows it
          const float2 w = a[(e + j) >> 1];
          const float lo = to_float(x.x[j]), hi = to_float(x.x[j + 1]);
          x.x[j] = from_float<T>(lo * w.x - hi * w.y);
          x.x[j + 1] = from_float<T>(lo * w.y + hi * w.x);
        }
      *reinterpret_cast<C*>(out + at) = x;
    } else if (e < pairs) {       // pairs % V == 0 here
      C lo = *reinterpret_cast<const C*>(qkv + at), hi = *reinterpret_cast<const C*>(qkv + at + pairs);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float2 w = a[e + j];
        const float x = to_float(lo.x[j]), y = to_float(hi.x[j]);
        lo.x[j] = from_float<T>(x * w.x - y * w.y);
        hi.x[j] = from_float<T>(x * w.y + y * w.x);
      }
      *reinterpret_cast<C*>(out + at) = lo;
      *reinterpret_cast<C*>(out + at + pairs) = hi;
    }
  }
}

// Halves of a number of pairs that no chunk divides: a chunk's partners then begin inside another chunk.  Every thread puts
// its chunk into LDS, the whole heads of a round at a time, and takes the partners from there one by one; a round's
// heads are in LDS before its first store, so that a call in place reads nothing that is turned already.  The next round's chunks are asked for before the
// barrier.  Against chunks as narrow as the halves allow (16384 bf16 rows of 16 + 2 x 2 heads of 128): 122 turned elements
// 85 -> 30 us, 120 (chunks of 4 before) 36 -> 30 us, next to 28 us for all 128; without the early loads 41 us.
template <typename T, int V>
__global__ __launch_bounds__(256) void rotary_odd_halves_kernel(const T* qkv, T* out, const int32_t* __restrict__ positions, int64_t rows,
                                                                int heads, int all_heads, int dh, int tokens, RotaryArgs r) {
  __shared__ float2 cs[8 * 64];
  __shared__ alignas(16) T part[2][256 * V];
  const int pairs = r.rot >> 1;
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int nt = (int)min((int64_t)tokens, rows - t0);
  rotary_angles(cs, positions, t0, nt, r);
  const bool copies = out != qkv;
  const int per_head = dh / V, round = 256 / per_head, own = (int)threadIdx.x / per_head, e = ((int)threadIdx.x - own * per_head) * V;
  const int turned = copies ? all_heads : heads;   // values move only into another array
  typedef Chunk<T, V> C;
  int buffer = 0;
  C next;
  auto where = [&](int i) {
    const int t = i / turned, h = i - t * turned;
    return ((t0 + t) * all_heads + h) * dh + e;
  };
  const bool placed = own < round;
  if (placed && own < nt * turned) next = *reinterpret_cast<const C*>(qkv + where(own));
  for (int i0 = 0; i0 < nt * turned; i0 += round, buffer ^= 1) {
    const int i = i0 + own;
    const bool mine = placed && i < nt * turned;
    const int t = i / turned, h = i - t * turned;
    const int64_t at = where(i);
    T* head = part[buffer] + own * dh;
    C x = next;
    if (mine) *reinterpret_cast<C*>(head + e) = x;
    if (placed && i + round < nt * turned) next = *reinterpret_cast<const C*>(qkv + where(i + round));
    __syncthreads();   // the round after next writes this buffer, behind the next round's barrier
    if (!mine) continue;
    if (h < heads && e < r.rot) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int p = e + j;
        if (p < r.rot) {
          const bool low = p < pairs;
          const float2 w = cs[t * 64 + (low ? p : p - pairs)];
          const float other = to_float(head[low ? p + pairs : p - pairs]);
          x.x[j] = from_float<T>(to_float(x.x[j]) * w.x + other * (low ? -w.y : w.y));
        }
      }
    } else if (!copies) {
      continue;
    }
    *reinterpret_cast<C*>(out + at) = x;
  }
}

hipError_t launch_rotary(int dtype, const void* qkv, void* out, const int32_t* positions, int64_t T, int H, int KV, int dh,
                         const RotaryArgs& r, hipStream_t s) {
  if (T <= 0) return hipSuccess;
  const int W = (H + 2 * KV) * dh, pairs = r.rot / 2;
  // Rows per workgroup: angles of several rows keep all threads busy, but a small call wants its rows on many CUs.
  const int tokens = T >= 8192 ? 8 : T >= 2048 ? 4 : T >= 1024 ? 2 : 1;
  const int64_t wgs = (T + tokens - 1) / tokens;
  if (wgs > kMostGroups) return kTooManyGroups;
  const int wide = dtype == 0 ? 4 : 8;
  const int v = dh % wide ? 4 : wide;   // dh % 4 == 0
#define OTAS_ROTARY(T_, V_)                                                                                                     \
  do {                                                                                                                          \
    const dim3 grid((unsigned)wgs), block(256);                                                                                 \
    if (r.interleaved || pairs % V_ == 0)                                                                                       \
      rotary_kernel<T_, V_><<<grid, block, 0, s>>>((const T_*)qkv, (T_*)out, positions, T, H + KV, W, dh, tokens, r);           \
    else                                                                                                                        \
      rotary_odd_halves_kernel<T_, V_><<<grid, block, 0, s>>>((const T_*)qkv, (T_*)out, positions, T, H + KV, H + 2 * KV, dh,   \
                                                              tokens, r);                                                       \
  } while (0)
  if (dtype == 0) OTAS_ROTARY(float, 4);
  else if (v == 8) OTAS_ROTARY(bf16_t, 8);
  else OTAS_ROTARY(bf16_t, 4);
#undef OTAS_ROTARY
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------- rows into the cache
// A workgroup copies one row: its 2 KV heads lie side by side in the row and capacity d_h elements apart in the cache, so
// that one head's keys are one run of memory for the attention that reads them.  Memory-bound: 12700 rows of 8 + 8 heads of 128 bf16
// (104 MB read and written) in 17.5 us, part of them from the last-level cache; 32 rows 3.1 us.
template <typename T, int V, typename P>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheRef c, const T* __restrict__ qkv, int H, const int32_t* __restrict__ positions,
                                                           P plan, int B, bool has_rows) {
  const int i = (int)blockIdx.x;
  int lo = 0, hi = B;                       // the query of row i: the last one that begins at or before it
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (plan[mid] <= i) lo = mid; else hi = mid;
  }
  const int q = lo;
  const int64_t slot = plan[B + 1 + q], entry = plan[2 * B + 1 + q] + (i - plan[q]);
  const int64_t row = has_rows ? plan[3 * B + 1 + i] : i;
  const int per_head = c.dh / V, n = c.KV * per_head;
  const T* src = qkv + (row * (H + 2 * c.KV) + H) * c.dh;
  typedef Chunk<T, V> C;
  for (int u = (int)threadIdx.x; u < 2 * n; u += 256) {
    const int h = u / per_head, e = (u - h * per_head) * V, kh = h < c.KV ? h : h - c.KV;
    T* dst = (T*)(h < c.KV ? c.k : c.v) + ((slot * c.KV + kh) * c.capacity + entry) * c.dh + e;
    *reinterpret_cast<C*>(dst) = *reinterpret_cast<const C*>(src + (int64_t)h * c.dh + e);
  }
  if (threadIdx.x == 0) {
    c.positions[slot * c.capacity + entry] = positions[row];
    if (c.mass) c.mass[slot * c.capacity + entry] = 0.f;
  }
}

hipError_t launch_cache_append(int dtype, const CacheRef& c, const void* qkv, int H, const int32_t* positions, const int32_t* plan,
                               size_t count, const int32_t* d_plan, int B, int64_t N, bool has_rows, hipStream_t s) {
  if (N <= 0) return hipSuccess;
  return with_plan(plan, count, d_plan, [&](auto p) {
    typedef decltype(p) P;
    const dim3 grid((unsigned)N), block(256);
    if (dtype == 0) cache_append_kernel<float, 4, P><<<grid, block, 0, s>>>(c, (const float*)qkv, H, positions, p, B, has_rows);
    else if (c.dh % 8 == 0) cache_append_kernel<bf16_t, 8, P><<<grid, block, 0, s>>>(c, (const bf16_t*)qkv, H, positions, p, B, has_rows);
    else cache_append_kernel<bf16_t, 4, P><<<grid, block, 0, s>>>(c, (const bf16_t*)qkv, H, positions, p, B, has_rows);
    return hipGetLastError();
  });
}

}  // namespace otas
