// Rows into a cache of 4 bits an element and back: every element read once, an element in eight bits' half written.
#include "cache4.h"
#include "plan_args.h"
#include "rotary_angles.h"

namespace otas {

// Eight elements as codes: v_cvt_scalef32_pk_fp4_f32 divides by the scale, rounds to the nearest (of two as near to the one of even code)
// and holds what is larger at 6.
template <typename T> __device__ __forceinline__ uint32_t codes4(const Oct<T>& x, float scale) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, to_float(x.x[0]), to_float(x.x[1]), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, to_float(x.x[2]), to_float(x.x[3]), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, to_float(x.x[4]), to_float(x.x[5]), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, to_float(x.x[6]), to_float(x.x[7]), scale, 3);
}

// Row of a workgroup: runs of rows to each XCD, whose L2 then puts together the scales of entries side by side.
__device__ __forceinline__ int row_of(int id, int each) { return (id & 7) * each + (id >> 3); }

template <typename P> __device__ __forceinline__ int query_of(const P& plan, int B, int i) {   // the last one that begins at or before row i
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (plan[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

// A workgroup has one row.  A thread has eight elements of a head, four threads a group, whose largest element goes round them in
// registers.
template <typename T, typename P>
__global__ __launch_bounds__(256) void cache4_append_kernel(Cache4Ref c, const T* __restrict__ qkv, int H, P plan, int B, int N, bool has_rows) {
  const int i = row_of((int)blockIdx.x, (N + 7) >> 3);
  if (i >= N) return;
  const int q = query_of(plan, B, i);
  const int64_t slot = plan[B + 1 + q], entry = plan[2 * B + 1 + q] + (i - plan[q]);
  const int64_t row = has_rows ? plan[3 * B + 1 + i] : i;
  const int words = c.dh / 8, per_head = 4 * c.groups, total = 2 * c.KV * per_head;
  const T* src = qkv + (row * (H + 2 * c.KV) + H) * c.dh;
  for (int u0 = 0; u0 < total; u0 += 256) {
    const int u = u0 + (int)threadIdx.x, h = u / per_head, w = u - h * per_head, kh = h < c.KV ? h : h - c.KV;
    const bool there = u < total && w < words;
    Oct<T> x;
    uint32_t largest = 0;
    if (there) {
      x = *reinterpret_cast<const Oct<T>*>(src + (int64_t)h * c.dh + w * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) largest = max(largest, __float_as_uint(to_float(x.x[j])) & 0x7FFFFFFFu);
    }
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, kDppXor1, 0xF, 0xF, true));
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, kDppXor2, 0xF, 0xF, true));
    if (!there) continue;
    const uint32_t byte = scale4_byte(largest), word = byte == kNoNumber ? 0 : codes4(x, scale4(byte));
    const int64_t head = slot * c.KV + kh;
    *reinterpret_cast<uint32_t*>((h < c.KV ? c.k : c.v) + (head * c.capacity + entry) * (c.dh / 2) + w * 4) = word;
    if (w % 4 == 0) (h < c.KV ? c.ks : c.vs)[(head * c.groups + w / 4) * c.capacity + entry] = (char)byte;
  }
}

hipError_t launch_cache4_append(int dtype, const Cache4Ref& c, const void* qkv, int H, const int32_t* plan, size_t count, const int32_t* d_plan, int B,
                                int64_t N, bool has_rows, hipStream_t s) {
  if (N <= 0) return hipSuccess;
  return with_plan(plan, count, d_plan, [&](auto p) {
    typedef decltype(p) P;
    const dim3 grid((unsigned)((N + 7) / 8 * 8)), block(256);
    if (dtype == 0) cache4_append_kernel<float, P><<<grid, block, 0, s>>>(c, (const float*)qkv, H, p, B, (int)N, has_rows);
    else cache4_append_kernel<bf16_t, P><<<grid, block, 0, s>>>(c, (const bf16_t*)qkv, H, p, B, (int)N, has_rows);
    return hipGetLastError();
  });
}

// A workgroup has one row, a thread eight elements of a head.
template <typename T, typename P>
__global__ __launch_bounds__(256) void cache4_read_kernel(Cache4Ref c, P plan, int B, int N, T* __restrict__ kv) {
  const int i = row_of((int)blockIdx.x, (N + 7) >> 3);
  if (i >= N) return;
  const int q = query_of(plan, B, i);
  const int64_t slot = plan[B + 1 + q], entry = plan[2 * B + 1 + q] + (i - plan[q]);
  const int words = c.dh / 8, total = 2 * c.KV * words;
  for (int u = (int)threadIdx.x; u < total; u += 256) {
    const int h = u / words, w = u - h * words, kh = h < c.KV ? h : h - c.KV;
    const int64_t head = slot * c.KV + kh;
    const uint32_t word = *reinterpret_cast<const uint32_t*>((h < c.KV ? c.k : c.v) + (head * c.capacity + entry) * (c.dh / 2) + w * 4);
    const uint32_t byte = (uint8_t)(h < c.KV ? c.ks : c.vs)[(head * c.groups + w / 4) * c.capacity + entry];
    const float f = scale4(byte);
    const floatx2 p0 = pair4<0>(word, f), p1 = pair4<1>(word, f), p2 = pair4<2>(word, f), p3 = pair4<3>(word, f);
    const float v[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    Oct<T> x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x.x[j] = from_float<T>(byte == kNoNumber ? __uint_as_float(0x7FC00000u) : v[j]);
    *reinterpret_cast<Oct<T>*>(kv + ((int64_t)i * 2 * c.KV + h) * c.dh + w * 8) = x;
  }
}

hipError_t launch_cache4_read(int dtype, const Cache4Ref& c, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int64_t N, void* kv,
                              hipStream_t s) {
  if (N <= 0) return hipSuccess;
  return with_plan(plan, count, d_plan, [&](auto p) {
    typedef decltype(p) P;
    const dim3 grid((unsigned)((N + 7) / 8 * 8)), block(256);
    if (dtype == 0) cache4_read_kernel<float, P><<<grid, block, 0, s>>>(c, p, B, (int)N, (float*)kv);
    else cache4_read_kernel<bf16_t, P><<<grid, block, 0, s>>>(c, p, B, (int)N, (bf16_t*)kv);
    return hipGetLastError();
  });
}

}  // namespace otas
