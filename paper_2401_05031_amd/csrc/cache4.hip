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

// A workgroup has ROWS rows, one after the other, and asks for them together; runs of workgroups to each XCD, whose L2 then puts together the
// scales of entries side by side.
__device__ __forceinline__ int first_row(int id, int N, int rows) { return ((id & 7) * ((N + 8 * rows - 1) / (8 * rows)) + (id >> 3)) * rows; }
inline unsigned row_groups(int64_t N, int rows) { return (unsigned)((N + 8 * rows - 1) / (8 * rows) * 8); }
inline int cache4_rows(int64_t N) { return N >= 4096 ? 4 : 1; }   // several where that leaves work for all CUs
// Where row i goes or comes from; lo: the query of an earlier row, or -1.
struct RowPlace { int64_t slot, entry; };
template <typename P> __device__ __forceinline__ RowPlace row_place(const P& plan, int B, int i, int& lo) {
  if (lo < 0) {   // the last query that begins at or before the row
    lo = 0;
    int hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan[mid] <= i) lo = mid; else hi = mid;
    }
  }
  while (plan[lo + 1] <= i) ++lo;
  return RowPlace{plan[B + 1 + lo], (int64_t)plan[2 * B + 1 + lo] + (i - plan[lo])};
}

// A thread has eight elements of a head, four threads a group, whose largest element goes round them in registers.  Memory-bound: 12700 rows of
// 8 + 8 heads of 128 bf16 (66 MB with what is written, part of it from and to the last-level cache) 14.5 us, 32 rows 3.9 us.  A row a workgroup 18 us;
// with conversions in plain arithmetic and no runs of rows to each XCD, whose scales then go out byte by byte, 24.
template <typename T, int ROWS, typename P>
__global__ __launch_bounds__(256) void cache4_append_kernel(Cache4Ref c, const T* __restrict__ qkv, int H, P plan, int B, int N, bool has_rows) {
  const int i0 = first_row((int)blockIdx.x, N, ROWS);
  if (i0 >= N) return;
  RowPlace at[ROWS];
  const T* src[ROWS];
  int lo = -1;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {   // rows past the last are that one again, and are not stored
    const int i = min(i0 + r, N - 1);
    at[r] = row_place(plan, B, i, lo);
    src[r] = qkv + ((int64_t)(has_rows ? plan[3 * B + 1 + i] : i) * (H + 2 * c.KV) + H) * c.dh;
  }
  const int words = c.dh / 8, per_head = 4 * c.groups, total = 2 * c.KV * per_head;
  for (int u0 = 0; u0 < total; u0 += 256) {
    const int u = u0 + (int)threadIdx.x, h = u / per_head, w = u - h * per_head, kh = h < c.KV ? h : h - c.KV;
    const bool there = u < total && w < words;
    Oct<T> x[ROWS];
    if (there) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) x[r] = *reinterpret_cast<const Oct<T>*>(src[r] + (int64_t)h * c.dh + w * 8);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      uint32_t largest = 0;
      if (there) {
#pragma unroll
        for (int j = 0; j < 8; ++j) largest = max(largest, __float_as_uint(to_float(x[r].x[j])) & 0x7FFFFFFFu);
      }
      largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, kDppXor1, 0xF, 0xF, true));
      largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, kDppXor2, 0xF, 0xF, true));
      if (!there || i0 + r >= N) continue;
      const uint32_t byte = scale4_byte(largest), word = byte == kNoNumber ? 0 : codes4(x[r], scale4(byte));
      const int64_t head = at[r].slot * c.KV + kh;
      *reinterpret_cast<uint32_t*>((h < c.KV ? c.k : c.v) + (head * c.capacity + at[r].entry) * (c.dh / 2) + w * 4) = word;
      if (w % 4 == 0) (h < c.KV ? c.ks : c.vs)[(head * c.groups + w / 4) * c.capacity + at[r].entry] = (char)byte;
    }
  }
}

// A thread has eight elements of a head.  Memory-bound: 12700 rows 14.3 us (a row a workgroup 16), 32 rows 3.7 us.
template <typename T, int ROWS, typename P>
__global__ __launch_bounds__(256) void cache4_read_kernel(Cache4Ref c, P plan, int B, int N, T* __restrict__ kv) {
  const int i0 = first_row((int)blockIdx.x, N, ROWS);
  if (i0 >= N) return;
  RowPlace at[ROWS];
  int lo = -1;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) at[r] = row_place(plan, B, min(i0 + r, N - 1), lo);
  const int words = c.dh / 8, total = 2 * c.KV * words;
  for (int u = (int)threadIdx.x; u < total; u += 256) {
    const int h = u / words, w = u - h * words, kh = h < c.KV ? h : h - c.KV;
    uint32_t word[ROWS], byte[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int64_t head = at[r].slot * c.KV + kh;
      word[r] = *reinterpret_cast<const uint32_t*>((h < c.KV ? c.k : c.v) + (head * c.capacity + at[r].entry) * (c.dh / 2) + w * 4);
      byte[r] = (uint8_t)(h < c.KV ? c.ks : c.vs)[(head * c.groups + w / 4) * c.capacity + at[r].entry];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (i0 + r >= N) break;
      const float f = scale4(byte[r]);
      const floatx2 p0 = pair4<0>(word[r], f), p1 = pair4<1>(word[r], f), p2 = pair4<2>(word[r], f), p3 = pair4<3>(word[r], f);
      const float v[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
      Oct<T> x;
#pragma unroll
      for (int j = 0; j < 8; ++j) x.x[j] = from_float<T>(byte[r] == kNoNumber ? __uint_as_float(0x7FC00000u) : v[j]);
      *reinterpret_cast<Oct<T>*>(kv + ((int64_t)(i0 + r) * 2 * c.KV + h) * c.dh + w * 8) = x;
    }
  }
}

hipError_t launch_cache4_append(int dtype, const Cache4Ref& c, const void* qkv, int H, const int32_t* plan, size_t count, const int32_t* d_plan, int B,
                                int64_t N, bool has_rows, hipStream_t s) {
  if (N <= 0) return hipSuccess;
  return with_plan(plan, count, d_plan, [&](auto p) {
    typedef decltype(p) P;
    auto run = [&](auto zero, auto rows) {
      typedef decltype(zero) E;
      constexpr int ROWS = decltype(rows)::value;
      cache4_append_kernel<E, ROWS, P><<<dim3(row_groups(N, ROWS)), dim3(256), 0, s>>>(c, (const E*)qkv, H, p, B, (int)N, has_rows);
      return hipGetLastError();
    };
    auto by_rows = [&](auto zero) { return cache4_rows(N) == 4 ? run(zero, std::integral_constant<int, 4>{}) : run(zero, std::integral_constant<int, 1>{}); };
    return dtype == 0 ? by_rows(0.f) : by_rows(bf16_t{});
  });
}

hipError_t launch_cache4_read(int dtype, const Cache4Ref& c, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int64_t N, void* kv,
                              hipStream_t s) {
  if (N <= 0) return hipSuccess;
  return with_plan(plan, count, d_plan, [&](auto p) {
    typedef decltype(p) P;
    auto run = [&](auto zero, auto rows) {
      typedef decltype(zero) E;
      constexpr int ROWS = decltype(rows)::value;
      cache4_read_kernel<E, ROWS, P><<<dim3(row_groups(N, ROWS)), dim3(256), 0, s>>>(c, p, B, (int)N, (E*)kv);
      return hipGetLastError();
    };
    auto by_rows = [&](auto zero) { return cache4_rows(N) == 4 ? run(zero, std::integral_constant<int, 4>{}) : run(zero, std::integral_constant<int, 1>{}); };
    return dtype == 0 ? by_rows(0.f) : by_rows(bf16_t{});
  });
}

}  // namespace otas
