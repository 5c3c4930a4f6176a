// A wave's 32 rows of fp32 attention, key by key: what the kernels of attention_decode.hip and attention_window.hip share.
#pragma once
#include "attention_decode.h"

namespace otas {

// Both products are formed transposed, so that a lane owns one row: of a block of 32 keys lane half h holds in
// accumulator element e the key 8 (e / 4) + 4 h + (e & 3), which the second product takes as k-slot h of its step e
// straight from registers.
template <typename T, int DT> struct FloatRows {
  floatx4 q[4 * DT];
  floatx16 o[DT];
  float m, l;   // largest logit so far; sum over the lane's keys
};

template <typename T, int DT>
__device__ __forceinline__ void load_heads(floatx4 (&x)[4 * DT], const T* p, int dh, int fk) {   // zero past the head's width
  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int g = 0; g < 4 * DT; ++g) x[g] = 8 * g + 4 * fk < dh ? load4<T>(p + 8 * g + 4 * fk) : zero;
}

template <typename T, int DT>
__device__ __forceinline__ void rows_begin(FloatRows<T, DT>& r, const T* q, int dh, int fk) {
  load_heads<T, DT>(r.q, q, dh, fk);
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) r.o[t][e] = 0.f;
  r.m = -INFINITY;
  r.l = 0.f;
}

// keys: kp, vp the first key's head, ld elements between keys, end their number; logits(s, kb), in place, of the
// products of a block (in units of ln 2, -inf where the lane's row does not see the key); sees(j); partial(kb) whether block kb
// has a pair that does not see each other.  Values are asked for when the first products are under way: one set of registers does
// for keys and values.  From offsets that the compiler knows to be the same in every iteration it forms the 64-bit addresses of all loads ahead of
// the loop, 60 registers a lane: keep_here.  Three waves fit a SIMD at widths up to 64 and two beyond, which is what the loop lives on: it waits for L2, then
// for the matrix cores (fp32, 2 queries of 1500 with 12 heads of 64: 94 -> 83 us from two waves to three; 16 heads of 128: 269 ->
// 215 us from one to two, 76 of 153 TFLOP/s).
template <typename T, int DT, class Keys>
__device__ __forceinline__ void rows_stream(FloatRows<T, DT>& r, const Keys& keys, int dh, int b0, int b1, int step, int fr, int fk) {
  bool odd = false;   // whether values that are not finite were left out where some row does not see some key
  for (int b = b0; b < b1; b += step) {
    const int kb = b * 32, last = keys.end - 1 - kb;   // rows past the last one are the last one again
    floatx16 s;
    {
      floatx4 kf[4 * DT];
      const char* kp = reinterpret_cast<const char*>(keys.kp + (size_t)kb * keys.ld);
      uint32_t mine = (uint32_t)(min(fr, last) * keys.ld + 4 * fk) * (uint32_t)sizeof(T);
      keep_here(mine);
#pragma unroll
      for (int g = 0; g < 4 * DT; ++g)
        kf[g] = 8 * g + 4 * fk < dh ? load4<T>(reinterpret_cast<const T*>(kp + (mine + 8 * g * (uint32_t)sizeof(T)))) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int g = 0; g < 4 * DT; ++g)
        if (8 * g < dh) {
#pragma unroll
          for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[g][u], r.q[g][u], s, 0, 0, 0);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    float vf[DT][16];
    const char* vb = reinterpret_cast<const char*>(keys.vp + (size_t)kb * keys.ld);
    const uint32_t row = (uint32_t)keys.ld * (uint32_t)sizeof(T);
    const bool full = last >= 31;   // wave-uniform: the rows' offsets within a lane half are scalars
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      uint32_t column = (uint32_t)min(32 * t + fr, dh - 1) * (uint32_t)sizeof(T);   // sums past the width are not stored
      if (full) {
        uint32_t at = 4 * fk * row + column;
        keep_here(at);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          vf[t][e] = to_float(*reinterpret_cast<const T*>(vb + (size_t)((8 * (e >> 2) + (e & 3)) * row) + at));
      } else {
        keep_here(column);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          vf[t][e] = to_float(*reinterpret_cast<const T*>(vb + ((uint32_t)min(8 * (e >> 2) + 4 * fk + (e & 3), last) * row + column)));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    keys.logits(s, kb);
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
    mx = xor32_max(mx);
    if (__any(mx > r.m)) {   // some row's maximum moved: rescale what there is
      const float m_new = fmaxf(r.m, mx);
      const float alpha = r.m == m_new ? 1.f : __builtin_amdgcn_exp2f(r.m - m_new);   // equal: also where both are -inf
      r.m = m_new;
      r.l *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) r.o[t][e] *= alpha;
    }
    const float m = r.m == -INFINITY ? 0.f : r.m;   // nothing seen so far: all weights 0
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f(s[e] - m);
      r.l += s[e];
    }
    if (keys.partial(kb)) {   // wave-uniform: a weight of 0 does not keep an infinite value out
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          odd |= !__builtin_isfinite(vf[t][e]);
          vf[t][e] = __builtin_isfinite(vf[t][e]) ? vf[t][e] : 0.f;
        }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int t = 0; t < DT; ++t) r.o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[t][e], s[e], r.o[t], 0, 0, 0);
  }
  if (!__any(odd)) return;
  for (int b = b0; b < b1; b += step) {   // they go to the rows that see them
    if (!keys.partial(b * 32)) continue;
    for (int j = b * 32; j < min(b * 32 + 32, keys.end); ++j) {
      const bool sees = keys.sees(j);
      const T* v = keys.vp + (size_t)j * keys.ld;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * t + 8 * g + 4 * fk;
          if (d < dh) {
            const floatx4 x = load4<T>(v + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) r.o[t][4 * g + e] += sees && !__builtin_isfinite(x[e]) ? x[e] : 0.f;
          }
        }
    }
  }
}

// The four waves' shares of 32 rows into one: every thread then has, of row tid / 8, columns 4 (tid & 7) + 32 i, as sums
// relative to the row's largest logit m, and the weights' sum l.  f(row, column, sums, m, l).
template <int DT> constexpr size_t float_rows_lds() { return sizeof(float) * (256 + 4 * 32 * (32 * DT + 4)); }
template <typename T, int DT, class F>
__device__ __forceinline__ void rows_join(const FloatRows<T, DT>& r, int dh, float* lds, F f) {
  constexpr int LDO = 32 * DT + 4;
  float* ml = lds;         // [4][2][32]
  float* osh = lds + 256;  // [4][32][LDO]
  const int tid = (int)threadIdx.x, wave = tid >> 6, lane = tid & 63, fr = lane & 31, fk = lane >> 5;
  const float l_run = xor32_sum(r.l);
  if (fk == 0) {
    ml[wave * 64 + fr] = r.m;
    ml[wave * 64 + 32 + fr] = l_run;
  }
  __syncthreads();
  float m_all = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) m_all = fmaxf(m_all, ml[w * 64 + fr]);
  const float k = to_top(r.m, m_all);
  float* mine = osh + (wave * 32 + fr) * LDO;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<floatx4*>(mine + 32 * t + 8 * g + 4 * fk) =
          floatx4{r.o[t][4 * g] * k, r.o[t][4 * g + 1] * k, r.o[t][4 * g + 2] * k, r.o[t][4 * g + 3] * k};
  __syncthreads();
  const int row = tid >> 3;
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w * 64 + row]);
#pragma unroll
  for (int w = 0; w < 4; ++w) l += ml[w * 64 + 32 + row] * to_top(ml[w * 64 + row], m);
  for (int d = (tid & 7) * 4; d < dh; d += 32) {
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) v += *reinterpret_cast<const floatx4*>(osh + (w * 32 + row) * LDO + d);
    f(row, d, v, m, l);
  }
}

template <typename T> __device__ __forceinline__ void store_row4(T* p, floatx4 v, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  Quad<T> out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out.x[e] = from_float<T>(l == 0.f ? 0.f : v[e] * inv);
  *reinterpret_cast<Quad<T>*>(p) = out;
}

}  // namespace otas
