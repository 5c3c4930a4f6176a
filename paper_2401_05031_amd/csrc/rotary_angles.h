// What the kernels that turn heads share: runs of elements and the angles of a workgroup's rows.
#pragma once
#include "common.h"
#include "decode_kernels.h"

namespace otas {

template <typename T, int V> struct alignas(V * sizeof(T)) Chunk { T x[V]; };

// The cosines and sines of the pairs of nt rows from t0 on, those of a row 64 apart.  All threads of the workgroup.
__device__ __forceinline__ void rotary_angles(float2* cs, const int32_t* __restrict__ positions, int64_t t0, int nt, const RotaryArgs& r) {
  const int pairs = r.rot >> 1;
  for (int i = (int)threadIdx.x; i < nt * pairs; i += 256) {
    const int t = i / pairs, p = i - t * pairs;
    const double turn = (double)positions[t0 + t] * r.turns[p];
    float sn, c;
    sincospif((float)(2.0 * (turn - rint(turn))), &sn, &c);
    cs[t * 64 + p] = make_float2(c * r.magnitude, sn * r.magnitude);
  }
  __syncthreads();
}

}  // namespace otas
