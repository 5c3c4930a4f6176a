// otas_attention_window with fp32 products (f32 models, and bf16 ones of head widths that attention_rows_bf16.hip is not built for):
// row i sees row j of its query where j <= i and (i - j < window or j < sinks).  As attention_masked_f32_kernel, over the blocks of
// 32 keys that any of a workgroup's 32 rows sees: first those of the sinks before its window, then the window's.  Bound by a workgroup's chain of
// latencies (launch, plan, queries, one block a wave, join: 8 us for 36 workgroups of one row each) and by how many workgroups go through it side by side:
// 3 x 182 .. 260 float rows, 12 heads on 4 of 64, window 64, 324 workgroups of one to four blocks: 12 us, 144 of the same 9.
#include "attention_rows_f32.h"
#include "window_kernels.h"

namespace otas {

template <typename T> struct WindowKeys {
  const T *kp, *vp;
  int ld, end;                        // keys from `end` on are seen by no row of the workgroup
  int row, window, sinks;
  int sure, late, fk;                 // keys below `sure` are no row's future, those from `late` on in every row's window; the lane's half
  RowScore score;
  __device__ bool sees(int j) const { return j <= row && (row - j < window || j < sinks); }
  __device__ void logits(floatx16& s, int kb) const {
    score.capped(s);
    if (score.sloped) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = score.with_distance(s[e], kb + 8 * (e >> 2) + 4 * fk + (e & 3));
    }
    if (partial(kb)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = sees(kb + 8 * (e >> 2) + 4 * fk + (e & 3)) ? s[e] : -INFINITY;
    }
  }
  __device__ bool partial(int kb) const { return kb + 32 > sure || (kb < late && kb + 32 > sinks); }
};

template <typename T, int DT, bool WHOLE>
__global__ __launch_bounds__(256, DT <= 2 ? 3 : 2) void attention_window_f32_kernel(PlanAny plan_, const T* __restrict__ qkv, int B, int H, int KV, int width,
                                                                   ScoreArgs sc, WindowShape shape, T* __restrict__ o) {
  extern __shared__ __attribute__((aligned(16))) float f32_lds[];
  const PlanFirst plan = PlanFirst::of(plan_);
  // The row blocks of a head on one XCD where heads divide so.
  int q, h, xblk;
  if (shape.firsts) {
    const WorkPlace at = shape.work(plan, (int)blockIdx.x, B, H);
    q = at.unit / H;
    h = at.unit % H;
    xblk = at.group;
  } else {
    const int id = (int)blockIdx.x, pairs = B * H, xblks = shape.groups;
    int pair;
    if (pairs % 8 == 0) {
      const int mine = pairs >> 3, k = id >> 3;
      pair = xcd_head(id & 7, k % mine, H);
      xblk = xblks - 1 - k / mine;
    } else {
      pair = id % pairs;
      xblk = xblks - 1 - id / pairs;
    }
    h = pair % H;
    q = pair / H;
  }
  const int dh = WHOLE ? 32 * DT : width, window = shape.window, sinks = shape.sinks;
  const int base = plan.at(q), n = plan.at(q + 1) - base, row0 = xblk * 32;
  if (row0 >= n) return;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), fr = lane & 31, fk = lane >> 5;
  const int last = min(row0 + 31, n - 1), row = min(row0 + fr, last);
  const size_t ld = (size_t)(H + 2 * KV) * dh;
  const T* first = qkv + (size_t)base * ld;
  const int kh = h / (H / KV);
  const WindowKeys<T> keys{first + (size_t)(H + kh) * dh, first + (size_t)(H + KV + kh) * dh, (int)ld, last + 1, row, window, sinks,
                           row0 + 1, max(0, last - window + 1), fk, RowScore::of(sc, h, row)};
  FloatRows<T, DT> r;
  rows_begin<T, DT>(r, first + (size_t)row * ld + (size_t)h * dh, dh, fk);
  const WindowTiles tiles = window_tiles(5, row0, last, window, sinks);
  rows_stream<T, DT>(r, keys, dh, wave, tiles.sinks, 4, fr, fk);
  rows_stream<T, DT>(r, keys, dh, tiles.first + ((wave - tiles.sinks) & 3), tiles.first + tiles.count - tiles.sinks, 4, fr, fk);
  T* out = o + ((size_t)base + row0) * H * dh + (size_t)h * dh;
  rows_join<T, DT>(r, dh, f32_lds, [&](int i, int d, floatx4 v, float, float l) {
    if (row0 + i < n) store_row4<T>(out + (size_t)i * H * dh + d, v, l);
  });
}

template <typename T>
static hipError_t attention_window_f32(const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int H, int KV, int dh,
                                       const ScoreArgs& sc, const WindowShape& shape, void* o, hipStream_t s) {
  const int64_t wgs = shape.workgroups(plan, B, H);
  if (wgs > kMostGroups) return kTooManyGroups;
  const PlanAny p = plan_any(plan, count, d_plan);
  return with_tiles(dh, [&](auto dt, auto whole) {
    constexpr int DT = decltype(dt)::value;
    auto kern = attention_window_f32_kernel<T, DT, decltype(whole)::value>;
    const hipError_t e = set_max_dynamic_lds((const void*)kern, (int)float_rows_lds<DT>());
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)wgs), dim3(256), float_rows_lds<DT>(), s>>>(p, (const T*)qkv, B, H, KV, dh, sc, shape, (T*)o);
    return hipGetLastError();
  });
}

hipError_t launch_attention_window(int dtype, const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int H, int KV, int dh,
                                   const ScoreArgs& sc, const WindowShape& shape, void* o, hipStream_t s) {
  if (shape.groups <= 0) return hipSuccess;
  if (shape.rows == kManyRows)
    return launch_attention_rows_bf16(false, Cache4Ref{nullptr, nullptr, nullptr, nullptr, 0, KV, dh, 0}, qkv, H, plan, count, d_plan, B, sc, shape,
                                      RecentBuffers{nullptr, nullptr, 0}, o, s);
  return dtype == 0 ? attention_window_f32<float>(qkv, plan, count, d_plan, B, H, KV, dh, sc, shape, o, s)
                    : attention_window_f32<bf16_t>(qkv, plan, count, d_plan, B, H, KV, dh, sc, shape, o, s);
}

}  // namespace otas
