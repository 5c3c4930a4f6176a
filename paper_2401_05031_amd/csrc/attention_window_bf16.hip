// otas_attention_window in bf16: four waves of 32 rows each walk the keys that any of them sees in tiles of 64, which travel from
// global memory into the one LDS buffer while the other is worked on; one barrier a tile, as in attention_masked_bf16.hip.
//   Where heads share a key head, the waves are HW of those heads and 32 * 4 / HW rows, in place of 128 rows of one head: the keys that
// rows see move with the rows, and a workgroup walks all that any of its rows sees.  With a window w and 128 rows that is
// w + 128 keys a workgroup, of which a wave sees w + 32; four heads of 32 rows see the same.
#include "attention_tiles.h"
#include "window_kernels.h"

namespace otas {

namespace {
constexpr int kKeys = 64;
}

template <int DH> constexpr size_t window_buffer() { return 2 * TileRows<DH>::bytes(kKeys) + value_slack<DH>(); }
template <int DH> constexpr size_t window_lds() { return 2 * window_buffer<DH>() + 16; }

template <int DH, int HW, int CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void attention_window_bf16_kernel(const bf16_t* __restrict__ qkv, PlanAny plan, int B, int H, int KV, int xblks,
                                                                       ScoreArgs sc, CapArgs cap, int window, int sinks, bf16_t* __restrict__ o) {
  typedef TileRows<DH> R;
  constexpr size_t KB = R::bytes(kKeys), BUF = window_buffer<DH>();   // keys | values | slack
  constexpr int ROWS = 32 * 4 / HW;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  // Row blocks of the same heads one XCD's, where the heads divide so: their windows overlap.
  const int id = (int)blockIdx.x, HG = H / HW, pairs = B * HG;
  int pair, xblk;
  if (pairs % 8 == 0) {
    const int mine = pairs >> 3, k = id >> 3;
    pair = xcd_head(id & 7, k % mine, HG);
    xblk = xblks - 1 - k / mine;
  } else {
    pair = id % pairs;
    xblk = xblks - 1 - id / pairs;
  }
  const int q = pair / HG, row0 = xblk * ROWS;
  const int base = plan.at(q), n = plan.at(q + 1) - base;
  if (row0 >= n) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), fr = lane & 31, fk = lane >> 5;
  const int h = pair % HG * HW + wave % HW, wrow0 = row0 + wave / HW * 32, row = min(wrow0 + fr, n - 1);
  const bool active = wrow0 < n;
  const size_t ld = (size_t)(H + 2 * KV) * DH;
  const bf16_t* first = qkv + (size_t)base * ld;
  const int kh = pair % HG * HW / (H / KV);
  const char* kbase = reinterpret_cast<const char*>(first + (size_t)(H + kh) * DH);
  const char* vbase = reinterpret_cast<const char*>(first + (size_t)(H + KV + kh) * DH);
  const uint32_t ldb = (uint32_t)(ld * sizeof(bf16_t));
  const int last = min(row0 + ROWS, n) - 1, wlast = min(wrow0 + 31, last);   // of the workgroup's rows, of the wave's
  const WindowTiles tiles = window_tiles<kKeys>(row0, last, window, sinks);

  TileLoader<DH, kKeys, 4, false> key_loader;
  TileLoader<DH, kKeys, 4, true> value_loader;
  key_loader.begin(wave, lane);
  value_loader.begin(wave, lane);
  auto fetch = [&](int t, char* buf) {
    const size_t at = (size_t)t * kKeys * ldb;
    key_loader.load(kbase + at, ldb, n - 1 - t * kKeys, buf);
    value_loader.load(vbase + at, ldb, n - 1 - t * kKeys, buf + KB);
  };
  const Score2 score = Score2::of(sc, BIAS ? sc.slopes[h] : 0.f, row);
  // Whether rows a .. b all see all of the tile from kb on, and whether any of them sees any.
  auto all_see = [&](int a, int b, int kb) { return kb + kKeys - 1 <= a && (kb > b - window || kb + kKeys <= sinks); };
  auto some_see = [&](int a, int b, int kb) { return kb <= b && (kb + kKeys - 1 > a - window || kb < sinks); };
  bool met = false;   // whether this wave took out a value that is not finite

  fetch(tiles.tile(0), lds);
  WaveRows<DH> w;
  w.begin(first + (size_t)row * ld + (size_t)h * DH, fk, sc.scale < 0.f);
  for (int i = 0; i < tiles.count; ++i) {
    wait_all();   // this wave's part of the tile is there
    char* buf = lds + (i & 1 ? BUF : 0);
    const int kb = tiles.tile(i) * kKeys;
    // Of a tile that some row does not see all of, values that are not finite are taken out and come back at the end, to
    // the rows that see them.
    if (!all_see(row0, last, kb)) met |= value_loader.make_finite(buf + KB, lane, [&](int r) { return kb + r <= last; });
    wait_lds_barrier();   // all of it, and nobody reads the other buffer any more
    if (i + 1 < tiles.count) fetch(tiles.tile(i + 1), lds + (i & 1 ? 0 : BUF));
    if (active && some_see(wrow0, wlast, kb)) {   // wave-uniform
      __builtin_amdgcn_s_setprio(0);
      floatx16 s[2];
      tile_products<DH, 2>(s, w, buf, 0, fr, fk);
      short8_t v[WaveRows<DH>::DT];
      first_values<DH>(v, buf + KB, 0, lane);
      __builtin_amdgcn_s_setprio(1);   // a wave that needs the vector ALU goes before one at its products, as in attention_masked_bf16.hip
      const bool whole = all_see(wrow0, wlast, kb);
      bool done = false;
      if (CAP && !BIAS && whole) done = tile_weights_capped<DH, 2>(w, s, cap);
      if (CAP && !done) tile_capped<CAP, 2>(s, score, cap);
      const int behind = row - kb - 4 * fk;   // the row's distance from the lane's first key
      if (BIAS) {
        const float near = (float)behind;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float d = near - (float)(32 * b + 8 * (e >> 2) + (e & 3));
            s[b][e] = fmaf(-score.slope2, fabsf(d), CAP ? s[b][e] : s[b][e] * score.scale2);
          }
      }
      if (!whole) {
        if (kb >= sinks) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[b][e] = (uint32_t)(behind - (32 * b + 8 * (e >> 2) + (e & 3))) < (uint32_t)window ? s[b][e] : -INFINITY;
        } else {
          const int left = sinks - kb - 4 * fk;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int j = 32 * b + 8 * (e >> 2) + (e & 3);
              const bool see = (j <= behind) & ((behind - j < window) | (j < left));
              s[b][e] = see ? s[b][e] : -INFINITY;
            }
        }
      }
      if (!done) tile_weights<DH, 2>(w, s, CAP || BIAS ? 1.f : score.scale2);
      __builtin_amdgcn_s_setprio(0);
      tile_sums<DH, 2>(w, s, v, buf + KB, 0, lane);
    }
  }
  if (any_wave(met, reinterpret_cast<int*>(lds + 2 * BUF), wave, lane)) {   // workgroup-uniform
    for (int i = 0; i < tiles.count; ++i) {
      const int kb = tiles.tile(i) * kKeys;
      if (all_see(row0, last, kb)) continue;
      for (int j = kb; j < min(kb + kKeys, last + 1); ++j) {
        const bool see = j <= row && (row - j < window || j < sinks);
        const bf16_t* v = reinterpret_cast<const bf16_t*>(vbase + (size_t)j * ldb);
#pragma unroll
        for (int c = 0; c < WaveRows<DH>::DT; ++c)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            if (c * 32 + g * 8 < DH) add_not_finite(w.o[c], g, v + c * 32 + g * 8 + fk * 4, see);
      }
    }
  }
  const float l = xor32_sum(w.l);
  if (wrow0 + fr >= n) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bf16_t* orow = o + (size_t)(base + wrow0 + fr) * H * DH + (size_t)h * DH;
#pragma unroll
  for (int c = 0; c < WaveRows<DH>::DT; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = c * 32 + g * 8 + fk * 4;
      if (d < DH) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (bf16_t)(l == 0.f ? 0.f : w.o[c][4 * g + e] * inv);
        *reinterpret_cast<bf16x4*>(orow + d) = v;
      }
    }
}

hipError_t launch_attention_window_bf16(const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int max_n, int H, int KV,
                                        int dh, const ScoreArgs& sc, int window, int sinks, void* o, hipStream_t s) {
  const int G = H / KV;
  const PlanAny p = plan_any(plan, count, d_plan);
  auto run = [&](auto width, auto hw, auto cap, auto bias) {
    constexpr int DH = decltype(width)::value, HW = decltype(hw)::value;
    const int xblks = (max_n + 32 * 4 / HW - 1) / (32 * 4 / HW);
    const int64_t wgs = (int64_t)xblks * (H / HW) * B;
    if (wgs > kMostGroups) return kTooManyGroups;
    auto kern = attention_window_bf16_kernel<DH, HW, decltype(cap)::value, decltype(bias)::value>;
    const hipError_t e = set_max_dynamic_lds((const void*)kern, (int)window_lds<DH>());
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)wgs), dim3(256), window_lds<DH>(), s>>>((const bf16_t*)qkv, p, B, H, KV, xblks, sc, CapArgs::of(sc), window, sinks, (bf16_t*)o);
    return hipGetLastError();
  };
  auto by_heads = [&](auto width, auto cap, auto bias) {
    if (G % 4 == 0) return run(width, std::integral_constant<int, 4>{}, cap, bias);
    if (G % 2 == 0) return run(width, std::integral_constant<int, 2>{}, cap, bias);
    return run(width, std::integral_constant<int, 1>{}, cap, bias);
  };
  auto pick = [&](auto width) {
    auto with_bias = [&](auto cap) { return sc.slopes ? by_heads(width, cap, std::true_type{}) : by_heads(width, cap, std::false_type{}); };
    switch (Score2::cap_form(sc.cap)) {
      case 0: return with_bias(std::integral_constant<int, 0>{});
      case 1: return with_bias(std::integral_constant<int, 1>{});
    }
    return with_bias(std::integral_constant<int, 2>{});
  };
  switch (dh) {
    case 64: return pick(std::integral_constant<int, 64>{});
    case 80: return pick(std::integral_constant<int, 80>{});
    case 96: return pick(std::integral_constant<int, 96>{});
    case 128: return pick(std::integral_constant<int, 128>{});
  }
  return hipErrorInvalidValue;
}

}  // namespace otas
