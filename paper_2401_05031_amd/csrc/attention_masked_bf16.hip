// otas_attention_masked in bf16: four waves have 128 rows of a head and walk the keys that any of them sees in tiles of 64, which
// travel from global memory into the one LDS buffer while the other is worked on; one barrier a tile.
//   Two workgroups, eight waves, fill a CU's registers (2 a SIMD; 3 would spill from width 80 on and gave nothing at 64).  128 rows read
// a tile once for four waves; with 64 keys a tile is as large as two buffers and two workgroups leave room for.  Bound by the matrix
// cores and the vector ALU in turn, which hardly overlap: 64 logits of a wave at width 128 take one matrix instruction (32 clocks) and 10
// vector ones (4 each, most at full rate), and of 8192 capped causal rows' 7.0e8 SIMD clocks the matrix cores are busy in 2.7e8 and the
// vector ALU in 4.0e8.  At a clock of 1.9 - 2.0 GHz those rows take 330 us with 16 heads of 128, 0.84 PFLOP/s where a large matrix product
// reaches 1.27; without a cap 290 us (0.95), 16 heads of 80 229 us (0.75), 64 199 us (0.69).
// 3 x 4000 rows of seven documents with slopes take 95 us: a workgroup has 7 tiles of 2.3 us each (3.5 where keys are masked) after
// 5 us for its plan, the kinds of tiles and the first tile.
#include "attention_tiles.h"

namespace otas {

namespace {
constexpr int kRows = 128, kKeys = 64;

// Which tiles of 64 keys a workgroup has to look at: one byte each, bit w: some row of wave w may see some key, bit 4 + w: every key has
// the one document of all rows of wave w (or is a prefix key, seen by all).
__device__ __forceinline__ int next_tile(const unsigned char* kinds, int t, int tiles, int lane) {   // wave-uniform
  for (; t < tiles; t += 64) {
    const uint64_t some = __ballot(t + lane < tiles && (kinds[min(t + lane, tiles - 1)] & 15));
    if (some) return t + __ffsll((unsigned long long)some) - 1;
  }
  return tiles;
}

// The smallest and the largest of every 16 lanes (rotations within them), in all of them.
template <int ROTATION> __device__ __forceinline__ int rotated(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x120 + ROTATION, 0xF, 0xF, false); }
__device__ __forceinline__ int least16(int x) {
  x = min(x, rotated<8>(x)); x = min(x, rotated<4>(x)); x = min(x, rotated<2>(x));
  return min(x, rotated<1>(x));
}
__device__ __forceinline__ int most16(int x) {
  x = max(x, rotated<8>(x)); x = max(x, rotated<4>(x)); x = max(x, rotated<2>(x));
  return max(x, rotated<1>(x));
}
}  // namespace

template <int DH> constexpr size_t masked_buffer() { return 2 * TileRows<DH>::bytes(kKeys) + value_slack<DH>() + 512; }
template <int DH> constexpr size_t masked_lds(int max_n, bool documents) {
  return 2 * masked_buffer<DH>() + 16 + (documents ? (size_t)(max_n + kKeys - 1) / kKeys + 64 : 0);
}

template <int DH, int CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void attention_masked_bf16_kernel(const bf16_t* __restrict__ qkv, PlanAny plan, int B, int H, int KV, int xblks,
                                                                       int by_xcd, ScoreArgs sc, CapArgs cap, MaskArgs mk, bf16_t* __restrict__ o) {
  typedef TileRows<DH> R;
  constexpr size_t KB = R::bytes(kKeys), BUF = masked_buffer<DH>();   // keys | values | slack | positions | documents
  extern __shared__ __attribute__((aligned(16))) char lds[];
  // Work in the order in which it is handed out: the last row blocks of all heads first (under a causal mask they have the most
  // keys).  Where the heads divide among the eight XCDs each XCD has its own, whose keys then stay in its L2: of every query as many
  // as of any other (a query's heads on one XCD would leave a long query of a ragged batch to it alone), side by side where a
  // query has eights of them (heads that share keys).
  int id = (int)blockIdx.x, pair, xblk;
  const int pairs = B * H;
  if (by_xcd) {
    const int mine = pairs >> 3, k = id >> 3;
    pair = xcd_head(id & 7, k % mine, H);
    xblk = xblks - 1 - k / mine;
  } else {
    pair = id % pairs;
    xblk = xblks - 1 - id / pairs;
  }
  const int h = pair % H, q = pair / H;
  const int base = plan.at(q), n = plan.at(q + 1) - base, row0 = xblk * kRows, prefix = plan.at(B + 1 + q);
  if (row0 >= n) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), fr = lane & 31, fk = lane >> 5;
  const int wrow0 = row0 + wave * 32, row = min(wrow0 + fr, n - 1);
  const bool active = wrow0 < n;
  const size_t ld = (size_t)(H + 2 * KV) * DH;
  const bf16_t* first = qkv + (size_t)base * ld;
  const int kh = h / (H / KV);
  const char* kbase = reinterpret_cast<const char*>(first + (size_t)(H + kh) * DH);
  const char* vbase = reinterpret_cast<const char*>(first + (size_t)(H + KV + kh) * DH);
  const int32_t* docs = mk.documents ? mk.documents + base : nullptr;
  const int32_t* pos = BIAS && mk.positions ? mk.positions + base : nullptr;
  const uint32_t ldb = (uint32_t)(ld * sizeof(bf16_t));

  const int end = mk.causal ? max(min(row0 + kRows, n), prefix) : n, tiles = (end + kKeys - 1) / kKeys;
  unsigned char* kinds = reinterpret_cast<unsigned char*>(lds + 2 * BUF + 16);
  const int my_doc = docs ? docs[row] : 0;
  WaveRows<DH> w;
  if (docs) {
    // A wave looks at 4 x 4 tiles at a time, 16 lanes each.  All that it needs for that and its queries are asked for together.
    int d[4][4], rows_doc[kRows / 64];
    auto ask = [&](int t0) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[u][i] = docs[min((t0 + 16 * u + (lane >> 4)) * kKeys + i * 16 + (lane & 15), n - 1)];
    };
#pragma unroll
    for (int i = 0; i < kRows / 64; ++i) rows_doc[i] = docs[min(row0 + i * 64 + lane, n - 1)];
    ask(wave * 4);
    w.begin(first + (size_t)row * ld + (size_t)h * DH, fk, sc.scale < 0.f);
    // The documents of each wave's rows: smallest and largest, padding aside, and whether there is but the one.  Lane l has wave l & 3's.
    int lo = 0, hi = 0;
    bool one = false;
#pragma unroll
    for (int i = 0; i < kRows / 64; ++i) {
      const int d = rows_doc[i];
      int least = d < 0 ? INT32_MAX : d, most = max(d, -1);
#pragma unroll
      for (int x = 16; x; x >>= 1) { least = min(least, __shfl_xor(least, x)); most = max(most, __shfl_xor(most, x)); }
      const uint64_t padded = __ballot(d < 0);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int l = __builtin_amdgcn_readlane(least, 32 * half), m = __builtin_amdgcn_readlane(most, 32 * half);
        if ((lane & 3) == 2 * i + half) { lo = l; hi = m; one = l == m && (uint32_t)(padded >> 32 * half) == 0; }
      }
    }
    for (int t0 = wave * 4; t0 < tiles; t0 += 64) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int t = t0 + 16 * u + (lane >> 4);
        int least = INT32_MAX, most = -1;
        bool rest = false;   // padding, or past the end
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool here = (t * kKeys + i * 16 + (lane & 15) < n) & (d[u][i] >= 0);
          least = here ? min(least, d[u][i]) : least;
          most = here ? max(most, d[u][i]) : most;
          rest |= !here;
        }
        least = least16(least);
        most = most16(most);
        const int sh = lane & 48;
        rest = (__ballot(rest) >> sh & 0xFFFF) != 0;
        const bool some = (hi >= 0) & (most >= 0) & ((t * kKeys < prefix) | ((least <= hi) & (most >= lo)));
        const bool all = one & !rest & (((t + 1) * kKeys <= prefix) | ((least == lo) & (most == lo)));
        const uint64_t ss = __ballot(some) >> sh & 15, aa = __ballot(all) >> sh & 15;
        if ((lane & 15) == 0 && t < tiles) kinds[t] = (unsigned char)(ss | (aa & ss) << 4);
      }
      if (t0 + 64 < tiles) ask(t0 + 64);
    }
    __syncthreads();
  }

  TileLoader<DH, kKeys, 4, false> key_loader;
  TileLoader<DH, kKeys, 4, true> value_loader;
  key_loader.begin(wave, lane);
  value_loader.begin(wave, lane);
  auto fetch = [&](int t, char* buf) {
    const size_t at = (size_t)t * kKeys * ldb;
    const int last = n - 1 - t * kKeys;
    key_loader.load(kbase + at, ldb, last, buf);
    value_loader.load(vbase + at, ldb, last, buf + KB);
    if (BIAS && pos && wave == 0)
      __builtin_amdgcn_global_load_lds(OTAS_GLOBAL(pos + t * kKeys + min(lane, last)), OTAS_LDS(buf + 2 * KB + value_slack<DH>()), 4, 0, 0);
    if (docs && wave == 1)
      __builtin_amdgcn_global_load_lds(OTAS_GLOBAL(docs + t * kKeys + min(lane, last)), OTAS_LDS(buf + 2 * KB + value_slack<DH>() + 256), 4, 0, 0);
  };

  const Score2 score = Score2::of(sc, BIAS ? sc.slopes[h] : 0.f, BIAS ? (pos ? pos[row] : row) : 0);
  // A key below `limit` is seen (with documents: if it is a prefix key or of the row's document).
  const int limit = my_doc < 0 ? 0 : max(mk.causal ? row + 1 : n, prefix);
  const int own_prefix = my_doc < 0 ? 0 : prefix;
  // Of the wave: below `sure` every row sees every key, from `none` on no row sees any.
  const int sure = mk.causal ? max(min(wrow0 + 1, n), prefix) : n, none = mk.causal ? max(min(wrow0 + 32, n), prefix) : n;

  // Of a tile that some row of the workgroup does not see all of, the values that are not finite are taken out and come back
  // at the end, to the rows that see them.
  const int wg_sure = mk.causal ? max(row0 + 1, prefix) : n;
  auto kind_of = [&](int t) { return docs ? __builtin_amdgcn_readfirstlane((int)kinds[t]) : 0xFF; };
  auto partly = [&](int t, int kind) { return (t + 1) * kKeys > wg_sure || (kind & ~(kind >> 4) & 15) != 0; };
  bool met = false;   // whether this wave took out a value that some row sees

  int t = docs ? next_tile(kinds, 0, tiles, lane) : 0;
  if (t < tiles) fetch(t, lds);
  if (!docs) w.begin(first + (size_t)row * ld + (size_t)h * DH, fk, sc.scale < 0.f);
  int side = 0;
  while (t < tiles) {
    const int next = docs ? next_tile(kinds, t + 1, tiles, lane) : t + 1;
    wait_all();   // this wave's part of tile t is there
    char* buf = lds + (side ? BUF : 0);
    const int kb = t * kKeys, kind = kind_of(t);
    if (partly(t, kind)) met |= value_loader.make_finite(buf + KB, lane, [&](int r) { return kb + r < end && (!docs || docs[kb + r] >= 0); });
    wait_lds_barrier();   // all of it, and nobody reads the other buffer any more
    if (next < tiles) fetch(next, lds + (side ? 0 : BUF));
    const bool one = (kind >> (4 + wave) & 1) != 0;
    if (active && kb < none && (kind >> wave & 1)) {   // wave-uniform
      __builtin_amdgcn_s_setprio(0);
      floatx16 s[2];
      tile_products<DH, 2>(s, w, buf, 0, fr, fk);
      short8_t v[WaveRows<DH>::DT];
      first_values<DH>(v, buf + KB, 0, lane);
      __builtin_amdgcn_s_setprio(1);   // a wave that needs the vector ALU, the busier of the two, goes before one at its products (358 -> 340 us, 8192 capped rows)
      const bool whole = kb + kKeys <= sure && one;
      bool done = false;
      if (CAP && !BIAS && whole) done = tile_weights_capped<DH, 2>(w, s, cap);
      if (CAP && !done) tile_capped<CAP, 2>(s, score, cap);
      if (BIAS) {
        const int* kp = reinterpret_cast<const int*>(buf + 2 * KB + value_slack<DH>());
        const float near = (float)(score.position - kb - 4 * fk);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            float d[4];
            if (pos) {
              const int4 p = read_four(kp, b * 8 + 2 * g + fk);
              d[0] = (float)(score.position - p.x); d[1] = (float)(score.position - p.y);
              d[2] = (float)(score.position - p.z); d[3] = (float)(score.position - p.w);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) d[e] = near - (float)(32 * b + 8 * g + e);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][4 * g + e] = fmaf(-score.slope2, fabsf(d[e]), CAP ? s[b][4 * g + e] : s[b][4 * g + e] * score.scale2);
          }
      }
      if (!whole && one) {   // of documents, all keys are the rows' (or prefix keys): as without
        const int left = limit - kb - 4 * fk;   // keys of this half that the row sees, from the tile's first on
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[b][e] = 32 * b + 8 * (e >> 2) + (e & 3) < left ? s[b][e] : -INFINITY;
      } else if (!whole) {
        const int* kd = reinterpret_cast<const int*>(buf + 2 * KB + value_slack<DH>() + 256);
        const int left = limit - kb - 4 * fk, early = own_prefix - kb - 4 * fk;
        // Past the prefix (wave-uniform) the row's document and its limit decide, which is 0 for padding (2 x 4000 with five documents, width 64:
        // 57 -> 54 us).  At 128 the second form's registers do not fit, and it gave nothing there.
        const bool beyond = DH < 128 && kb >= prefix;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int4 d = read_four(kd, b * 8 + 2 * g + fk);
            const int dd[4] = {d.x, d.y, d.z, d.w};
            if (beyond) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const bool see = (32 * b + 8 * g + e < left) & (dd[e] == my_doc);
                s[b][4 * g + e] = see ? s[b][4 * g + e] : -INFINITY;
              }
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int j = 32 * b + 8 * g + e;
                const bool see = (j < left) & (dd[e] >= 0) & ((j < early) | (dd[e] == my_doc));
                s[b][4 * g + e] = see ? s[b][4 * g + e] : -INFINITY;
              }
            }
          }
      }
      if (!done) tile_weights<DH, 2>(w, s, CAP || BIAS ? 1.f : score.scale2);
      __builtin_amdgcn_s_setprio(0);
      tile_sums<DH, 2>(w, s, v, buf + KB, 0, lane);
    }
    t = next;
    side ^= 1;
  }
  if (any_wave(met, reinterpret_cast<int*>(lds + 2 * BUF), wave, lane)) {   // workgroup-uniform
    for (int j = 0; j < end; ++j) {
      if (!partly(j / kKeys, kind_of(j / kKeys))) continue;
      const int d = docs ? docs[j] : 0;
      const bool see = (j < limit) & (d >= 0) & ((j < own_prefix) | (d == my_doc));
      const bf16_t* v = reinterpret_cast<const bf16_t*>(vbase + (size_t)j * ldb);
#pragma unroll
      for (int c = 0; c < WaveRows<DH>::DT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if (c * 32 + g * 8 < DH) add_not_finite(w.o[c], g, v + c * 32 + g * 8 + fk * 4, see);
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

hipError_t launch_attention_masked_bf16(const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int max_n, int H,
                                        int KV, int dh, const ScoreArgs& sc, const MaskArgs& mk, void* o, hipStream_t s) {
  const int xblks = (max_n + kRows - 1) / kRows;
  const int64_t wgs = (int64_t)xblks * H * B;
  if (wgs > kMostGroups) return kTooManyGroups;
  const PlanAny p = plan_any(plan, count, d_plan);
  const int by_xcd = (int64_t)B * H % 8 == 0;
  auto run = [&](auto width, auto cap, auto bias) {
    constexpr int DH = decltype(width)::value;
    auto kern = attention_masked_bf16_kernel<DH, decltype(cap)::value, decltype(bias)::value>;
    const size_t lds = masked_lds<DH>(max_n, mk.documents != nullptr);
    const hipError_t e = set_max_dynamic_lds((const void*)kern, (int)masked_lds<DH>(1 << 20, true));
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)wgs), dim3(256), lds, s>>>((const bf16_t*)qkv, p, B, H, KV, xblks, by_xcd, sc, CapArgs::of(sc), mk, (bf16_t*)o);
    return hipGetLastError();
  };
  auto pick = [&](auto width) {
    auto with_bias = [&](auto cap) { return sc.slopes ? run(width, cap, std::true_type{}) : run(width, cap, std::false_type{}); };
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
