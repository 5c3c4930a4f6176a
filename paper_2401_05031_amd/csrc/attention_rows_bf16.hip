// Attention through a window in bf16 for many rows: otas_attention_window, and otas_attention_recent and otas_attention_cache4 where a query
// has more than 32 rows a key head.  Four waves of 32 rows each walk the keys that any of them sees in tiles of 64; while one LDS buffer
// is worked on, the other is filled; one barrier a tile, as in attention_masked_bf16.hip.
//   Rows are tokens x heads that share a key head, one after the other: what rows see moves with their tokens, and a workgroup
// walks all that any of its rows sees.  With a window w, 128 rows of one head walk w + 128 keys, of which a wave sees w + 32; of eight heads they
// walk w + 16 and a wave sees w + 4.
//   Keys of the model's dtype travel from global memory straight into LDS.  Keys in 4 bits are asked for a tile ahead, 16 bytes of a
// group a thread, and written to LDS as bf16, which holds them exactly, beneath the products of the tile before.
//   Products, exponentials and a start and end of 10 us or more that all workgroups of a round have at once add up: 8192 rows, 16 heads on 2 of 128, window
// 1024: 88 us, 735 TFLOP/s of 64.7 GFLOP (matrix cores busy for 39 % of it, the vector ALU for 46 %); 12 x 600 .. 1500 rows, 12 heads on 4 of 64, window 300, capped:
// 42 us; 4 x 256 rows over 2291 .. 4000 entries in 4 bits, 16 heads on 2 of 128, capped: 39 us and the join of its four parts 10.  (After some hundred launches in
// a row; the first twenty take 97, 46 and 42.)
#include "attention_tiles.h"
#include "cache4.h"

namespace otas {

namespace {

constexpr int kKeys = 1 << kRowsShift;
// Bits 0 .. n - 1 of a word; all ones where bit i is one.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : 0xFFFFFFFFu >> (32 - min(n, 32)); }
__device__ __forceinline__ uint32_t bit_everywhere(uint32_t word, int i) { return (uint32_t)((int32_t)(word << (31 - i)) >> 31); }

}  // namespace

// A tile's groups of 32 elements in 4 bits, one of keys and one of values a thread.
template <int DH> struct GroupLoader {
  typedef TileRows<DH> R;
  static constexpr int GROUPS = (DH + 31) / 32, TOTAL = kKeys * GROUPS;   // at most 256
  static constexpr int LAST = DH % 32 / 8;                                // words of the last group, 0: all four
  static_assert(TOTAL <= 256, "a group a thread");
  const char *k, *v, *ks, *vs;   // the thread's
  uint32_t kw[4], vw[4], kb, vb;
  int64_t capacity;
  int row, g;
  bool mine;
  __device__ __forceinline__ void begin(const char* k_, const char* v_, const char* ks_, const char* vs_, int64_t capacity_, int tid) {
    capacity = capacity_;
    mine = tid < TOTAL;
    row = min(tid, TOTAL - 1) / GROUPS;
    g = min(tid, TOTAL - 1) - row * GROUPS;
    k = k_ + row * (DH / 2) + g * 16;
    v = v_ + row * (DH / 2) + g * 16;
    ks = ks_ + g * capacity + row;
    vs = vs_ + g * capacity + row;
  }
  __device__ __forceinline__ void load(int tile) {   // the capacity is a multiple of 32: where the tile runs past it, its upper half is its lower
    const int64_t at = (int64_t)tile * kKeys - ((int64_t)tile * kKeys + row < capacity ? 0 : 32);
    auto words = [&](const char* p, uint32_t (&w)[4]) {
      if (LAST == 0) {
        __builtin_memcpy(w, p, 16);
      } else {
        __builtin_memcpy(w, p, 4 * LAST);
        w[2] = w[3] = 0;
        if (g < GROUPS - 1) __builtin_memcpy(w + LAST, p + 4 * LAST, 16 - 4 * LAST);
      }
    };
    words(k + at * (DH / 2), kw);
    words(v + at * (DH / 2), vw);
    kb = *reinterpret_cast<const uint8_t*>(ks + at);
    vb = *reinterpret_cast<const uint8_t*>(vs + at);
  }
  // What was loaded made ready for LDS: keys from `end` of the tile on, whose scales may be anything, have no values, and neither have groups
  // that are no numbers.  Whether there were any of the latter before `end`.
  __device__ __forceinline__ bool prepare(int end) {
    const bool here = row < end, odd = here && vb == kNoNumber;
    if (!here || odd) {
      vb = 0;
#pragma unroll
      for (int c = 0; c < 4; ++c) vw[c] = 0;
    }
    if (TURNS) {
      auto swap_if = [](bool b, uint32_t& x, uint32_t& y) {
        const uint32_t t = b ? y : x;
        y = b ? x : y;
        x = t;
      };
      swap_if(turn() & 1, vw[0], vw[1]);
      swap_if(turn() & 1, vw[2], vw[3]);
      swap_if(turn() & 2, vw[0], vw[2]);
      swap_if(turn() & 2, vw[1], vw[3]);
    }
    return mine && odd;
  }
  // Values' pieces of four rows (eight of width 64) would lie on the same banks: every thread begins with another of its four.
  static constexpr bool TURNS = DH % 64 == 0;
  __device__ __forceinline__ int turn() const { return TURNS ? (DH == 128 ? row : row >> 1) & 3 : 0; }
  static constexpr int PIECES = 8;
  // Piece c of these: eight keys' elements (c < 4), or values'.  A key's group that is no number has elements that are none.
  __device__ __forceinline__ void store(int c, char* __restrict__ keys, char* __restrict__ values) const {
    const int p = g * 4 + (c < 4 ? c : (c & 3) ^ turn());
    if (!mine || (LAST != 0 && (c & 3) >= LAST && g == GROUPS - 1)) return;
    const uint32_t word = c < 4 ? kw[c & 3] : vw[c & 3], all = c < 4 && kb == kNoNumber ? 0x7FC07FC0u : 0u;
    const float f = scale4(c < 4 ? kb : vb);
    const uint4 u = {pair4_bf16<0>(word, f) | all, pair4_bf16<1>(word, f) | all, pair4_bf16<2>(word, f) | all, pair4_bf16<3>(word, f) | all};
    *reinterpret_cast<uint4*>((c < 4 ? keys : values) + row * R::ROW_BYTES + (c < 4 ? R::key_piece(row, p) : R::value_piece(row, p)) * 16) = u;
  }
  __device__ __forceinline__ void store_all(char* __restrict__ keys, char* __restrict__ values) const {
#pragma unroll
    for (int c = 0; c < PIECES; ++c) store(c, keys, values);
  }
};

template <int DH> constexpr size_t rows_buffer() { return 2 * TileRows<DH>::bytes(kKeys) + value_slack<DH>(); }
template <int DH> constexpr size_t rows_lds() { return 2 * rows_buffer<DH>() + 16; }

template <int DH, bool FOUR, int CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void attention_rows_bf16_kernel(PlanAny plan_, Cache4Ref c, const bf16_t* __restrict__ qkv, int H, int B, WindowShape shape,
                                                                     ScoreArgs sc, CapArgs cap, RecentBuffers out, bf16_t* __restrict__ o) {
  typedef TileRows<DH> R;
  constexpr size_t KB = R::bytes(kKeys), BUF = rows_buffer<DH>();   // keys | values | slack
  // Blocks of 32 keys at a time.  One by one, halves of a tile that no row of the wave sees are left out; two at once cover each other's latencies.
  // Width 64 (4 x 1500 rows, window 300 / 2 x 6000, 1000 / 8192, all), one 27 / 87 / 219 us, two 29 / 89 / 216; 80: 42 / 115 / 264 and 43 / 115 / 238;
  // 128: 49 / 149 / 337 and 50 / 140 / 312.  In 4 bits at width 64 (4 x 2000 rows over 4096 entries, window 1024) 121 and 144 us, with which three waves
  // a SIMD have the registers.
  constexpr int ROWS = kManyRows, NB = DH == 64 ? 1 : 2;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const PlanFirst plan = PlanFirst::of(plan_);
  const WorkPlace at = shape.work(plan, (int)blockIdx.x, B, c.KV);
  const int kh = at.unit % c.KV, q = at.unit / c.KV, G = H / c.KV, group0 = at.group * ROWS;
  const bool packed = !FOUR && c.k == nullptr;
  const int base = plan.at(q), n = plan.at(q + 1) - base, rows = n * G;
  if (group0 >= rows) return;
  const int len = packed ? n : plan.at(2 * B + 1 + q), place0 = len - n;
  const WindowTiles tiles = shape.tiles(at.group, n, G, len);
  // a division is a tenth of a microsecond before the first load: none without parts
  const int each = shape.parts == 1 ? tiles.count : shape.each_of(tiles), begin = at.part * each, end = min(tiles.count, begin + each);
  if (begin >= end) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), fr = lane & 31, fk = lane >> 5;
  const int wrow0 = group0 + wave * 32, row = min(wrow0 + fr, rows - 1), token = row / G, head = kh * G + row % G, place = place0 + token;
  const bool active = wrow0 < rows;
  const size_t ld = (size_t)(H + 2 * c.KV) * DH;
  const bf16_t* first = qkv + (size_t)base * ld;
  const int64_t slot_head = packed ? 0 : (int64_t)plan.at(B + 1 + q) * c.KV + kh;
  const char *kbase, *vbase;
  if (packed) {
    kbase = reinterpret_cast<const char*>(first + (size_t)(H + kh) * DH);
    vbase = reinterpret_cast<const char*>(first + (size_t)(H + c.KV + kh) * DH);
  } else {
    const int64_t bytes = slot_head * c.capacity * (FOUR ? DH / 2 : 2 * DH);
    kbase = c.k + bytes;
    vbase = c.v + bytes;
  }
  const uint32_t ldb = (uint32_t)((packed ? ld : DH) * sizeof(bf16_t));
  // places of the workgroup's rows and of the wave's
  const int p0 = place0 + group0 / G, p1 = place0 + (min(group0 + ROWS, rows) - 1) / G;
  const int w0 = place0 + min(wrow0, rows - 1) / G, w1 = place0 + (min(wrow0 + 32, rows) - 1) / G;
  const int window = min(shape.window, 1 << 21), sinks = shape.sinks;   // twice the longest query: differences stay within 32 bits

  TileLoader<DH, kKeys, 4, false> key_loader;
  TileLoader<DH, kKeys, 4, true> value_loader;
  GroupLoader<DH> groups;
  if constexpr (FOUR) {
    const int64_t scales = slot_head * c.groups * c.capacity;
    groups.begin(kbase, vbase, c.ks + scales, c.vs + scales, c.capacity, tid);
  } else {
    key_loader.begin(wave, lane);
    value_loader.begin(wave, lane);
  }
  auto fetch = [&](int t, char* buf) {
    const size_t from = (size_t)t * kKeys * ldb;
    key_loader.load(kbase + from, ldb, len - 1 - t * kKeys, buf);
    value_loader.load(vbase + from, ldb, len - 1 - t * kKeys, buf + KB);
  };
  const Score2 score = Score2::of(sc, BIAS ? sc.slopes[head] : 0.f, place);
  // Whether rows at places a .. b all see all of the `keys` keys from kb on, and whether any of them sees any.
  auto all_see = [&](int a, int b, int kb, int keys) { return kb + keys - 1 <= a && (kb > b - window || kb + keys <= sinks); };
  auto some_see = [&](int a, int b, int kb, int keys) { return kb <= b && (kb + keys - 1 > a - window || kb < sinks); };
  bool met = false;   // whether this thread took out a value that is not finite

  if constexpr (FOUR) {
    groups.load(tiles.tile(begin));
    met |= groups.prepare(p1 + 1 - tiles.tile(begin) * kKeys);
    groups.store_all(lds, lds + KB);
    if (begin + 1 < end) groups.load(tiles.tile(begin + 1));
  } else {
    fetch(tiles.tile(begin), lds);
  }
  WaveRows<DH> w;
  w.begin(first + (size_t)token * ld + (size_t)head * DH, fk, sc.scale < 0.f);
  for (int i = begin; i < end; ++i) {
    char* buf = lds + ((i - begin) & 1 ? BUF : 0);
    char* other = lds + ((i - begin) & 1 ? 0 : BUF);
    const int kb = tiles.tile(i) * kKeys;
    if constexpr (FOUR) {
      wait_lds_barrier();   // the tile is there, and nobody reads the other buffer any more
      if (i + 1 < end) met |= groups.prepare(p1 + 1 - tiles.tile(i + 1) * kKeys);
    } else {
      wait_all();   // this wave's part of the tile is there
      // Of a tile that some row does not see all of, values that are not finite are taken out and come back at the end, to
      // the rows that see them.
      if (!all_see(p0, p1, kb, kKeys)) met |= value_loader.make_finite(buf + KB, lane, [&](int r) { return kb + r <= p1; });
      wait_lds_barrier();   // all of it, and nobody reads the other buffer any more
      if (i + 1 < end) fetch(tiles.tile(i + 1), other);
    }
    bool stored = !FOUR;   // the next tile in 4 bits; behind the last one what is there once more, where nobody reads it
#pragma unroll 1
    for (int b0 = 0; b0 < 2; b0 += NB) {
      const int from = kb + 32 * b0;
      if (!active || !some_see(w0, w1, from, 32 * NB)) continue;   // wave-uniform
      const char* keys = buf + b0 * 32 * R::ROW_BYTES;
      __builtin_amdgcn_s_setprio(0);
      floatx16 s[NB];
      if constexpr (FOUR && NB == 2) {
        tile_products<DH, NB>(s, w, keys, 0, fr, fk, [&](int j) {
#pragma unroll
          for (int c = 0; c < groups.PIECES; ++c)
            if (c * (WaveRows<DH>::KS * NB) / groups.PIECES == j) groups.store(c, other, other + KB);
        });
        stored = true;
        if (i + 2 < end) groups.load(tiles.tile(i + 2));
      } else {
        tile_products<DH, NB>(s, w, keys, 0, fr, fk);
      }
      short8_t v[WaveRows<DH>::DT];
      first_values<DH>(v, keys + KB, 0, lane);
      __builtin_amdgcn_s_setprio(1);   // a wave that needs the vector ALU goes before one at its products, as in attention_masked_bf16.hip
      const bool whole = all_see(w0, w1, from, 32 * NB);
      bool done = false;
      if (CAP && !BIAS && whole) done = tile_weights_capped<DH, NB>(w, s, cap);
      const int behind = place - from - 4 * fk;   // the row's distance from the lane's first key
      // Which keys the row sees, a bit each: two operations an element to take the others out, where comparisons are three and more (8192 rows, window
      // 1024, width 128, first launches: 99.5 -> 97.9 us).
      uint32_t seen[NB];
      if (!whole) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const int d = behind - 32 * b;
          seen[b] = bits_below(d + 1) & (~bits_below(d + 1 - window) | bits_below(sinks - from - 4 * fk - 32 * b));
        }
      }
      if (CAP && !done) {
        // The cap's form hangs on the wave's largest product: not on one with a key that no row of it sees, or with what lies behind a slot's entries.
        // (1.2 % of the capped cases' time.)
        if (!whole) {
#pragma unroll
          for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[b][e] = __uint_as_float(__float_as_uint(s[b][e]) & bit_everywhere(seen[b], 8 * (e >> 2) + (e & 3)));
            if (NB > 1) keep_here(seen[b]);    // or each bit's word stays in a register, which there are not
          }
        }
        tile_capped<CAP, NB>(s, score, cap);
      }
      if (BIAS) {
        const float near = (float)behind;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float d = near - (float)(32 * b + 8 * (e >> 2) + (e & 3));
            s[b][e] = fmaf(-score.slope2, fabsf(d), CAP ? s[b][e] : s[b][e] * score.scale2);
          }
      }
      if (!whole) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t mine = bit_everywhere(seen[b], 8 * (e >> 2) + (e & 3));
            s[b][e] = __uint_as_float((__float_as_uint(s[b][e]) & mine) | (__float_as_uint(-INFINITY) & ~mine));
          }
      }
      if (!done) tile_weights<DH, NB>(w, s, CAP || BIAS ? 1.f : score.scale2);
      __builtin_amdgcn_s_setprio(0);
      tile_sums<DH, NB>(w, s, v, keys + KB, 0, lane);
    }
    if (!stored) {
      groups.store_all(other, other + KB);
      if (i + 2 < end) groups.load(tiles.tile(i + 2));
    }
  }
  if (any_wave(met, reinterpret_cast<int*>(lds + 2 * BUF), wave, lane)) {   // workgroup-uniform
    for (int i = begin; i < end; ++i) {
      const int kb = tiles.tile(i) * kKeys;
      if (!FOUR && all_see(p0, p1, kb, kKeys)) continue;
      for (int j = kb; j < min(kb + kKeys, p1 + 1); ++j) {
        const bool see = j <= place && (place - j < window || j < sinks);
#pragma unroll
        for (int t = 0; t < WaveRows<DH>::DT; ++t) {
          if constexpr (FOUR) {
            const bool odd = *reinterpret_cast<const uint8_t*>(c.vs + (slot_head * c.groups + t) * c.capacity + j) == kNoNumber;
#pragma unroll
            for (int e = 0; e < 16; ++e) w.o[t][e] = odd && see ? __uint_as_float(0x7FC00000u) : w.o[t][e];
          } else {
            const bf16_t* v = reinterpret_cast<const bf16_t*>(vbase + (size_t)j * ldb);
#pragma unroll
            for (int g = 0; g < 4; ++g)
              if (t * 32 + g * 8 < DH) add_not_finite(w.o[t], g, v + t * 32 + g * 8 + fk * 4, see);
          }
        }
      }
    }
  }
  const float l = xor32_sum(w.l);
  if (!active) return;
  const bool mine = wrow0 + fr < rows;   // both lanes of a row
  const int64_t to = (int64_t)(base + token) * H + head;
  const bool only = shape.parts == 1 || shape.parts_of(tiles) == 1;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int t = 0; t < WaveRows<DH>::DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; g += 2)
      if (t * 32 + g * 8 < DH) {
        if (only) {   // the lane's halves of two eights change places with the other half's: whole eights are stored
          uint32_t x[2][2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int at = 4 * (g + i) + 2 * e;
              const bf16x2 v = {(bf16_t)(l == 0.f ? 0.f : w.o[t][at] * inv), (bf16_t)(l == 0.f ? 0.f : w.o[t][at + 1] * inv)};
              __builtin_memcpy(&x[i][e], &v, 4);
            }
          const auto lo = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false), hi = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
          if (mine) *reinterpret_cast<uint4*>(o + to * DH + t * 32 + (g + fk) * 8) = uint4{lo[0], hi[0], lo[1], hi[1]};
        } else if (mine) {
#pragma unroll
          for (int i = g; i < g + 2; ++i)
            *reinterpret_cast<floatx4*>(out.sums + ((int64_t)at.part * out.TH + to) * DH + t * 32 + i * 8 + fk * 4) =
                floatx4{w.o[t][4 * i], w.o[t][4 * i + 1], w.o[t][4 * i + 2], w.o[t][4 * i + 3]};
        }
      }
  if (!only && mine && fk == 0) {
    out.tops[2 * (at.part * out.TH + to)] = w.m;
    out.tops[2 * (at.part * out.TH + to) + 1] = l;
  }
}

hipError_t launch_attention_rows_bf16(bool four, const Cache4Ref& c, const void* qkv, int H, const int32_t* plan, size_t count, const int32_t* d_plan, int B,
                                      const ScoreArgs& sc, const WindowShape& shape, const RecentBuffers& buf, void* o, hipStream_t s) {
  const int64_t wgs = shape.workgroups(plan, B, c.KV);
  if (wgs > kMostGroups) return kTooManyGroups;
  const PlanAny p = plan_any(plan, count, d_plan);
  auto run = [&](auto width, auto four_, auto cap, auto bias) {
    constexpr int DH = decltype(width)::value;
    auto kern = attention_rows_bf16_kernel<DH, decltype(four_)::value, decltype(cap)::value, decltype(bias)::value>;
    const hipError_t e = set_max_dynamic_lds((const void*)kern, (int)rows_lds<DH>());
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)wgs), dim3(256), rows_lds<DH>(), s>>>(p, c, (const bf16_t*)qkv, H, B, shape, sc, CapArgs::of(sc), buf, (bf16_t*)o);
    return hipGetLastError();
  };
  auto pick = [&](auto width, auto four_) {
    auto with_bias = [&](auto cap) { return sc.slopes ? run(width, four_, cap, std::true_type{}) : run(width, four_, cap, std::false_type{}); };
    switch (Score2::cap_form(sc.cap)) {
      case 0: return with_bias(std::integral_constant<int, 0>{});
      case 1: return with_bias(std::integral_constant<int, 1>{});
    }
    return with_bias(std::integral_constant<int, 2>{});
  };
  auto either = [&](auto width) { return four ? pick(width, std::true_type{}) : pick(width, std::false_type{}); };
  switch (c.dh) {
    case 64: return either(std::integral_constant<int, 64>{});
    case 80: return either(std::integral_constant<int, 80>{});
    case 96: return either(std::integral_constant<int, 96>{});
    case 128: return either(std::integral_constant<int, 128>{});
  }
  return hipErrorInvalidValue;
}

}  // namespace otas
