// otas_attention_tree in bf16.  A workgroup of four waves has up to 32 RW rows (nodes x heads that share a key head) and a chunk
// of the query's cache, whose tiles travel from global memory into the one LDS buffer while the other is worked on.  RW of the
// waves have 32 rows each, and 4 / RW share those rows, every one with its own keys of a tile, to be joined at the end: the usual
// single token has few rows, and then all four waves work on keys.  What bounds few rows is the cache's own bytes; what bounds
// many is the matrix cores and the exponentials, as in otas_attention_masked.
//   32 queries of one token over 5700 .. 8192 entries (8 key heads of 128, with weights added up): 198 us and 8 for the join, 919 MB at
// 4.5 TB/s.  8 x 48 nodes over 2000 .. 4000: 31 and 7.5 us (576 workgroups of up to 8 tiles, the first 6 us after the launch).  One token over
// 1537 entries: 8.8 and 3.8 us, a chain of launch, plan, queries, one tile, the waves' join.
#include "attention_tiles.h"
#include "attention_tree_join.h"

namespace otas {

template <int DH, int RW> struct TreeTile {
  static constexpr int KG = 4 / RW, NB = RW == 4 ? 2 : 1, KEYS = 32 * KG * NB;   // waves that share rows, blocks of 32 keys a wave and tile
  static constexpr size_t KB = TileRows<DH>::bytes(KEYS), BUF = 2 * KB + value_slack<DH>() + 512;   // keys | values | slack | positions
  static constexpr int LDO = DH + 4;
  static constexpr size_t JOIN = KG > 1 ? 4 * (256 + 32 * LDO * 4) : 0;   // [4][2][32] tops and sums | [4][32][LDO]
  static constexpr size_t LDS = (2 * BUF > JOIN ? 2 * BUF : JOIN) + 16;
};

// logits (of the cached entries, where their weights are to be added up and rows are few): [T H][stride], 4 bytes a row and
// key written and read once, where forming them again would read the key's 2 d_h bytes once more.
template <int DH, int RW, int CAP, bool BIAS>
__global__ __launch_bounds__(256, RW == 1 && DH > 64 ? 1 : 2) void attention_tree_bf16_kernel(CacheRef c, const bf16_t* __restrict__ qkv, int H,
                                                                                              const int32_t* __restrict__ positions, PlanAny plan, int B,
                                                                                              bool has_parents, TreeShape shape, ScoreArgs sc, CapArgs cap,
                                                                                              TreeBuffers out, bf16_t* __restrict__ o) {
  typedef TreeTile<DH, RW> S;
  typedef TileRows<DH> R;
  constexpr int KG = S::KG, NB = S::NB, KEYS = S::KEYS;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  // The row groups of a chunk run side by side on one XCD, whose L2 then has the chunk once.
  const int units = B * c.KV * shape.parts;
  int id = (int)blockIdx.x;
  const int eights = units & ~7, span = 8 * shape.groups;
  int group, unit;
  if (id < eights * shape.groups) {
    group = id % span / 8;
    unit = id / span * 8 + id % 8;
  } else {
    id -= eights * shape.groups;
    group = id / (units - eights);
    unit = eights + id % (units - eights);
  }
  const int part = unit % shape.parts, kh = unit / shape.parts % c.KV, q = unit / shape.parts / c.KV, G = H / c.KV;
  const int base = plan.at(q), n = plan.at(q + 1) - base, len = plan.at(2 * B + 1 + q), rows = n * G, group0 = group * 32 * RW;
  const int64_t slot = plan.at(B + 1 + q);
  // The last part may be the nodes' of queries of several chunks.
  const int chunks = shape.chunks(len);
  const bool apart = shape.apart && shape.parts > 1 && part == shape.parts - 1, nodes = apart || (part == 0 && (chunks <= 1 || !shape.apart));
  if (group0 >= rows || (apart ? chunks <= 1 : part > 0 && part >= chunks)) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), fr = lane & 31, fk = lane >> 5;
  const int rw = wave % RW, kg = wave / RW, row0 = group0 + rw * 32;
  const bool active = row0 < rows;
  const int row = min(row0 + fr, rows - 1), node = row / G, head = kh * G + row % G;
  const size_t ld = (size_t)(H + 2 * c.KV) * DH;
  const bf16_t* first = qkv + (size_t)base * ld;
  const int begin = apart ? 0 : part * shape.chunk, end = apart ? 0 : min(len, begin + shape.chunk);
  const char* cached_k = reinterpret_cast<const char*>((const bf16_t*)c.k + ((slot * c.KV + kh) * c.capacity + begin) * DH);
  const char* cached_v = reinterpret_cast<const char*>((const bf16_t*)c.v + ((slot * c.KV + kh) * c.capacity + begin) * DH);
  const char* draft_k = reinterpret_cast<const char*>(first + (size_t)(H + kh) * DH);
  const char* draft_v = reinterpret_cast<const char*>(first + (size_t)(H + c.KV + kh) * DH);
  const int32_t* cached_pos = c.positions + slot * c.capacity + begin;
  const int cached_tiles = (max(0, end - begin) + KEYS - 1) / KEYS, steps = cached_tiles + (nodes ? 1 : 0);   // the nodes themselves last

  TileLoader<DH, KEYS, 4, false> key_loader;
  TileLoader<DH, KEYS, 4, true> value_loader;
  key_loader.begin(wave, lane);
  value_loader.begin(wave, lane);
  auto fetch = [&](int i, char* buf) {
    const bool cached = i < cached_tiles;   // wave-uniform
    const int last = cached ? end - begin - 1 - i * KEYS : n - 1;
    const size_t at = cached ? (size_t)i * KEYS * (DH * sizeof(bf16_t)) : 0;
    const uint32_t stride = cached ? (uint32_t)(DH * sizeof(bf16_t)) : (uint32_t)(ld * sizeof(bf16_t));
    key_loader.load((cached ? cached_k : draft_k) + at, stride, last, buf);
    value_loader.load((cached ? cached_v : draft_v) + at, stride, last, buf + S::KB);
    if (BIAS && wave < KEYS / 64) {
      const int32_t* p = cached ? cached_pos + i * KEYS : positions + base;
      __builtin_amdgcn_global_load_lds(OTAS_GLOBAL(p + min(wave * 64 + lane, last)), OTAS_LDS(buf + 2 * S::KB + value_slack<DH>() + wave * 256), 4, 0, 0);
    }
  };
  const Score2 score = Score2::of(sc, BIAS ? sc.slopes[head] : 0.f, BIAS ? positions[base + node] : 0);
  uint64_t line = 0;
  if (nodes) line = lane_value(tree_lines(plan, 3 * B + 1, base, n, has_parents, lane), node);
  bool met = false;   // whether this wave took out a sibling's value

  fetch(0, lds);
  WaveRows<DH> w;
  w.begin(first + (size_t)node * ld + (size_t)head * DH, fk, sc.scale < 0.f);
  for (int i = 0; i < steps; ++i) {
    wait_all();   // this wave's part of tile i is there
    char* buf = lds + (i & 1 ? S::BUF : 0);
    const bool cached = i < cached_tiles;
    const int valid = cached ? min(KEYS, end - begin - i * KEYS) : n;
    if (!cached) {   // of siblings, values that are not finite are taken out and come back at the end to the nodes that see them
      met |= value_loader.make_finite(buf + S::KB, lane, [&](int r) { return r < n; });
    } else if (valid < KEYS) {   // rows past the end repeat the last one, which may be infinite
      value_loader.zero_rows(buf + S::KB, lane, valid);
    }
    wait_lds_barrier();   // all of it, and nobody reads the other buffer any more
    if (i + 1 < steps) fetch(i + 1, lds + (i & 1 ? 0 : S::BUF));
    const int k0 = kg * 32 * NB;
    if (active && k0 < valid) {   // wave-uniform
      floatx16 s[NB];
      tile_products<DH, NB>(s, w, buf, kg * NB, fr, fk);
      short8_t v[WaveRows<DH>::DT];
      first_values<DH>(v, buf + S::KB, 2 * kg * NB, lane);
      const bool whole = cached && k0 + 32 * NB <= valid;
      bool done = false;
      if (CAP && !BIAS && whole && !(RW == 1 && out.logits)) done = tile_weights_capped<DH, NB>(w, s, cap);
      if (CAP && !done) tile_capped<CAP, NB>(s, score, cap);
      if (BIAS) {
        const int* kp = reinterpret_cast<const int*>(buf + 2 * S::KB + value_slack<DH>()) + k0;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int4 p = read_four(kp, b * 8 + 2 * g + fk);
            const float d[4] = {(float)(score.position - p.x), (float)(score.position - p.y), (float)(score.position - p.z), (float)(score.position - p.w)};
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][4 * g + e] = fmaf(-score.slope2, fabsf(d[e]), CAP ? s[b][4 * g + e] : s[b][4 * g + e] * score.scale2);
          }
      }
      constexpr bool SCALED = CAP != 0 || BIAS;
      if (!whole) {
        // of this half's keys, from the wave's first on: how many are left, and which of the nodes the row sees
        const int left = valid - k0 - 4 * fk;
        const uint64_t mine = cached ? ~0ull : line >> (k0 + 4 * fk);
        const uint32_t sees[2] = {(uint32_t)mine, (uint32_t)(mine >> 32)};
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int j = 8 * (e >> 2) + (e & 3);
            const bool see = (32 * b + j < left) & (int)(sees[b] >> j & 1);
            s[b][e] = see ? s[b][e] : -INFINITY;
          }
      }
      if (RW == 1 && out.logits && cached && row0 + fr < rows) {
        float* to = out.logits + ((int64_t)(base + node) * H + head) * out.stride + begin + i * KEYS + k0 + 4 * fk;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            if (begin + i * KEYS + k0 + 32 * b + 8 * g + 4 * fk < out.stride) {   // a multiple of 4
              const float f = SCALED ? 1.f : score.scale2;
              *reinterpret_cast<floatx4*>(to + 32 * b + 8 * g) = floatx4{s[b][4 * g] * f, s[b][4 * g + 1] * f, s[b][4 * g + 2] * f, s[b][4 * g + 3] * f};
            }
      }
      if (!done) tile_weights<DH, NB>(w, s, SCALED ? 1.f : score.scale2);
      tile_sums<DH, NB>(w, s, v, buf + S::KB, 2 * kg * NB, lane);
    }
  }
  const bool not_finite = nodes && any_wave(met, reinterpret_cast<int*>(lds + S::LDS - 16), wave, lane);
  if (not_finite && kg == 0) {   // one of the waves that share rows
    for (int j = 0; j < n; ++j) {
      const bf16_t* v = reinterpret_cast<const bf16_t*>(draft_v) + (size_t)j * ld;
#pragma unroll
      for (int t = 0; t < WaveRows<DH>::DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if (t * 32 + g * 8 < DH) add_not_finite(w.o[t], g, v + t * 32 + g * 8 + fk * 4, line >> j & 1);
    }
  }

  const bool only = chunks <= 1;   // the rows' one chunk: done
  const int64_t place = apart ? chunks : part;
  auto finish = [&](int r, int d, floatx4 v, float m, float l) {   // columns d .. d + 3 of row r of the query's
    const int64_t at = (int64_t)(base + r / G) * H + kh * G + r % G;
    if (only) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (bf16_t)(l == 0.f ? 0.f : v[e] * inv);
      *reinterpret_cast<bf16x4*>(o + at * DH + d) = x;
    } else {
      *reinterpret_cast<floatx4*>(out.sums + (place * out.TH + at) * DH + d) = v;
    }
    if (d == 0) {
      if (!only) { out.tops[2 * (place * out.TH + at)] = m; out.tops[2 * (place * out.TH + at) + 1] = l; }
      else if (out.ends) { out.ends[2 * at] = m; out.ends[2 * at + 1] = l; }
    }
  };
  const float l_run = xor32_sum(w.l);
  if constexpr (KG == 1) {
    if (row0 + fr >= rows) return;
#pragma unroll
    for (int t = 0; t < WaveRows<DH>::DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = t * 32 + g * 8 + fk * 4;
        if (d < DH) finish(row0 + fr, d, floatx4{w.o[t][4 * g], w.o[t][4 * g + 1], w.o[t][4 * g + 2], w.o[t][4 * g + 3]}, w.m, l_run);
      }
  } else {
    float* ml = reinterpret_cast<float*>(lds);         // [4][2][32]
    float* osh = ml + 256;                             // [4][32][LDO]
    wait_lds_barrier();                                // all have read the flag: the buffers may be overwritten
    if (fk == 0) {
      ml[wave * 64 + fr] = w.m;
      ml[wave * 64 + 32 + fr] = l_run;
    }
    wait_lds_barrier();
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < KG; ++k) top = fmaxf(top, ml[(k * RW + rw) * 64 + fr]);
    const float f = to_top(w.m, top);
    float* mine = osh + (wave * 32 + fr) * S::LDO;
#pragma unroll
    for (int t = 0; t < WaveRows<DH>::DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = t * 32 + g * 8 + fk * 4;
        if (d < DH) *reinterpret_cast<floatx4*>(mine + d) = floatx4{w.o[t][4 * g] * f, w.o[t][4 * g + 1] * f, w.o[t][4 * g + 2] * f, w.o[t][4 * g + 3] * f};
      }
    wait_lds_barrier();
    constexpr int TPR = 8 / RW;                        // threads per row
    const int r = tid / TPR, rb = r >> 5, ri = r & 31;
    if (group0 + r >= rows) return;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < KG; ++k) m = fmaxf(m, ml[(k * RW + rb) * 64 + ri]);
#pragma unroll
    for (int k = 0; k < KG; ++k) l += ml[(k * RW + rb) * 64 + 32 + ri] * to_top(ml[(k * RW + rb) * 64 + ri], m);
    for (int d = (tid % TPR) * 4; d < DH; d += 4 * TPR) {
      floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KG; ++k) v += *reinterpret_cast<const floatx4*>(osh + ((k * RW + rb) * 32 + ri) * S::LDO + d);
      finish(group0 + r, d, v, m, l);
    }
  }
}

// mass_j += sum_i exp(s_ij - m_i) / l_i with the logits formed again, for many rows.  A workgroup has 32 entries; its waves share out the key heads,
// whose keys a lane holds while it goes through the rows 32 at a time: here a lane owns a key, so that the sum over rows is one
// over its own registers.  Waves are added in order.  A block of 32 x 32 takes 32 cross-lane reads of the rows' maxima and
// sums, 64 with slopes, beside 4 to 8 matrix instructions, and the cache's keys are read a second time: 8 x 48 nodes over
// 2000 .. 4000 entries of 8 key heads of 128 take 36 us without and 67 with weights.
template <int DH, int CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void attention_tree_mass_bf16_kernel(CacheRef c, const bf16_t* __restrict__ qkv, int H, const int32_t* __restrict__ positions,
                                                                          PlanAny plan, int B, int xblks, ScoreArgs sc, const float* __restrict__ ends) {
  __shared__ float part[4][32];
  const int id = (int)blockIdx.x, q = id / xblks, e0 = (id % xblks) * 32, G = H / c.KV;
  const int base = plan.at(q), n = plan.at(q + 1) - base, len = plan.at(2 * B + 1 + q), rows = n * G;
  const int64_t slot = plan.at(B + 1 + q);
  if (e0 >= len || n == 0) return;
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, fr = lane & 31, fk = lane >> 5;
  const size_t ld = (size_t)(H + 2 * c.KV) * DH;
  const int entry = min(e0 + fr, len - 1);
  const int kpos = BIAS ? c.positions[slot * c.capacity + entry] : 0;
  const Score2 score = Score2::of(sc, 0.f, 0);
  const float sign = sc.scale < 0.f ? -1.f : 1.f;
  float got = 0.f;
  for (int kh = wave; kh < c.KV; kh += 4) {
    bf16x8 kf[DH / 16];
    const bf16_t* k = (const bf16_t*)c.k + ((slot * c.KV + kh) * c.capacity + entry) * DH + fk * 8;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) kf[ks] = *reinterpret_cast<const bf16x8*>(k + ks * 16);
    for (int row0 = 0; row0 < rows; row0 += 32) {
      const int mine = min(row0 + fr, rows - 1);
      const bf16_t* x = qkv + (size_t)(base + mine / G) * ld + (size_t)(kh * G + mine % G) * DH + fk * 8;
      floatx16 s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < DH / 16; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(x + ks * 16), kf[ks], s, 0, 0, 0);
      // what the rows' logits are relative to: lane fr of either half has row row0 + fr
      const int64_t my_at = (int64_t)(base + mine / G) * H + kh * G + mine % G;
      const float my_m = ends[2 * my_at], my_l = ends[2 * my_at + 1];
      const float my_inv = my_l == 0.f || row0 + fr >= rows ? 0.f : 1.f / my_l;
      const float my_slope = BIAS ? sc.slopes[kh * G + mine % G] * 1.44269504088896340736f : 0.f;
      const int my_pos = BIAS ? positions[base + mine / G] : 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int r = 8 * (e >> 2) + 4 * fk + (e & 3);
        const float m = __shfl(my_m, r), inv = __shfl(my_inv, r);
        float v = CAP ? score.capped<CAP>(s[e] * sign) : s[e] * sign * score.scale2;
        if (BIAS) v -= __shfl(my_slope, r) * fabsf((float)(__shfl(my_pos, r) - kpos));
        got += inv == 0.f ? 0.f : __builtin_amdgcn_exp2f(v - m) * inv;
      }
    }
  }
  got = xor32_sum(got);
  if (fk == 0) part[wave][fr] = got;
  __syncthreads();
  if (threadIdx.x < 32 && e0 + (int)threadIdx.x < len)
    c.mass[slot * c.capacity + e0 + threadIdx.x] += (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}

hipError_t launch_attention_tree_bf16(const CacheRef& c, const void* qkv, int H, const int32_t* positions, const int32_t* plan, size_t count,
                                      const int32_t* d_plan, int B, int64_t T, int max_len, bool has_parents, const ScoreArgs& sc, bool add_mass,
                                      const TreeShape& shape, float* workspace, void* o, hipStream_t s) {
  const int64_t TH = T * H, wgs = (int64_t)B * c.KV * shape.groups * shape.parts;
  const int64_t join_wgs = shape.parts > 1 ? (TH + 3) / 4 : 0;
  const bool by_logits = add_mass && shape.rows == 32 && max_len > 0;
  const int xblks = (max_len + 255) / 256, kblks = (max_len + 31) / 32;
  if (wgs > kMostGroups || join_wgs + (int64_t)B * kblks > kMostGroups) return kTooManyGroups;
  const PlanAny p = plan_any(plan, count, d_plan);
  TreeBuffers buf;
  buf.TH = TH;
  buf.stride = tree_logit_stride(max_len);
  buf.ends = workspace;
  buf.tops = workspace + 2 * TH;
  buf.sums = workspace + tree_sums_at(shape, T, H);
  buf.logits = by_logits ? workspace + tree_logits_at(shape, T, H, c.dh) : nullptr;
  if (!add_mass) buf.ends = nullptr;
  auto run = [&](auto width, auto rw, auto cap, auto bias) {
    constexpr int DH = decltype(width)::value, RW = decltype(rw)::value;
    auto kern = attention_tree_bf16_kernel<DH, RW, decltype(cap)::value, decltype(bias)::value>;
    hipError_t e = set_max_dynamic_lds((const void*)kern, (int)TreeTile<DH, RW>::LDS);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)wgs), dim3(256), TreeTile<DH, RW>::LDS, s>>>(c, (const bf16_t*)qkv, H, positions, p, B, has_parents, shape, sc, CapArgs::of(sc), buf, (bf16_t*)o);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t second = join_wgs + (by_logits ? (int64_t)B * xblks : 0);
    if (second > 0) {
      e = launch_attention_tree_join<bf16_t>(c, p, B, H, shape, buf, join_wgs, by_logits ? xblks : 0, o, s);
      if (e != hipSuccess) return e;
    }
    if (add_mass && !by_logits && max_len > 0) {
      attention_tree_mass_bf16_kernel<DH, decltype(cap)::value, decltype(bias)::value>
          <<<dim3((unsigned)(B * kblks)), dim3(256), 0, s>>>(c, (const bf16_t*)qkv, H, positions, p, B, kblks, sc, buf.ends);
      e = hipGetLastError();
    }
    return e;
  };
  auto by_rows = [&](auto width, auto cap, auto bias) {
    switch (shape.rows) {
      case 32: return run(width, std::integral_constant<int, 1>{}, cap, bias);
      case 64: return run(width, std::integral_constant<int, 2>{}, cap, bias);
      case 128: return run(width, std::integral_constant<int, 4>{}, cap, bias);
    }
    return hipErrorInvalidValue;
  };
  auto pick = [&](auto width) {
    auto with_bias = [&](auto cap) { return sc.slopes ? by_rows(width, cap, std::true_type{}) : by_rows(width, cap, std::false_type{}); };
    switch (Score2::cap_form(sc.cap)) {
      case 0: return with_bias(std::integral_constant<int, 0>{});
      case 1: return with_bias(std::integral_constant<int, 1>{});
    }
    return with_bias(std::integral_constant<int, 2>{});
  };
  switch (c.dh) {
    case 64: return pick(std::integral_constant<int, 64>{});
    case 80: return pick(std::integral_constant<int, 80>{});
    case 96: return pick(std::integral_constant<int, 96>{});
    case 128: return pick(std::integral_constant<int, 128>{});
  }
  return hipErrorInvalidValue;
}

}  // namespace otas
