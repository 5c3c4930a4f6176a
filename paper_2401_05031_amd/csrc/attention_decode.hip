// Attention of the decoder's operators with fp32 products (f32 models, and bf16 ones of head widths that the kernels of
// attention_masked_bf16.hip and attention_tree_bf16.hip are not built for):
//   o_i = sum_j w_ij v_j / sum_j w_ij,  w_ij = exp(s_ij - max_j s_ij) over the keys j that row i sees,
// in one pass over the keys with the running maximum and sum of the softmax.  All arithmetic is fp32, on
// v_mfma_f32_32x32x2_f32 for both products; bf16 operands are widened, at the fp32 rate: 2 x 2000 causal bf16 rows of 16 heads of 48, 72
// and 112 take 171, 258 and 400 us (72 TFLOP/s) where 64, 80 and 128 take 45, 50 and 61; a token of 24 queries over 4000 entries of 4 key
// heads of 72 takes 78 us, of 80 38.
#include "attention_decode.h"
#include "attention_rows_f32.h"
#include "attention_tree_join.h"

namespace otas {

// --------------------------------------------------------------------------------------------------------- packed rows
template <typename T> struct PackedKeys {
  const T *kp, *vp;
  int ld, end;                            // keys from `end` on are seen by no row of the workgroup
  RowMask mask;
  RowScore score;
  const int32_t *documents, *positions;   // the query's, or NULL
  int full, fk;                           // keys below `full` are seen by every row of the wave; the lane's half
  __device__ bool sees(int j) const { return j < end && mask.sees(j, documents ? documents[j] : 0); }
  __device__ void logits(floatx16& s, int kb) const {
    score.capped(s);
    if (score.sloped) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = min(kb + 8 * (e >> 2) + 4 * fk + (e & 3), end - 1);
        s[e] = score.with_distance(s[e], positions ? positions[j] : j);
      }
    }
    if (documents) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        int d[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] = documents[min(kb + 8 * g + 4 * fk + e, end - 1)];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = kb + 8 * g + 4 * fk + e;
          s[4 * g + e] = ((j < end) & mask.sees(j, d[e])) ? s[4 * g + e] : -INFINITY;
        }
      }
    } else if (kb + 32 > full) {
      const int left = min(end, max(mask.prefix, mask.causal ? mask.row + 1 : end)) - kb - 4 * fk;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + (e & 3) < left ? s[e] : -INFINITY;
    }
  }
  __device__ bool partial(int kb) const { return documents || kb + 32 > full; }
};

// Four waves have 32 rows of a head between them and take the key blocks in turn: a short query of few heads then still has a
// wave for every SIMD.  8 queries of 209 .. 261 rows behind a prefix of 197, 12 heads of 64: 29 us, where the products alone would
// take 8 (756 workgroups of two or three blocks of keys a wave, 3 us before the first; 16 of them find no room in the first round).
template <typename T, int DT, bool WHOLE>
__global__ __launch_bounds__(256, DT <= 2 ? 3 : 2) void attention_masked_f32_kernel(const T* __restrict__ qkv, PlanAny plan, int B, int H, int KV, int width, int xblks,
                                                                   ScoreArgs sc, MaskArgs mk, T* __restrict__ o) {
  extern __shared__ __attribute__((aligned(16))) float f32_lds[];
  // The last rows first (under a causal mask they have the most keys); the row blocks of a head on one XCD where heads divide so.
  const int id = (int)blockIdx.x, pairs = B * H;
  int pair, xblk;
  if (pairs % 8 == 0) {
    const int mine = pairs >> 3, k = id >> 3;
    pair = xcd_head(id & 7, k % mine, H);
    xblk = xblks - 1 - k / mine;
  } else {
    pair = id % pairs;
    xblk = xblks - 1 - id / pairs;
  }
  const int h = pair % H, q = pair / H, dh = WHOLE ? 32 * DT : width;
  const int base = plan.at(q), n = plan.at(q + 1) - base, row0 = xblk * 32;
  if (row0 >= n) return;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), fr = lane & 31, fk = lane >> 5;
  const int row = min(row0 + fr, n - 1), prefix = plan.at(B + 1 + q);
  const size_t ld = (size_t)(H + 2 * KV) * dh;
  const T* first = qkv + (size_t)base * ld;
  const int kh = h / (H / KV);
  const int32_t* docs = mk.documents ? mk.documents + base : nullptr;
  const int32_t* pos = mk.positions ? mk.positions + base : nullptr;
  const int end = mk.causal ? max(min(row0 + 32, n), prefix) : n;
  const PackedKeys<T> keys{first + (size_t)(H + kh) * dh, first + (size_t)(H + KV + kh) * dh, (int)ld, end,
                           RowMask{row, docs ? docs[row] : 0, prefix, mk.causal},
                           RowScore::of(sc, h, pos ? pos[row] : row), docs, pos, mk.causal ? max(min(row0 + 1, n), prefix) : n, fk};
  FloatRows<T, DT> r;
  rows_begin<T, DT>(r, first + (size_t)row * ld + (size_t)h * dh, dh, fk);
  rows_stream<T, DT>(r, keys, dh, wave, (end + 31) >> 5, 4, fr, fk);
  T* out = o + ((size_t)base + row0) * H * dh + (size_t)h * dh;
  rows_join<T, DT>(r, dh, f32_lds, [&](int i, int d, floatx4 v, float, float l) {
    if (row0 + i < n) store_row4<T>(out + (size_t)i * H * dh + d, v, l);
  });
}

template <typename T>
static hipError_t attention_masked_f32(const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B, int max_n,
                                       int H, int KV, int dh, const ScoreArgs& sc, const MaskArgs& mk, void* o, hipStream_t s) {
  const int xblks = (max_n + 31) / 32;
  const int64_t wgs = (int64_t)xblks * H * B;
  if (wgs > kMostGroups) return kTooManyGroups;
  const PlanAny p = plan_any(plan, count, d_plan);
  return with_tiles(dh, [&](auto dt, auto whole) {
    constexpr int DT = decltype(dt)::value;
    auto kern = attention_masked_f32_kernel<T, DT, decltype(whole)::value>;
    const hipError_t e = set_max_dynamic_lds((const void*)kern, (int)float_rows_lds<DT>());
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)wgs), dim3(256), float_rows_lds<DT>(), s>>>((const T*)qkv, p, B, H, KV, dh, xblks, sc, mk, (T*)o);
    return hipGetLastError();
  });
}

hipError_t launch_attention_masked(int dtype, const void* qkv, const int32_t* plan, size_t count, const int32_t* d_plan, int B,
                                   int max_n, int H, int KV, int dh, const ScoreArgs& sc, const MaskArgs& mk, void* o, hipStream_t s) {
  if (max_n <= 0) return hipSuccess;
  if (dtype != 0 && bf16_width(dh)) return launch_attention_masked_bf16(qkv, plan, count, d_plan, B, max_n, H, KV, dh, sc, mk, o, s);
  return dtype == 0 ? attention_masked_f32<float>(qkv, plan, count, d_plan, B, max_n, H, KV, dh, sc, mk, o, s)
                    : attention_masked_f32<bf16_t>(qkv, plan, count, d_plan, B, max_n, H, KV, dh, sc, mk, o, s);
}

// ------------------------------------------------------------------------------------------------ a tree over the cache
template <typename T> struct CachedKeys {
  const T *kp, *vp;   // the slot's key head
  int ld, end, fk;    // entries; the lane's half
  RowScore score;
  const int32_t* positions;   // of the slot, read where there are slopes
  __device__ bool sees(int j) const { return j < end; }
  __device__ void logits(floatx16& s, int kb) const {
    score.capped(s);
    if (score.sloped) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = score.with_distance(s[e], positions[min(kb + 8 * (e >> 2) + 4 * fk + (e & 3), end - 1)]);
    }
    if (partial(kb)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = sees(kb + 8 * (e >> 2) + 4 * fk + (e & 3)) ? s[e] : -INFINITY;
    }
  }
  __device__ bool partial(int kb) const { return kb + 32 > end; }
};
template <typename T> struct DraftKeys {
  const T *kp, *vp;
  int ld, end, fk;
  uint64_t line;   // the nodes that the lane's node sees
  RowScore score;
  const int32_t* positions;
  __device__ bool sees(int j) const { return j < end && (line >> (j & 63) & 1); }
  __device__ void logits(floatx16& s, int kb) const {
    score.capped(s);
    if (score.sloped) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = score.with_distance(s[e], positions[min(kb + 8 * (e >> 2) + 4 * fk + (e & 3), end - 1)]);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = sees(kb + 8 * (e >> 2) + 4 * fk + (e & 3)) ? s[e] : -INFINITY;
  }
  __device__ bool partial(int) const { return true; }
};

// A workgroup has 32 rows (nodes x heads that share a key head) and one chunk of the cache, or the nodes themselves; with one chunk
// both, and the rows are done, else the sums go to the workspace for the join.
template <typename T, int DT, bool WHOLE>
__global__ __launch_bounds__(256, DT <= 2 ? 3 : 2) void attention_tree_f32_kernel(CacheRef c, const T* __restrict__ qkv, int H, const int32_t* __restrict__ positions,
                                                                 PlanAny plan, int B, bool has_parents, TreeShape shape, ScoreArgs sc,
                                                                 float* __restrict__ sums, float* __restrict__ tops, float* __restrict__ ends, int64_t TH,
                                                                 T* __restrict__ o) {
  extern __shared__ __attribute__((aligned(16))) float f32_lds[];
  int id = (int)blockIdx.x;
  const int part = id % shape.parts;
  id /= shape.parts;
  const int group = id % shape.groups;
  id /= shape.groups;
  const int kh = id % c.KV, q = id / c.KV, dh = WHOLE ? 32 * DT : c.dh, G = H / c.KV;
  const int base = plan.at(q), n = plan.at(q + 1) - base, len = plan.at(2 * B + 1 + q), row0 = group * 32;
  const int64_t slot = plan.at(B + 1 + q);
  // The last part may be the nodes' of queries of several chunks.
  const int chunks = shape.chunks(len);
  const bool apart = shape.apart && shape.parts > 1 && part == shape.parts - 1, nodes = apart || (part == 0 && (chunks <= 1 || !shape.apart));
  if (row0 >= n * G || (apart ? chunks <= 1 : part > 0 && part >= chunks)) return;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), fr = lane & 31, fk = lane >> 5;
  const int row = min(row0 + fr, n * G - 1), node = row / G, head = kh * G + row % G;
  const size_t ld = (size_t)(H + 2 * c.KV) * dh;
  const T* first = qkv + (size_t)base * ld;
  const RowScore score = RowScore::of(sc, head, sc.slopes ? positions[base + node] : 0);
  FloatRows<T, DT> r;
  rows_begin<T, DT>(r, first + (size_t)node * ld + (size_t)head * dh, dh, fk);
  const int begin = apart ? 0 : part * shape.chunk, end = apart ? 0 : min(len, begin + shape.chunk);   // chunks are whole blocks
  if (begin < end) {
    const T* heads_k = (const T*)c.k + (slot * c.KV + kh) * c.capacity * dh;
    const T* heads_v = (const T*)c.v + (slot * c.KV + kh) * c.capacity * dh;
    const CachedKeys<T> keys{heads_k, heads_v, dh, end, fk, score, c.positions + slot * c.capacity};
    rows_stream<T, DT>(r, keys, dh, (begin >> 5) + wave, (end + 31) >> 5, 4, fr, fk);
  }
  if (nodes) {
    const uint64_t line = tree_lines(plan, 3 * B + 1, base, n, has_parents, lane);
    const DraftKeys<T> keys{first + (size_t)(H + kh) * dh, first + (size_t)(H + c.KV + kh) * dh, (int)ld, n, fk, lane_value(line, node), score, positions + base};
    rows_stream<T, DT>(r, keys, dh, wave, (n + 31) >> 5, 4, fr, fk);
  }
  const bool only = chunks <= 1;   // the rows' one chunk
  const int64_t place = apart ? chunks : part;
  rows_join<T, DT>(r, dh, f32_lds, [&](int i, int d, floatx4 v, float m, float l) {
    if (row0 + i >= n * G) return;
    const int64_t at = (int64_t)(base + (row0 + i) / G) * H + kh * G + (row0 + i) % G;
    if (only) {
      store_row4<T>(o + at * dh + d, v, l);
      if (ends && d == 0) { ends[2 * at] = m; ends[2 * at + 1] = l; }
    } else {
      *reinterpret_cast<floatx4*>(sums + (place * TH + at) * dh + d) = v;
      if (d == 0) { tops[2 * (place * TH + at)] = m; tops[2 * (place * TH + at) + 1] = l; }
    }
  });
}

// mass_j += sum over rows and heads of exp(s_ij - m_i) / l_i, with the logits formed again (the weights of one pass are
// relative to maxima that the next chunk may change, and keeping them all would be 4 bytes a row and key).  A workgroup has 32
// entries; its waves share out the key heads, whose keys a lane holds while it goes through the rows 32 at a time: here a lane owns
// a key, so that the sum over rows is one over its own registers.  Waves are added in order.
template <typename T, int DT, bool WHOLE>
__global__ __launch_bounds__(256) void attention_tree_mass_kernel(CacheRef c, const T* __restrict__ qkv, int H, const int32_t* __restrict__ positions,
                                                                  PlanAny plan, int B, int xblks, ScoreArgs sc, const float* __restrict__ ends) {
  __shared__ float part[4][32];
  const int id = (int)blockIdx.x, q = id / xblks, e0 = (id % xblks) * 32, dh = WHOLE ? 32 * DT : c.dh, G = H / c.KV;
  const int base = plan.at(q), n = plan.at(q + 1) - base, len = plan.at(2 * B + 1 + q);
  const int64_t slot = plan.at(B + 1 + q);
  if (e0 >= len || n == 0) return;
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, fr = lane & 31, fk = lane >> 5;
  const size_t ld = (size_t)(H + 2 * c.KV) * dh;
  const int entry = min(e0 + fr, len - 1);
  const int kpos = sc.slopes ? c.positions[slot * c.capacity + entry] : 0;
  float got = 0.f;
  for (int kh = wave; kh < c.KV; kh += 4) {
    floatx4 kf[4 * DT];
    load_heads<T, DT>(kf, (const T*)c.k + ((slot * c.KV + kh) * c.capacity + entry) * dh, dh, fk);
    for (int row0 = 0; row0 < n * G; row0 += 32) {
      const int mine = min(row0 + fr, n * G - 1);
      floatx4 qf[4 * DT];
      load_heads<T, DT>(qf, qkv + (size_t)(base + mine / G) * ld + (size_t)(kh * G + mine % G) * dh, dh, fk);
      // what the rows' logits are formed with and relative to: lane fr of either half has row row0 + fr
      const int64_t my_at = (int64_t)(base + mine / G) * H + kh * G + mine % G;
      const float my_m = ends[2 * my_at], my_l = ends[2 * my_at + 1];
      const float my_inv = my_l == 0.f || row0 + fr >= n * G ? 0.f : 1.f / my_l;
      const RowScore my = RowScore::of(sc, kh * G + mine % G, sc.slopes ? positions[base + mine / G] : 0);
      floatx16 s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int g = 0; g < 4 * DT; ++g)
        if (8 * g < dh) {
#pragma unroll
          for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_32x32x2f32(qf[g][u], kf[g][u], s, 0, 0, 0);
        }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (row0 + 8 * (e >> 2) + (e & 3) >= n * G) continue;   // of either half
        const int r = 8 * (e >> 2) + 4 * fk + (e & 3);
        const float m = __shfl(my_m, r), inv = __shfl(my_inv, r);
        float v = my.scaled(s[e]);
        if (my.sloped) v -= __shfl(my.slope2, r) * fabsf((float)(__shfl(my.position, r) - kpos));
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

template <typename T>
static hipError_t attention_tree_any(const CacheRef& c, const void* qkv, int H, const int32_t* positions, const int32_t* plan, size_t count,
                                     const int32_t* d_plan, int B, int64_t T_, int max_len, bool has_parents, const ScoreArgs& sc,
                                     bool add_mass, const TreeShape& shape, float* workspace, void* o, hipStream_t s) {
  const int64_t TH = T_ * H, wgs = (int64_t)B * c.KV * shape.groups * shape.parts;
  const int xblks = (max_len + 31) / 32;
  if (wgs > kMostGroups || (TH + 3) / 4 > kMostGroups || (int64_t)B * xblks > kMostGroups) return kTooManyGroups;
  float* ends = workspace;
  float* tops = workspace + 2 * TH;
  float* sums = workspace + tree_sums_at(shape, T_, H);
  const PlanAny p = plan_any(plan, count, d_plan);
  return with_tiles(c.dh, [&](auto dt, auto whole) {
    constexpr int DT = decltype(dt)::value;
    constexpr bool WHOLE = decltype(whole)::value;
    auto kern = attention_tree_f32_kernel<T, DT, WHOLE>;
    const hipError_t e = set_max_dynamic_lds((const void*)kern, (int)float_rows_lds<DT>());
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)wgs), dim3(256), float_rows_lds<DT>(), s>>>(c, (const T*)qkv, H, positions, p, B, has_parents, shape, sc, sums, tops,
                                                                       add_mass ? ends : nullptr, TH, (T*)o);
    if (shape.parts > 1) {
      const TreeBuffers buf{sums, tops, add_mass ? ends : nullptr, nullptr, TH, 0};
      const hipError_t j = launch_attention_tree_join<T>(c, p, B, H, shape, buf, (TH + 3) / 4, 0, o, s);
      if (j != hipSuccess) return j;
    }
    if (add_mass && max_len > 0)
      attention_tree_mass_kernel<T, DT, WHOLE><<<dim3((unsigned)(B * xblks)), dim3(256), 0, s>>>(c, (const T*)qkv, H, positions, p, B, xblks, sc, ends);
    return hipGetLastError();
  });
}

hipError_t launch_attention_tree(int dtype, const CacheRef& c, const void* qkv, int H, const int32_t* positions, const int32_t* plan,
                                 size_t count, const int32_t* d_plan, int B, int64_t T, int max_len, bool has_parents, const ScoreArgs& sc,
                                 bool add_mass, const TreeShape& shape, float* workspace, void* o, hipStream_t s) {
  if (T <= 0) return hipSuccess;
  if (dtype != 0 && bf16_width(c.dh))
    return launch_attention_tree_bf16(c, qkv, H, positions, plan, count, d_plan, B, T, max_len, has_parents, sc, add_mass, shape, workspace, o, s);
  return dtype == 0 ? attention_tree_any<float>(c, qkv, H, positions, plan, count, d_plan, B, T, max_len, has_parents, sc, add_mass, shape, workspace, o, s)
                    : attention_tree_any<bf16_t>(c, qkv, H, positions, plan, count, d_plan, B, T, max_len, has_parents, sc, add_mass, shape, workspace, o, s);
}

}  // namespace otas
