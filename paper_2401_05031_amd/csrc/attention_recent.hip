// Attention of a query's last tokens over its cache, through a window: otas_attention_recent (a cache of the model's dtype) and
// otas_attention_cache4 (one of 4 bits an element).
//   A workgroup has 16 R rows (tokens x heads that share a key head) and a share of the tiles of 32 entries that they see.  Its four
// waves have the same rows and take tiles in turn, each on its own: no barrier and no LDS before the end, where the four are joined.
//   Both products are formed transposed on v_mfma_f32_16x16x32_bf16,
//     S^T[key, row] = K Q^T,   O^T[d, row] += V^T P^T,
// lane (i = lane & 15, b = lane >> 4) supplying row i and k-slots 8 b .. 8 b + 7 of either operand.  Sums over k do not care which k
// lies in which slot, nor the rows of a tile which d they are, so that operands are taken from memory as they lie:
//   K: of a key's head lane b has the b-th run of STEPS words of eight elements (16 bytes at 4 bits and width 128); queries likewise.
//   V: of the tile's 32 keys lane b has 8 b .. 8 b + 7, and lane i the head's i-th eight elements of each: V^T's row i of product t is
//      element 8 i + t.  A pair of keys' elements change places between two registers (v_perm_b32), nothing leaves the lane.
//   S: rows 4 b + e of the first and second product are keys 8 b + e and 8 b + 4 + e: what lane b needs of P for its keys is what it has.
// bf16 models: queries, keys and values as they are, weights rounded to bf16 (by 2^-8 of themselves at most, as much as the output's own
// rounding), their sum unrounded.  f32 models: every float operand x is cut into three bf16 pieces whose sum is x (8 bits each, by
// truncation, so that none overflows), and the products of all pieces but the last two's are added up.  What is held in 4 bits is one
// piece.
//   Bound by HBM where there are tokens enough: one token of each of 32 queries, 8 key heads of 128: the last 2048 of 8192 entries (268 MB) 44 us,
// 6.1 TB/s, part from the last-level cache; 5700 .. 8192 entries in 4 bits (244 MB) 48 us, 5.1 TB/s, and the join 5.  f32: 32 tokens over 4000 entries, 8 heads of
// 128 (1.05 GB) 200 us.  A small call is a chain of latencies: launch and plan 3 us, queries and the first tiles 2, a step of a tile 1 (f32 2), the
// waves' join 1.  Two tiles ahead in 4 bits; of the model's dtype one (two: bf16 equal, f32 1.4 to 2.8 times as long, for registers).
#include "attention_tiles.h"
#include "cache4.h"

namespace otas {

namespace {

constexpr int kTile = 1 << kRecentShift;

__device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }
// The upper halves, or the lower ones, of two words as a pair, the first's in the lower half.
__device__ __forceinline__ uint32_t uppers(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t lowers(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// Pieces of two floats, as pairs.
__device__ __forceinline__ void cut(float x, float y, uint32_t (&piece)[3]) {
  constexpr uint32_t upper = 0xFFFF0000u;
  piece[0] = uppers(bits(x), bits(y));
  x -= __uint_as_float(bits(x) & upper);
  y -= __uint_as_float(bits(y) & upper);
  piece[1] = uppers(bits(x), bits(y));
  x -= __uint_as_float(bits(x) & upper);
  y -= __uint_as_float(bits(y) & upper);
  piece[2] = uppers(bits(x), bits(y));
}

struct Words { uint32_t x[4]; };   // eight bf16
__device__ __forceinline__ bf16x8 operand(const Words& w) {
  bf16x8 f;
  __builtin_memcpy(&f, &w, 16);
  return f;
}
__device__ __forceinline__ floatx4 product(const Words& a, const Words& b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(a), operand(b), c, 0, 0, 0);
}

// Eight elements of the model's dtype as pieces.
template <typename T> constexpr int pieces_of() { return sizeof(T) == 4 ? 3 : 1; }
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  uint4 u;
  __device__ __forceinline__ void load(const char* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void clear() { u = uint4{0, 0, 0, 0}; }
  __device__ __forceinline__ void negate() { u.x ^= 0x80008000u; u.y ^= 0x80008000u; u.z ^= 0x80008000u; u.w ^= 0x80008000u; }
  template <int I> __device__ __forceinline__ void pair(uint32_t (&piece)[1]) const { piece[0] = I == 0 ? u.x : I == 1 ? u.y : I == 2 ? u.z : u.w; }
  // Elements that are not finite become 0; whether there were any.
  __device__ __forceinline__ bool make_finite() {
    uint32_t* x = &u.x;
    uint32_t any = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t odd = ((((x[k] & 0x7F807F80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xFFFFu;   // ones over elements whose exponent is all ones
      any |= odd;
      x[k] &= ~odd;
    }
    return any != 0;
  }
  __device__ __forceinline__ float element(int j) const { const uint32_t w = (&u.x)[j >> 1]; return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16); }
};
template <> struct Eight<float> {
  floatx4 a, b;
  __device__ __forceinline__ void load(const char* p) { a = *reinterpret_cast<const floatx4*>(p); b = *reinterpret_cast<const floatx4*>(p + 16); }
  __device__ __forceinline__ void clear() { a = b = floatx4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void negate() { a = -a; b = -b; }
  template <int I> __device__ __forceinline__ void pair(uint32_t (&piece)[3]) const {
    if (I < 2) cut(a[2 * I & 3], a[(2 * I & 3) + 1], piece); else cut(b[2 * I & 3], b[(2 * I & 3) + 1], piece);
  }
  __device__ __forceinline__ bool make_finite() {
    bool any = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!__builtin_isfinite(a[k])) { a[k] = 0.f; any = true; }
      if (!__builtin_isfinite(b[k])) { b[k] = 0.f; any = true; }
    }
    return any;
  }
  __device__ __forceinline__ float element(int j) const { return j < 4 ? a[j & 3] : b[j & 3]; }
};

// What a lane has loaded of a tile, and the operands it makes of that.  KeyPieces: pieces of a key's and a value's elements.
template <typename T, bool FOUR, int STEPS, bool EXACT> struct Tile;

// Where the heads of a slot lie, and which parts of a tile are a lane's: bytes from the tile's first key on.
struct Source {
  const char *k, *v, *ks, *vs;       // the slot's key head; ks, vs: its scales
  int64_t capacity;
  int words, b;                      // runs of eight elements a head; the lane's block
  uint32_t row;                      // bytes of a key
  uint32_t k_at, v_at, ks_at[3], vs_at;
};

template <int STEPS, bool EXACT> struct Codes {
  static constexpr int PIECES = 1, SCALES = STEPS == 3 ? 3 : 1;
  uint32_t k[2][STEPS], ks[2][SCALES], v[8];
  uint2 vs;
  static __device__ __forceinline__ void places(Source& s, int i16) {
    s.row = s.words * 4;
    s.k_at = (8 * (i16 >> 2) + (i16 & 3)) * s.row + s.b * STEPS * 4;
    const int word = min(i16, s.words - 1);
    s.v_at = 8 * s.b * s.row + word * 4;
    s.vs_at = (uint32_t)((word >> 2) * s.capacity) + 8 * s.b;
#pragma unroll
    for (int g = 0; g < SCALES; ++g) s.ks_at[g] = (uint32_t)((min(s.b * STEPS + g, s.words - 1) >> 2) * s.capacity) + 8 * (i16 >> 2) + (i16 & 3);
  }
  __device__ __forceinline__ void load(const Source& s, int tile) {
    const char* k0 = s.k + (size_t)tile * kTile * s.row;
    const char* v0 = s.v + (size_t)tile * kTile * s.row;
    const char* ks0 = s.ks + tile * kTile;
    const char* vs0 = s.vs + tile * kTile;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t at = s.k_at + 4 * h * s.row;
      if (EXACT) {
        __builtin_memcpy(k[h], k0 + at, STEPS * 4);
      } else {
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          const bool there = s.b * STEPS + st < s.words;
          const uint32_t w = *reinterpret_cast<const uint32_t*>(k0 + (there ? at + 4 * st : at - s.b * STEPS * 4));
          k[h][st] = there ? w : 0;
        }
      }
#pragma unroll
      for (int g = 0; g < SCALES; ++g) ks[h][g] = *reinterpret_cast<const uint8_t*>(ks0 + (s.ks_at[g] + 4 * h));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const uint32_t*>(v0 + (s.v_at + j * s.row));
    vs = *reinterpret_cast<const uint2*>(vs0 + s.vs_at);
  }
  // The lane's key of the first (H = 0) or second product: its words ST as operands.
  template <int H, int ST> __device__ __forceinline__ void key(Words (&w)[1]) const {
    const uint32_t byte = ks[H][SCALES == 1 ? 0 : ST];
    const float f = scale4(byte);
    w[0].x[0] = pair4_bf16<0>(k[H][ST], f);
    w[0].x[1] = pair4_bf16<1>(k[H][ST], f);
    w[0].x[2] = pair4_bf16<2>(k[H][ST], f);
    w[0].x[3] = pair4_bf16<3>(k[H][ST], f);
    if ((SCALES == 3 || ST == 0) && byte == kNoNumber) w[0].x[0] = 0x7FC07FC0u;   // a product with it is NaN, whatever the others are
  }
  uint32_t vb[8];   // scales of the lane's keys
  // Values ready for use: keys from `end` on of the tile (their scales may be anything) and groups that are no numbers become 0.
  // Whether there were any of the latter among the former keys.
  __device__ __forceinline__ bool prepare(int b, int end, bool) {
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      vb[j] = (j < 4 ? vs.x : vs.y) >> (8 * (j & 3)) & 255;
      if (end < kTile) vb[j] = 8 * b + j < end ? vb[j] : 0;
      most = max(most, vb[j]);
    }
    if (!__any(most == kNoNumber)) return false;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (vb[j] == kNoNumber) { vb[j] = 0; v[j] = 0; }
    return true;
  }
  template <int I> __device__ __forceinline__ void value_pair(int j, uint32_t (&piece)[1]) const { piece[0] = pair4_bf16<I>(v[j], scale4(vb[j])); }
};

template <typename T, int STEPS, bool EXACT> struct Plain {
  static constexpr int PIECES = pieces_of<T>();
  Eight<T> k[2][STEPS], v[8];
  static constexpr uint32_t RUN = 8 * sizeof(T);
  static __device__ __forceinline__ void places(Source& s, int i16) {
    s.row = s.words * RUN;
    s.k_at = 8 * (i16 >> 2) + (i16 & 3);   // the key: the slot may end within the tile
    s.v_at = min(i16, s.words - 1) * RUN;
  }
  __device__ __forceinline__ void load(const Source& s, int tile) {
    const char* k0 = s.k + (size_t)tile * kTile * s.row;
    const char* v0 = s.v + (size_t)tile * kTile * s.row;
    const int last = (int)min(s.capacity - 1 - (int64_t)tile * kTile, (int64_t)kTile - 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t at = min((int)s.k_at + 4 * h, last) * s.row;
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const int w = s.b * STEPS + st;
        k[h][st].load(k0 + (at + (EXACT ? w : min(w, s.words - 1)) * RUN));
        if (!EXACT && w >= s.words) k[h][st].clear();
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j].load(v0 + (min(8 * s.b + j, last) * s.row + s.v_at));
  }
  template <int H, int ST> __device__ __forceinline__ void key(Words (&w)[PIECES]) const {
    uint32_t p[PIECES];
    k[H][ST].template pair<0>(p);
#pragma unroll
    for (int n = 0; n < PIECES; ++n) w[n].x[0] = p[n];
    k[H][ST].template pair<1>(p);
#pragma unroll
    for (int n = 0; n < PIECES; ++n) w[n].x[1] = p[n];
    k[H][ST].template pair<2>(p);
#pragma unroll
    for (int n = 0; n < PIECES; ++n) w[n].x[2] = p[n];
    k[H][ST].template pair<3>(p);
#pragma unroll
    for (int n = 0; n < PIECES; ++n) w[n].x[3] = p[n];
  }
  // Of a tile that some row does not see all of, values that are not finite become 0 too.
  __device__ __forceinline__ bool prepare(int b, int end, bool whole) {
    if (whole) return false;
    bool any = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (8 * b + j >= end) v[j].clear();
      any |= v[j].make_finite();
    }
    return any;
  }
  template <int I> __device__ __forceinline__ void value_pair(int j, uint32_t (&piece)[PIECES]) const { v[j].template pair<I>(piece); }
};

template <typename T, bool FOUR, int STEPS, bool EXACT> struct TileOf { typedef Plain<T, STEPS, EXACT> type; };
template <typename T, int STEPS, bool EXACT> struct TileOf<T, true, STEPS, EXACT> { typedef Codes<STEPS, EXACT> type; };

__device__ __forceinline__ float xor16_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

}  // namespace

constexpr size_t recent_lds(int steps) { return sizeof(float) * (4 * 2 * 16 + 4 * 16 * (32 * (size_t)steps + 4)); }

// cap, slopes: whether the call has them.
template <typename T, bool FOUR, int STEPS, bool EXACT, int R>
__global__ __launch_bounds__(256, R == 1 ? (FOUR && sizeof(T) == 2 ? 3 : 2) : 1) void attention_recent_kernel(PlanAny plan_, Cache4Ref c, const T* __restrict__ qkv, int H, int B, WindowShape shape,
                                                               ScoreArgs sc, RecentBuffers out, T* __restrict__ o) {
  typedef typename TileOf<T, FOUR, STEPS, EXACT>::type Held;
  constexpr int NQ = pieces_of<T>(), NK = Held::PIECES, DEPTH = FOUR ? 2 : 1, LDO = 32 * STEPS + 4;
  extern __shared__ __attribute__((aligned(16))) float lds_recent[];
  const PlanFirst plan = PlanFirst::of(plan_);
  const WorkPlace work = shape.work(plan, (int)blockIdx.x, B, c.KV);
  const int part = work.part, kh = work.unit % c.KV, q = work.unit / c.KV, G = H / c.KV;
  const int base = plan.at(q), n = plan.at(q + 1) - base, len = plan.at(2 * B + 1 + q), rows = n * G, group0 = work.group * 16 * R;
  const int window = shape.window, sinks = shape.sinks;
  const int64_t slot = plan.at(B + 1 + q);
  if (group0 >= rows) return;
  const WindowTiles tiles = shape.tiles(work.group, n, G, len);
  // (Other control flow here, such as a way round the divisions, has cost float rows of 128 fifty spilled registers, and 1.4 times the time.)
  const int each = shape.each_of(tiles), begin = part * each, end = min(tiles.count, begin + each);
  if (begin >= end) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i16 = lane & 15, b = lane >> 4;
  const int words = c.dh / 8;
  const int64_t head_of = slot * c.KV + kh, row_bytes = FOUR ? words * 4 : c.dh * (int)sizeof(T);
  Source src;
  src.k = c.k + head_of * c.capacity * row_bytes;
  src.v = c.v + head_of * c.capacity * row_bytes;
  src.ks = FOUR ? c.ks + head_of * c.groups * c.capacity : nullptr;
  src.vs = FOUR ? c.vs + head_of * c.groups * c.capacity : nullptr;
  src.capacity = c.capacity;
  src.words = words;
  src.b = b;
  Held::places(src, i16);

  const size_t ld = (size_t)(H + 2 * c.KV) * c.dh;
  Words qf[R][STEPS][NQ];
  int place[R];          // the row's token
  float slope2[R];
  constexpr float log2e = 1.44269504088896340736f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = min(group0 + 16 * r + i16, rows - 1), token = row / G, head = kh * G + row % G;
    place[r] = len - n + token;
    slope2[r] = sc.slopes ? sc.slopes[head] * log2e : 0.f;
    const char* p = reinterpret_cast<const char*>(qkv + (size_t)(base + token) * ld + (size_t)head * c.dh);
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int w = b * STEPS + st;
      Eight<T> x;
      x.load(p + (EXACT ? w : min(w, words - 1)) * 8 * (int)sizeof(T));
      if (!EXACT && w >= words) x.clear();
      if (sc.scale < 0.f) x.negate();   // its size alone is applied later
      uint32_t piece[NQ];
      x.template pair<0>(piece);
#pragma unroll
      for (int m = 0; m < NQ; ++m) qf[r][st][m].x[0] = piece[m];
      x.template pair<1>(piece);
#pragma unroll
      for (int m = 0; m < NQ; ++m) qf[r][st][m].x[1] = piece[m];
      x.template pair<2>(piece);
#pragma unroll
      for (int m = 0; m < NQ; ++m) qf[r][st][m].x[2] = piece[m];
      x.template pair<3>(piece);
#pragma unroll
      for (int m = 0; m < NQ; ++m) qf[r][st][m].x[3] = piece[m];
    }
  }
  // of the workgroup's rows: the first's and the last's token
  const int p0 = len - n + group0 / G, p1 = len - n + min(group0 + 16 * R, rows) / G - (min(group0 + 16 * R, rows) % G == 0);
  auto is_whole = [&](int k0) { return k0 + kTile - 1 <= p0 && (k0 > p1 - window || k0 + kTile <= sinks); };

  floatx4 acc[R][8];
  float m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[r][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  // Logits in units of ln 2.  Without cap and slopes products stay as they are and the exponent takes the factor.
  const bool scaled = sc.cap > 0.f || sc.slopes;
  const float scale = fabsf(sc.scale), factor = sc.cap > 0.f ? scale / sc.cap : scale * log2e, cap2 = sc.cap * log2e, last_factor = scaled ? 1.f : factor;
  bool met = false;   // whether this wave took out values that are no numbers

  auto consume = [&](Held& x, int at) {
    const int k0 = tiles.tile(at) * kTile;
    const bool whole = is_whole(k0);
    floatx4 s[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r) s[r][0] = s[r][1] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto step = [&](auto st_) {
      constexpr int st = decltype(st_)::value;
      if constexpr (st < STEPS) {
        auto half = [&](auto h_) {
          constexpr int h = decltype(h_)::value;
          Words kf[NK];
          x.template key<h, st>(kf);
#pragma unroll
          for (int u = 0; u < NK; ++u)
#pragma unroll
            for (int w = 0; w < NQ; ++w)
              if (u + w < 4) {
#pragma unroll
                for (int r = 0; r < R; ++r) s[r][h] = product(kf[u], qf[r][st][w], s[r][h]);
              }
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
    Words pf[R][NQ];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (sc.cap > 0.f) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r][h][e] = cap2 * tanhf(s[r][h][e] * factor);
      } else if (scaled) {
        s[r][0] *= factor;
        s[r][1] *= factor;
      }
      const int behind = place[r] - k0 - 8 * b;   // the row's distance from the lane's first key
      if (sc.slopes) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r][h][e] -= slope2[r] * fabsf((float)(behind - 4 * h - e));
      }
      if (!whole) {
        const int left = sinks - k0 - 8 * b;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = 4 * h + e;
            const bool see = (j <= behind) & ((behind - j < window) | (j < left));
            s[r][h][e] = see ? s[r][h][e] : -INFINITY;
          }
      }
      float mx = fmaxf(fmaxf(fmaxf(s[r][0][0], s[r][0][1]), fmaxf(s[r][0][2], s[r][0][3])), fmaxf(fmaxf(s[r][1][0], s[r][1][1]), fmaxf(s[r][1][2], s[r][1][3])));
      if (__any(mx * last_factor > m[r] + 8.f)) {   // a weight may be up to 2^8: no accuracy is lost in a floating format, and of its range 2^8
        const float top = fmaxf(m[r], xor16_max(xor32_max(mx)) * last_factor);
        const float alpha = m[r] == top ? 1.f : __builtin_amdgcn_exp2f(m[r] - top);   // equal: also where both are -inf
        m[r] = top;
        l[r] *= alpha;
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[r][t] *= alpha;
      }
      const float top = m[r] == -INFINITY ? 0.f : m[r];   // nothing seen so far: all weights are 0
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[r][h][e] = __builtin_amdgcn_exp2f(fmaf(s[r][h][e], last_factor, -top));
          l[r] += s[r][h][e];
        }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          if constexpr (NQ == 1) {
            const bf16x2 v = {(bf16_t)s[r][h][e], (bf16_t)s[r][h][e + 1]};
            __builtin_memcpy(&pf[r][0].x[2 * h + e / 2], &v, 4);
          } else {
            uint32_t piece[3];
            cut(s[r][h][e], s[r][h][e + 1], piece);
#pragma unroll
            for (int w = 0; w < 3; ++w) pf[r][w].x[2 * h + e / 2] = piece[w];
          }
        }
    }
    met |= x.prepare(b, p1 + 1 - k0, whole);
    auto column = [&](auto t_) {   // elements 2 t and 2 t + 1 of every eight
      constexpr int t = decltype(t_)::value;
      Words lo[NK], hi[NK];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        uint32_t even[NK], odd[NK];
        x.template value_pair<t>(j, even);
        x.template value_pair<t>(j + 1, odd);
#pragma unroll
        for (int u = 0; u < NK; ++u) {
          lo[u].x[j / 2] = lowers(even[u], odd[u]);
          hi[u].x[j / 2] = uppers(even[u], odd[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < NK; ++u)
#pragma unroll
        for (int w = 0; w < NQ; ++w)
          if (u + w < 4) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
              acc[r][2 * t] = product(lo[u], pf[r][w], acc[r][2 * t]);
              acc[r][2 * t + 1] = product(hi[u], pf[r][w], acc[r][2 * t + 1]);
            }
          }
    };
    column(std::integral_constant<int, 0>{});
    column(std::integral_constant<int, 1>{});
    column(std::integral_constant<int, 2>{});
    column(std::integral_constant<int, 3>{});
  };
  // Tiles are asked for DEPTH ahead.
  Held held[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; ++i)
    if (begin + wave + 4 * i < end) held[i].load(src, tiles.tile(begin + wave + 4 * i));
  for (int at = begin + wave; at < end; at += 4 * DEPTH) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      const int mine = at + 4 * i;
      if (mine < end) {
        consume(held[i], mine);
        if (mine + 4 * DEPTH < end) held[i].load(src, tiles.tile(mine + 4 * DEPTH));
      }
    }
  }

  if (__any(met)) {   // what was taken out goes to the rows that see it.  Lane b has elements 32 b .. 32 b + 31 of its rows
    for (int at = begin + wave; at < end; at += 4) {
      const int k0 = tiles.tile(at) * kTile;
      if (!FOUR && is_whole(k0)) continue;
      for (int j = 0; j < kTile && k0 + j <= p1; ++j) {
        const int key = k0 + j;
        if constexpr (FOUR) {
          if (b >= c.groups || (uint8_t)src.vs[b * c.capacity + key] != kNoNumber) continue;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const bool see = key <= place[r] && (place[r] - key < window || key < sinks);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (FOUR) {
#pragma unroll
              for (int t = 0; t < 8; ++t) acc[r][t][e] = see ? __uint_as_float(0x7FC00000u) : acc[r][t][e];
            } else if (4 * b + e < words) {
              Eight<T> x;
              x.load(src.v + key * row_bytes + (4 * b + e) * 8 * (int)sizeof(T));
#pragma unroll
              for (int t = 0; t < 8; ++t) {
                const float f = x.element(t);
                acc[r][t][e] += see && !__builtin_isfinite(f) ? f : 0.f;
              }
            }
          }
        }
      }
    }
  }

  // The four waves' sums into one.
  float* ml = lds_recent;           // [4][2][16]
  float* osh = lds_recent + 128;    // [4][16][LDO]
  const bool only = shape.parts_of(tiles) == 1;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float sum = xor16_sum(xor32_sum(l[r]));
    if (r > 0) __syncthreads();
    if (b == 0) {
      ml[wave * 32 + i16] = m[r];
      ml[wave * 32 + 16 + i16] = sum;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w * 32 + i16]);
    const float f = to_top(m[r], top);
    float* mine = osh + (wave * 16 + i16) * LDO;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 8 * (4 * b + e);
      if (d < c.dh) {
        *reinterpret_cast<floatx4*>(mine + d) = floatx4{acc[r][0][e] * f, acc[r][1][e] * f, acc[r][2][e] * f, acc[r][3][e] * f};
        *reinterpret_cast<floatx4*>(mine + d + 4) = floatx4{acc[r][4][e] * f, acc[r][5][e] * f, acc[r][6][e] * f, acc[r][7][e] * f};
      }
    }
    __syncthreads();
    const int ri = tid >> 4, row = group0 + 16 * r + ri;
    if (row >= rows) continue;
    float most = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) most = fmaxf(most, ml[w * 32 + ri]);
#pragma unroll
    for (int w = 0; w < 4; ++w) total += ml[w * 32 + 16 + ri] * to_top(ml[w * 32 + ri], most);
    const int64_t to = (int64_t)(base + row / G) * H + kh * G + row % G;
    for (int d = (tid & 15) * 4; d < c.dh; d += 64) {
      floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) v += *reinterpret_cast<const floatx4*>(osh + (w * 16 + ri) * LDO + d);
      if (only) {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        Quad<T> y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y.x[e] = from_float<T>(total == 0.f ? 0.f : v[e] * inv);
        *reinterpret_cast<Quad<T>*>(o + to * c.dh + d) = y;
      } else {
        *reinterpret_cast<floatx4*>(out.sums + ((int64_t)part * out.TH + to) * c.dh + d) = v;
        if (d == 0) {
          out.tops[2 * (part * out.TH + to)] = most;
          out.tops[2 * (part * out.TH + to) + 1] = total;
        }
      }
    }
  }
}

// The parts of every row (a head of a token) of several: ROWS rows a wave, or where there are few, one a workgroup, whose waves share its parts
// (SHARED).  Lane d has elements 2 d and 2 d + 1.  Bound by latency, of many rows by the parts' bytes: what a wave needs is asked for together.
template <typename T, int ROWS, bool SHARED>
__global__ __launch_bounds__(256) void attention_recent_join_kernel(PlanAny plan_, int B, int H, int G, int dh, WindowShape shape,
                                                                    RecentBuffers in, T* __restrict__ o) {
  static_assert(!SHARED || ROWS == 1, "a row a workgroup");
  __shared__ float shares[4][2 + 128];
  const PlanFirst plan = PlanFirst::of(plan_);
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t first = SHARED ? blockIdx.x : ((int64_t)blockIdx.x * 4 + wave) * ROWS;
  if (first >= in.TH) return;
  int parts[ROWS], most = 0;
  int token = (int)first / H, head = (int)first - token * H, of_key = head % G;   // TH is below 2^24
  int lo = 0;   // the query of the first row, then of the next
  {
    int hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.at(mid) <= token) lo = mid; else hi = mid;
    }
  }
  int known = -1, of_group = 0;   // a group of rows and its parts: rows side by side mostly are of one, and counting is a chain of divisions
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    parts[r] = 0;   // none, or written already
    if (first + r >= in.TH) continue;
    for (; plan.at(lo + 1) <= token; ++lo) known = -1;
    const int base = plan.at(lo), n = plan.at(lo + 1) - base, group = ((token - base) * G + of_key) >> __builtin_ctz(shape.rows);
    if (group != known) {
      of_group = shape.parts_of(shape.tiles(group, n, G, plan.at(2 * B + 1 + lo)));
      known = group;
    }
    if (of_group > 1) parts[r] = of_group;
    most = max(most, parts[r]);
    if (++of_key == G) of_key = 0;
    if (++head == H) {
      head = 0;
      ++token;
    }
  }
  if (SHARED && most == 0) return;   // workgroup-uniform
  const bool mine = 2 * lane < dh;
  constexpr int N = 8 / ROWS, STEP = SHARED ? 4 : 1;
  float2 acc[ROWS];
  float top[ROWS], total[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    acc[r] = float2{0.f, 0.f};
    top[r] = -INFINITY;
    total[r] = 0.f;
  }
  for (int p0 = SHARED ? wave : 0; p0 < most; p0 += N * STEP) {
    float2 t[ROWS][N], v[ROWS][N];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t p = (int64_t)max(min(p0 + i * STEP, parts[r] - 1), 0) * in.TH + min(first + r, in.TH - 1);   // of a row of none: read, and not used
        t[r][i] = *reinterpret_cast<const float2*>(in.tops + 2 * p);
        v[r][i] = *reinterpret_cast<const float2*>(in.sums + p * dh + (mine ? 2 * lane : 0));
      }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (p0 >= parts[r]) continue;   // wave-uniform
      float m = top[r];
#pragma unroll
      for (int i = 0; i < N; ++i) m = fmaxf(m, t[r][i].x);
      const float f = to_top(top[r], m);
      acc[r].x *= f; acc[r].y *= f; total[r] *= f;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (p0 + i * STEP < parts[r]) {   // wave-uniform; also where the factor is 0: NaN stays
          const float k = to_top(t[r][i].x, m);
          total[r] += k * t[r][i].y;
          acc[r].x += k * v[r][i].x;
          acc[r].y += k * v[r][i].y;
        }
      top[r] = m;
    }
  }
  if constexpr (SHARED) {   // in the order of the waves
    if (lane == 0) {
      shares[wave][0] = top[0];
      shares[wave][1] = total[0];
    }
    *reinterpret_cast<float2*>(&shares[wave][2 + 2 * lane]) = acc[0];
    __syncthreads();
    if (wave > 0) return;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, shares[w][0]);
    acc[0] = float2{0.f, 0.f};
    total[0] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float k = to_top(shares[w][0], m);
      total[0] += k * shares[w][1];
      acc[0].x += k * shares[w][2 + 2 * lane];
      acc[0].y += k * shares[w][3 + 2 * lane];
    }
  }
  if (!mine) return;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (parts[r] == 0) continue;
    const float inv = total[r] == 0.f ? 0.f : 1.f / total[r];
    struct alignas(2 * sizeof(T)) Pair { T x[2]; } y;
    y.x[0] = from_float<T>(total[r] == 0.f ? 0.f : acc[r].x * inv);
    y.x[1] = from_float<T>(total[r] == 0.f ? 0.f : acc[r].y * inv);
    *reinterpret_cast<Pair*>(o + (first + r) * dh + 2 * lane) = y;
  }
}

template <typename T, bool FOUR>
static hipError_t attention_recent(const Cache4Ref& c, const void* qkv, int H, const PlanAny& p, int B, int64_t wgs, const ScoreArgs& sc, const WindowShape& shape,
                                   const RecentBuffers& buf, void* o, hipStream_t s) {
  auto run = [&](auto steps, auto exact, auto r) {
    constexpr int STEPS = decltype(steps)::value;
    auto kern = attention_recent_kernel<T, FOUR, STEPS, decltype(exact)::value, decltype(r)::value>;
    kern<<<dim3((unsigned)wgs), dim3(256), recent_lds(STEPS), s>>>(p, c, (const T*)qkv, H, B, shape, sc, buf, (T*)o);
    return hipGetLastError();
  };
  auto by_rows = [&](auto steps, auto exact) {
    return shape.rows == 16 ? run(steps, exact, std::integral_constant<int, 1>{}) : run(steps, exact, std::integral_constant<int, 2>{});
  };
  auto by_width = [&](auto steps) { return c.dh == 32 * decltype(steps)::value ? by_rows(steps, std::true_type{}) : by_rows(steps, std::false_type{}); };
  switch ((c.dh + 31) / 32) {
    case 1: return by_width(std::integral_constant<int, 1>{});
    case 2: return by_width(std::integral_constant<int, 2>{});
    case 3: return by_width(std::integral_constant<int, 3>{});
    case 4: return by_width(std::integral_constant<int, 4>{});
  }
  return hipErrorInvalidValue;
}

hipError_t launch_attention_recent(int dtype, bool four, const Cache4Ref& c, const void* qkv, int H, const int32_t* plan, size_t count,
                                   const int32_t* d_plan, int B, int64_t T, const ScoreArgs& sc, const WindowShape& shape, float* workspace, void* o,
                                   hipStream_t s) {
  if (T <= 0) return hipSuccess;
  const int64_t TH = T * H;
  const int64_t wgs = shape.workgroups(plan, B, c.KV);
  // The join counts rows in 32 bits, and has no more workgroups than there are rows.
  if (wgs > kMostGroups || (shape.parts > 1 && TH > kMostGroups)) return kTooManyGroups;
  const PlanAny p = plan_any(plan, count, d_plan);
  const RecentBuffers buf{workspace + recent_sums_at(shape, TH), workspace, TH};
  hipError_t e;
  if (shape.rows == kManyRows)
    e = launch_attention_rows_bf16(four, c, qkv, H, plan, count, d_plan, B, sc, shape, buf, o, s);
  else if (dtype == 0)
    e = four ? attention_recent<float, true>(c, qkv, H, p, B, wgs, sc, shape, buf, o, s) : attention_recent<float, false>(c, qkv, H, p, B, wgs, sc, shape, buf, o, s);
  else
    e = four ? attention_recent<bf16_t, true>(c, qkv, H, p, B, wgs, sc, shape, buf, o, s) : attention_recent<bf16_t, false>(c, qkv, H, p, B, wgs, sc, shape, buf, o, s);
  if (e != hipSuccess || shape.parts <= 1) return e;
  auto join = [&](auto zero, auto rows, auto shared) {
    typedef decltype(zero) E;
    constexpr int ROWS = decltype(rows)::value;
    const int64_t groups = decltype(shared)::value ? TH : (TH + 4 * ROWS - 1) / (4 * ROWS);
    attention_recent_join_kernel<E, ROWS, decltype(shared)::value><<<dim3((unsigned)groups), dim3(256), 0, s>>>(p, B, H, H / c.KV, c.dh, shape, buf, (E*)o);
    return hipGetLastError();
  };
  // Four rows a wave where that still leaves a wave for every SIMD; a row's parts shared where one wave would take them in several turns.
  auto by_rows = [&](auto zero) {
    if (TH >= 4096) return join(zero, std::integral_constant<int, 4>{}, std::false_type{});
    return shape.parts > 8 ? join(zero, std::integral_constant<int, 1>{}, std::true_type{}) : join(zero, std::integral_constant<int, 1>{}, std::false_type{});
  };
  return dtype == 0 ? by_rows(0.f) : by_rows(bf16_t{});
}

}  // namespace otas
