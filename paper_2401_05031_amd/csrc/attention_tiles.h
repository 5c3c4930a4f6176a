// bf16 attention over tiles of keys that travel from global memory straight into LDS: what the masked and the tree kernels
// share.  A wave owns 32 rows; both products are formed transposed (as in attention.hip),
//   S^T[key, row] = K Q^T,   O^T[d, row] += V^T P^T    (v_mfma_f32_32x32x16_bf16)
// so that lane (row = lane & 31, half = lane >> 5) holds, of 32 keys, the keys 8 (e / 4) + 4 half + (e & 3), e = 0 .. 15: maxima
// and sums are over its own registers and one exchange with the other half, and the weights feed the second product as they lie.
#pragma once
#include "attention_decode.h"

namespace otas {

#define OTAS_GLOBAL(p) ((const __attribute__((address_space(1))) void*)(p))
#define OTAS_LDS(p) ((__attribute__((address_space(3))) void*)(p))
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));

// This wave's loads have landed and its LDS reads are back.
__device__ __forceinline__ void wait_all() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(7 << 4);   // vmcnt(0) lgkmcnt(0)
  asm volatile("" ::: "memory");
}
// LDS reads are back and writes done, of every wave of the workgroup; loads may be under way.
__device__ __forceinline__ void wait_lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xF | (7 << 4) | (3 << 14));   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Where the 16-byte pieces of a tile's rows lie.  A load instruction fills 64 consecutive pieces of LDS, so that no padding comes
// for free; in its place pieces change places within a row by a rule on the row.  Keys are read 16 bytes a lane from 16 rows at
// a time, values 8 bytes a lane by the transposing read, 4 rows x 64 bytes per 32 lanes: the rules put either on all 64 banks
// once.  Rows of 80 and 96 elements take 12 pieces, turned by a place every four rows.
template <int DH> struct TileRows {
  static constexpr int PIECES = DH / 8;
  static constexpr int STRIDE = DH % 64 == 0 ? PIECES : 12;   // pieces from row to row
  static_assert(PIECES <= STRIDE, "widths of 64, 80, 96 and 128");
  static constexpr int ROW_BYTES = STRIDE * 16;
  static constexpr size_t bytes(int rows) { return (size_t)rows * ROW_BYTES; }
  static __device__ __forceinline__ int turned(int row, int c) { const int p = c + ((row >> 2) & 3); return p >= 12 ? p - 12 : p; }
  static __device__ __forceinline__ int unturned(int row, int p) { const int c = p - ((row >> 2) & 3); return c < 0 ? c + 12 : c; }
  static __device__ __forceinline__ int key_piece(int row, int c) { return DH == 128 ? c ^ (row & 15) : DH == 64 ? c ^ ((row >> 1) & 7) : turned(row, c); }
  static __device__ __forceinline__ int value_piece(int row, int c) { return DH == 128 ? c ^ 4 * (row & 3) : DH == 64 ? c ^ 4 * ((row >> 1) & 1) : turned(row, c); }
  // the piece of a row that lies at place p
  static __device__ __forceinline__ int key_at(int row, int p) { return DH % 64 == 0 ? key_piece(row, p) : unturned(row, p); }
  static __device__ __forceinline__ int value_at(int row, int p) { return DH % 64 == 0 ? value_piece(row, p) : unturned(row, p); }
};

// LDS is read and written through restricted pointers below: unless the compiler can tell that a read is not of a place that a load
// straight into LDS is still on its way to, it waits for all such loads before the read, the next tile's among them.
__device__ __forceinline__ int4 read_four(const int* __restrict__ p, int i) { return *reinterpret_cast<const int4*>(p + 4 * i); }

// Values that are not finite, in a tile of which some row does not see some key: a weight of 0 would not keep them out of that
// row.  They become 0 in LDS, and those that some row sees are added at the end (add_not_finite).  Here one 16-byte piece: whether
// it had any.
__device__ __forceinline__ bool piece_make_finite(char* __restrict__ at) {
  uint4 u = *reinterpret_cast<const uint4*>(at);
  uint32_t* x = &u.x;
  uint32_t odd[4];   // ones over the elements whose exponent is all ones, two at a time
#pragma unroll
  for (int k = 0; k < 4; ++k) odd[k] = ((((x[k] & 0x7F807F80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xFFFFu;
  if (!(odd[0] | odd[1] | odd[2] | odd[3])) return false;
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] &= ~odd[k];
  *reinterpret_cast<uint4*>(at) = u;
  return true;
}

// Loads of one wave's share (WAVES waves share the work) of ROWS rows of keys (VALUES: of values) into LDS.  The same lane loads
// the same piece of every tile: its place within the row is formed once.
template <int DH, int ROWS, int WAVES, bool VALUES> struct TileLoader {
  typedef TileRows<DH> R;
  static constexpr int TOTAL = ROWS * R::STRIDE / 64;                  // load instructions a tile
  static constexpr int OWN = (TOTAL + WAVES - 1) / WAVES;
  static_assert(ROWS * R::STRIDE % 64 == 0, "whole instructions");
  // Where a row's pieces are a power of two, a lane's share of every instruction is the same piece of a row STEP further on.
  static constexpr bool EVEN = DH % 64 == 0;
  static constexpr int PLACES = EVEN ? 1 : OWN, STEP = EVEN ? 64 * WAVES / R::STRIDE : 0;
  int row[PLACES];
  uint32_t col[PLACES];   // bytes within the row
  int wave;
  __device__ __forceinline__ void begin(int wave_, int lane) {
    wave = VALUES ? WAVES - 1 - wave_ : wave_;   // where the instructions do not divide, the waves with one fewer of keys have one more of values
#pragma unroll
    for (int i = 0; i < PLACES; ++i) {
      const int at = (wave + i * WAVES) * 64 + lane, r = at / R::STRIDE, p = at - r * R::STRIDE;
      row[i] = r;
      col[i] = (uint32_t)min(VALUES ? R::value_at(r, p) : R::key_at(r, p), R::PIECES - 1) * 16u;
    }
  }
  // from: the tile's first row; ld: bytes from row to row; last: the last row that may be read (later ones repeat it).  All but
  // the lanes' places are the wave's: a tile that is all there costs an addition or two per instruction.
  __device__ __forceinline__ void load(const char* from, uint32_t ld, int last, char* lds) const {
    if (last >= ROWS - 1) {
#pragma unroll
      for (int i = 0; i < OWN; ++i)
        if (TOTAL % WAVES == 0 || wave + i * WAVES < TOTAL) {
          const size_t step = (size_t)(EVEN ? i * STEP : 0) * ld;
          one(from + step, __umul24((uint32_t)row[EVEN ? 0 : i], ld) + col[EVEN ? 0 : i], lds + (wave + i * WAVES) * 1024);
        }
    } else {
#pragma unroll
      for (int i = 0; i < OWN; ++i)
        if (TOTAL % WAVES == 0 || wave + i * WAVES < TOTAL)
          one(from, __umul24((uint32_t)min(EVEN ? row[0] + i * STEP : row[EVEN ? 0 : i], last), ld) + col[EVEN ? 0 : i], lds + (wave + i * WAVES) * 1024);
    }
  }
  // Of the pieces that this lane loaded, once they are there (no other wave need have waited); whether harmful(row) of the tile
  // holds for one that had values to be taken out.
  template <class F> __device__ __forceinline__ bool make_finite(char* __restrict__ lds, int lane, F harmful) const {
    bool met = false;
#pragma unroll
    for (int i = 0; i < OWN; ++i)
      if (TOTAL % WAVES == 0 || wave + i * WAVES < TOTAL) {
        const int c = (wave + i * WAVES) * 64 + lane;
        if (piece_make_finite(lds + c * 16)) met |= harmful(c / R::STRIDE);
      }
    return met;
  }
  // 0 in the place of those from row `valid` of the tile on.
  __device__ __forceinline__ void zero_rows(char* __restrict__ lds, int lane, int valid) const {
#pragma unroll
    for (int i = 0; i < OWN; ++i)
      if (TOTAL % WAVES == 0 || wave + i * WAVES < TOTAL) {
        const int c = (wave + i * WAVES) * 64 + lane;
        if (c >= valid * R::STRIDE) *reinterpret_cast<uint4*>(lds + c * 16) = uint4{0, 0, 0, 0};
      }
  }
  static __device__ __forceinline__ void one(const char* __restrict__ from, uint32_t at, char* __restrict__ lds) {
    __builtin_amdgcn_global_load_lds(OTAS_GLOBAL(from + at), OTAS_LDS(lds), 16, 0, 0);
  }
};

template <int DH> struct WaveRows {   // a wave's 32 rows
  static constexpr int KS = DH / 16, DT = (DH + 31) / 32;
  bf16x8 q[KS];
  floatx16 o[DT];
  float m, l;   // the largest logit that the sums are relative to, in units of ln 2; the weights' sum over the lane's keys
  __device__ __forceinline__ void begin(const bf16_t* qrow, int fk, bool negative) {   // negative: of a negative scale, whose size alone is applied later
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint4 u = *reinterpret_cast<const uint4*>(qrow + ks * 16 + fk * 8);
      if (negative) { u.x ^= 0x80008000u; u.y ^= 0x80008000u; u.z ^= 0x80008000u; u.w ^= 0x80008000u; }
      __builtin_memcpy(&q[ks], &u, 16);
    }
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
};

// Products of the rows with NB blocks of 32 keys of the tile, from block b0 on.  The keys of a block are read while the products of
// the one before it run (left alone the compiler reads each piece just before its product, and waits for it there).  beneath(i): other work,
// behind product i.
struct NoWork { __device__ __forceinline__ void operator()(int) const {} };
template <int DH, int NB, class F = NoWork>
__device__ __forceinline__ void tile_products(floatx16 (&s)[NB], const WaveRows<DH>& w, const char* __restrict__ lds_k, int b0, int fr, int fk, F beneath = F()) {
  typedef TileRows<DH> R;
  constexpr int KS = WaveRows<DH>::KS;
  auto piece = [&](int b, int ks) {   // 32 b does not change the rule
    return *reinterpret_cast<const bf16x8*>(lds_k + ((b0 + b) * 32 + fr) * R::ROW_BYTES + R::key_piece(fr, 2 * ks + fk) * 16);
  };
  bf16x8 kf[2][KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kf[0][ks] = piece(0, ks);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[b][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[b & 1][ks], w.q[ks], s[b], 0, 0, 0);
      if (b + 1 < NB) kf[(b + 1) & 1][ks] = piece(b + 1, ks);
      beneath(b * KS + ks);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// V^T fragment of columns 32 t .. 32 t + 31 and keys 16 kk .. 16 kk + 15 of the tile (transposing reads: in every 16 lanes lane
// s points at V[k0 + s / 4][4 (s & 3) ..] and lane i receives V[k0 .. k0 + 3][i]).
template <int DH>
__device__ __forceinline__ short8_t tile_values(const char* __restrict__ lds_v, int kk, int t, int lane) {
  typedef TileRows<DH> R;
  const int s16 = lane & 15, row = 4 * (lane >> 5) + (s16 >> 2), c = t * 4 + ((lane >> 4) & 1) * 2 + ((s16 & 3) >> 1);
  const char* p = lds_v + (kk * 16 + row) * R::ROW_BYTES + (s16 & 1) * 8;   // 16 rows: the rules' period
  const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(p + R::value_piece(row, c) * 16));
  const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)(p + 8 * R::ROW_BYTES + R::value_piece(row + 8, c) * 16));
  return short8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}
template <int DH> constexpr int value_slack() { return 64; }   // bytes that the last columns' reads of the last row may run past a tile

__device__ __forceinline__ bf16x8 as_bf16(short8_t v) {
  bf16x8 f;
  __builtin_memcpy(&f, &v, 16);
  return f;
}
// The tile's first values, read ahead of the exponentials that come before their products.
template <int DH>
__device__ __forceinline__ void first_values(short8_t (&v)[WaveRows<DH>::DT], const char* lds_v, int kk0, int lane) {
#pragma unroll
  for (int t = 0; t < WaveRows<DH>::DT; ++t) v[t] = tile_values<DH>(lds_v, kk0, t, lane);
  __builtin_amdgcn_sched_barrier(0);
}

// o += V^T P^T over NB blocks of 32 keys; s holds the weights, v the first 16 keys' values; the next 16 keys' are read beneath the
// products.  The weights are rounded to bf16 for the product: 2^-8 of each at most, as much as the output's own rounding; their
// sum l takes them unrounded.
template <int DH, int NB>
__device__ __forceinline__ void tile_sums(WaveRows<DH>& w, const floatx16 (&s)[NB], short8_t (&v)[WaveRows<DH>::DT], const char* lds_v, int kk0, int lane) {
  constexpr int DT = WaveRows<DH>::DT;
  short8_t u[DT];
#pragma unroll
  for (int kk = 0; kk < 2 * NB; ++kk) {
    bf16x8 pf;
#pragma unroll
    for (int i = 0; i < 8; ++i) pf[i] = (bf16_t)s[kk >> 1][8 * (kk & 1) + i];
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      w.o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(kk & 1 ? u[t] : v[t]), pf, w.o[t], 0, 0, 0);
      if (kk + 1 < 2 * NB) (kk & 1 ? v[t] : u[t]) = tile_values<DH>(lds_v, kk0 + kk + 1, t, lane);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// Whether any lane of the workgroup's four waves says so; flags: 16 bytes of LDS of its own.
__device__ __forceinline__ bool any_wave(bool mine, int* flags, int wave, int lane) {
  const bool any = __any(mine);
  if (lane == 0) flags[wave] = any;
  wait_lds_barrier();
  return (flags[0] | flags[1] | flags[2] | flags[3]) != 0;
}

// Four consecutive values v of a key that the lane's row sees: what of them is not finite, added to its sums.
__device__ __forceinline__ void add_not_finite(floatx16& o, int g, const bf16_t* v, bool sees) {
  const Quad<bf16_t> x = *reinterpret_cast<const Quad<bf16_t>*>(v);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float f = (float)x.x[e];
    o[4 * g + e] += sees && !__builtin_isfinite(f) ? f : 0.f;
  }
}

// Scores in units of ln 2: exp(s - m) is then one v_exp_f32.
struct Score2 {
  float scale2;    // scale log2 e; with a cap the factor of the exponent below
  float cap2;      // cap log2 e
  float slope2;    // the row's
  int position;    // the row's
  static __device__ __forceinline__ Score2 of(const ScoreArgs& sc, float slope, int position) {
    constexpr float log2e = 1.44269504088896340736f;
    const float scale = fabsf(sc.scale);   // the sign is in the rows
    return Score2{sc.cap > 0.f ? 2.f * log2e * (scale / sc.cap) : scale * log2e, sc.cap * log2e, slope * log2e, position};
  }
  // cap tanh(x), x = s scale / cap, as cap - 2 cap / (1 + exp(2 x)): off by 3e-7 cap at most, near zero, where the two cancel.  CAP 2 (caps past
  // kFarCap, where that would be more than 8e-5 of a logit, however small the logit): x - x^3 / 3 + 2 x^5 / 15 up to 3 / 32 (4e-8 of it
  // off) and 1 - 2 / (1 + exp(2 x)) beyond (4e-6 of it off).
  template <int CAP> __device__ __forceinline__ float capped(float s) const {
    const float t = s * scale2, r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t));
    if (CAP == 1) return fmaf(-2.f * cap2, r, cap2);
    constexpr float h = 0.34657359028f;   // ln 2 / 2: x = h t
    const float y = t * t, near = h * t * fmaf(fmaf(2.f / 15 * h * h * h * h, y, -h * h / 3), y, 1.f);
    return cap2 * (fabsf(t) <= kSeries / h ? near : fmaf(-2.f, r, 1.f));
  }
  static constexpr float kFarCap = 256.f, kSeries = 3.f / 32;
  static int cap_form(float cap) { return cap > kFarCap ? 2 : cap > 0.f ? 1 : 0; }   // the kernels' CAP
};

// cap tanh(s scale / cap) for products that stay below three eighths of the cap, as they mostly do: an odd polynomial of degree 5
// (least squares on a fine grid, re-weighted until the error is flat: 8e-7 of the cap) takes three full-rate instructions and no
// more for the exponent, where exponential and reciprocal are two at quarter rate and four more; the vector ALU is what these
// kernels keep busiest.  Past kFarCap the series, whose error goes with the logit, up to 3 / 32 of the cap: logits of 24 and more.
// limit < 0: scale / cap is too large for its powers; 2^24 at most, where none of them is too small.
struct CapArgs {
  float a0, a1, a2, limit;   // logits in units of ln 2 = s (a0 + a1 s^2 + a2 s^4) while |s| <= limit
  static CapArgs of(const ScoreArgs& sc) {
    CapArgs r = {0.f, 0.f, 0.f, -1.f};
    if (!(sc.cap > 0.f)) return r;
    const double x = fabs((double)sc.scale) / sc.cap, k = sc.cap * 1.4426950408889634 * x;
    const bool far = Score2::cap_form(sc.cap) == 2;
    const double c0 = far ? 1.0 : 0.9999854, c1 = far ? -1.0 / 3 : -0.33248851, c2 = far ? 2.0 / 15 : 0.120988494;
    if (x > 65536.0 || c2 * k * x * x * x * x > 1e38) return r;
    r.a0 = (float)(c0 * k);
    r.a1 = (float)(c1 * k * x * x);
    r.a2 = (float)(c2 * k * x * x * x * x);
    r.limit = (float)std::min((far ? (double)Score2::kSeries : 0.375) / x, 16777216.0);
    return r;
  }
  __device__ __forceinline__ float slope(float s) const {   // logit / s
    const float y = s * s;
    return fmaf(fmaf(a2, y, a1), y, a0);
  }
};

// Products into capped logits, in units of ln 2, where slopes or masks come between them and the weights: by the polynomial if all
// of the wave's are small enough, those of keys that no row sees among them where the caller has not taken them out.
template <int CAP, int NB> __device__ __forceinline__ void tile_capped(floatx16 (&s)[NB], const Score2& score, const CapArgs& cap) {
  float most = 0.f;   // NaN is passed over here and stays one in either form
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int e = 0; e < 16; e += 2) most = fmaxf(fmaxf(most, fabsf(s[b][e])), fabsf(s[b][e + 1]));
  if (__all(most <= cap.limit)) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[b][e] *= cap.slope(s[b][e]);
  } else {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[b][e] = score.capped<CAP>(s[b][e]);
  }
}

// The sums are rescaled only when a maximum has grown by more than 8 (a weight may be up to 2^8 then: no accuracy is lost in a
// floating format; of its range 2^8 is, so that 2^20 values of 1e30, what the header takes, still have a sum).
template <int DH>
__device__ __forceinline__ void raise_top(WaveRows<DH>& w, float mx) {
  if (__any(mx > w.m + 8.f)) {
    const float m_new = fmaxf(w.m, mx);
    const float alpha = w.m == m_new ? 1.f : __builtin_amdgcn_exp2f(w.m - m_new);   // equal: also where both are -inf
    w.m = m_new;
    w.l *= alpha;
#pragma unroll
    for (int t = 0; t < WaveRows<DH>::DT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) w.o[t][e] *= alpha;
  }
}

// Products of a tile that every row sees all of into weights, if they are small enough for the polynomial (wave-uniform; else nothing
// is done).  tanh grows with its argument: the largest product gives the largest logit.
template <int DH, int NB>
__device__ __forceinline__ bool tile_weights_capped(WaveRows<DH>& w, floatx16 (&s)[NB], const CapArgs& cap) {
  float hi = -INFINITY, lo = INFINITY;   // NaN is passed over here and stays one in either form
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      hi = fmaxf(fmaxf(hi, s[b][e]), s[b][e + 1]);
      lo = fminf(fminf(lo, s[b][e]), s[b][e + 1]);
    }
  if (!__all(fmaxf(hi, -lo) <= cap.limit)) return false;
  hi = xor32_max(hi);
  raise_top<DH>(w, hi * cap.slope(hi));
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], cap.slope(s[b][e]), -w.m));
      w.l += s[b][e];
    }
  return true;
}

// The tile's logits (times a positive factor; -inf where not seen) into weights, the running maximum and sum moved on.
template <int DH, int NB>
__device__ __forceinline__ void tile_weights(WaveRows<DH>& w, floatx16 (&s)[NB], float factor) {
  float mx = -INFINITY;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int e = 0; e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[b][e]), s[b][e + 1]);
  raise_top<DH>(w, xor32_max(mx) * factor);
  const float m = w.m == -INFINITY ? 0.f : w.m;   // nothing seen so far: all weights are 0
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], factor, -m));
      w.l += s[b][e];
    }
}

}  // namespace otas
