// Walks the host side of the entry points of include/otas_decode.h with norms of heads, windows and the cache in 4 bits, with the HIP runtime and
// the kernel launchers stubbed out: every refusal, calls at the edges of what is accepted, and how calls are cut up.  Run under a sanitizer, see
// test_window_api.py.
#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime.h>
#ifndef __align__
#define __align__(n) __attribute__((aligned(n)))
#endif
#ifndef HIP_SYMBOL
#define HIP_SYMBOL(x) (&x)
#endif
#include <cmath>
#include "../paper_2401_05031_amd/csrc/api.hip"
#include "../paper_2401_05031_amd/csrc/window_api.hip"

extern "C" hipError_t hipMalloc(void** p, size_t n) { *p = std::calloc(1, n); return hipSuccess; }
extern "C" hipError_t hipHostMalloc(void** p, size_t n, unsigned) { *p = std::calloc(1, n); return hipSuccess; }
extern "C" hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
extern "C" hipError_t hipHostFree(void* p) { std::free(p); return hipSuccess; }
extern "C" hipError_t hipGetSymbolAddress(void** p, const void*) { static int32_t cell[64]; *p = cell; return hipSuccess; }
static bool capturing = false;
extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  *s = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}

#define CHECK(e) do { if (!(e)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #e); return 1; } } while (0)
#define IS(want, call) do { const otas_status got_ = (call); if (got_ != (want)) { std::fprintf(stderr, "line %d: %s -> %d\n", __LINE__, #call, (int)got_); return 1; } } while (0)

// Every tile that some row sees is among the tiles that its group of rows is given, once and in order, and the parts cover them.
static int shapes() {
  for (int G : {1, 3, 8})
    for (int n : {1, 5, 64, 300})
      for (int length : {1, 31, 32, 33, 700, 5000})
        for (int window : {1, 31, 64, 1000, INT32_MAX})
          for (int sinks : {0, 1, 32, 100, INT32_MAX})
            for (int dtype : {0, 1}) {
              if (n > length) continue;
              const int32_t off[] = {0, n}, len[] = {length};
              const WindowShape t = recent_shape(dtype, dtype == 1, 128, 4 * G, 4, off, len, 1, window, sinks);
              CHECK(t.room >= t.parts && t.parts >= 1 && t.groups == (n * G + t.rows - 1) / t.rows);
              for (int g = 0; g < t.groups; ++g) {
                const WindowTiles w = t.tiles(g, n, G, length);
                CHECK(w.count >= 1 && t.parts_of(w) <= t.parts);
                std::vector<char> have((length >> t.shift) + 1, 0);
                int before = -1;
                for (int i = 0; i < w.count; ++i) {
                  const int x = w.tile(i);
                  CHECK(x > before && x <= (length - 1) >> t.shift);
                  before = x;
                  have[x] = 1;
                }
                int next = 0;
                for (int p = 0; p < t.parts + 1; ++p) {
                  const int each = t.each_of(w), begin = p * each, end = std::min(w.count, begin + each);
                  if (p < t.parts_of(w)) {
                    CHECK(begin == next && end > begin && each <= t.each && each % t.at_once() == 0);
                    next = end;
                  } else {
                    CHECK(begin >= end);
                  }
                }
                CHECK(next == w.count);
                for (int r = g * t.rows; r < std::min((g + 1) * t.rows, n * G); ++r) {
                  const int place = length - n + r / G;
                  for (int j = 0; j <= place; ++j)
                    if (place - j < window || j < sinks) CHECK(have[j >> t.shift]);
                }
              }
              CHECK(recent_sums_at(t, n * 4 * G) % 4 == 0);
              CHECK(recent_workspace_floats(t, n * 4 * G, 128) <= recent_room_floats(t, n * 4 * G, 128));
            }
  // the workspace of long queries is enough for shorter ones
  uint32_t seed = 1;
  auto draw = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int)((uint64_t)(seed >> 8) * n >> 24); };
  for (int round = 0; round < 400; ++round) {
    const int B = 1 + draw(6), G = 1 << draw(4), KV = 1 + draw(8), dh = 8 * (1 + draw(16)), dtype = draw(2), window = draw(3) ? 1 + draw(3000) : INT32_MAX,
              sinks = draw(2) * draw(200);
    std::vector<int32_t> off{0}, before, after;
    for (int q = 0; q < B; ++q) {
      off.push_back(off.back() + draw(draw(2) ? 3 : 300));
      before.push_back(off[q + 1] - off[q] + draw(9000));
      after.push_back(before[q] + draw(draw(2) ? 40 : 30000));
    }
    for (bool four : {false, true}) {
      const WindowShape small = recent_shape(dtype, four, dh, G * KV, KV, off.data(), before.data(), B, window, sinks);
      const WindowShape large = recent_shape(dtype, four, dh, G * KV, KV, off.data(), after.data(), B, window, sinks);
      const int64_t TH = (int64_t)off[B] * G * KV;
      CHECK(recent_workspace_floats(small, TH, dh) <= recent_room_floats(small, TH, dh));
      CHECK(recent_room_floats(small, TH, dh) <= recent_room_floats(large, TH, dh));
    }
  }
  // every share of a call has a place of its own
  for (int groups : {1, 2, 7})
    for (int parts : {1, 3})
      for (int units : {1, 5, 16}) {
        WindowShape t{1, 0, 5, 16, groups, 1, parts, parts};
        std::vector<char> seen((size_t)units * groups * parts, 0);
        for (int id = 0; id < units * groups * parts; ++id) {
          const WorkPlace p = t.place(id, units);
          CHECK(p.unit >= 0 && p.unit < units && p.group >= 0 && p.group < groups && p.part >= 0 && p.part < parts);
          char& c = seen[((size_t)p.unit * groups + p.group) * parts + p.part];
          CHECK(!c);
          c = 1;
        }
      }
  // and of a call whose queries are counted one by one
  struct Plan {
    std::vector<int32_t> v;
    int at(int i) const { return v[i]; }
  };
  for (int G : {1, 4})
    for (int KV : {1, 3, 8})
      for (int parts : {1, 2}) {
        const int32_t off[] = {0, 0, 300, 301, 301, 301, 306, 500, 500};
        const int B = 8;
        WindowShape t{1, 0, 5, 32, (300 * G + 31) / 32, 1, parts, parts};
        Plan plan{std::vector<int32_t>(off, off + B + 1)};
        WindowShape none = t;
        none.count_groups(plan.v, off, B, G, 17, 1000);   // 18 numbers would not fit
        CHECK(none.firsts == 0 && plan.v.size() == 9 && none.workgroups(plan.v.data(), B, KV) == (int64_t)B * t.groups * KV * parts);
        t.count_groups(plan.v, off, B, G, 18, 18);
        CHECK(t.firsts == 9 && plan.v.size() == 18);
        std::vector<int> seen(B * KV * t.groups * parts, 0);
        const int64_t wgs = t.workgroups(plan.v.data(), B, KV);
        int64_t rows = 0;
        for (int q = 0; q < B; ++q) rows += ((off[q + 1] - off[q]) * G + 31) / 32;
        CHECK(wgs == rows * KV * parts);
        for (int id = 0; id < wgs; ++id) {
          const WorkPlace p = t.work(plan, id, B, KV);
          const int q = p.unit / KV;
          CHECK(p.unit >= 0 && q < B && p.group >= 0 && p.group * 32 < (off[q + 1] - off[q]) * G && p.part >= 0 && p.part < parts);
          CHECK(!seen[(p.unit * t.groups + p.group) * parts + p.part]++);
        }
        Plan even{{0, 300, 580, 870}};
        WindowShape same = t;
        same.firsts = 0;
        same.count_groups(even.v, even.v.data(), 3, G, 960, 2000);
        CHECK(same.firsts == 0 && even.v.size() == 4);
      }
  return 0;
}

int main() {
  if (shapes()) return 1;
  // addresses that no stub touches, far enough apart
  char* const base = (char*)(uintptr_t)(1ull << 40);
  void *qkv = base, *o = base + (1ull << 36), *ws = base + (2ull << 36), *gain = base + (8ull << 36);
  int32_t* pos = (int32_t*)(base + (3ull << 36));
  for (int dtype : {(int)OTAS_F32, (int)OTAS_BF16}) {
    const size_t e = dtype == OTAS_F32 ? 4 : 2;
    const otas_model_desc d = {1, 256, 4, 128, dtype, 1e-6f, 1};
    otas_layer_weights w;
    std::fill((const void**)&w, (const void**)(&w + 1), qkv);
    otas_ctx* c = nullptr;
    CHECK(otas_create(&c, &d, &w, nullptr) == OTAS_OK);

    const otas_rotary_desc r = {64, OTAS_ROTARY_HALF, OTAS_ROTARY_PLAIN, 0, 10000.0, 0.0, 0.0, 0.0, 0.0, 1.0};
    otas_rotary_desc none = r, odd = r;
    none.rot_dim = 0;
    odd.rot_dim = 3;
    const otas_head_norm_desc n = {gain, gain, 1e-6f, 0, 0};
    IS(OTAS_OK, otas_norm_rotary(c, qkv, 5, 2, &n, pos, &r, qkv));
    IS(OTAS_OK, otas_norm_rotary(c, qkv, 5, 2, &n, pos, &r, o));
    IS(OTAS_OK, otas_norm_rotary(c, qkv, 5, 2, &n, nullptr, &none, o));
    IS(OTAS_OK, otas_norm_rotary(c, nullptr, 0, 2, &n, nullptr, &r, nullptr));
    IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &n, nullptr, &r, o));
    IS(OTAS_EINVAL, otas_norm_rotary(nullptr, qkv, 5, 2, &n, pos, &r, o));
    IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, nullptr, pos, &r, o));
    IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &n, pos, nullptr, o));
    IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &n, pos, &odd, o));
    IS(OTAS_EINVAL, otas_norm_rotary(c, nullptr, 5, 2, &n, pos, &r, o));
    IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, -1, 2, &n, pos, &r, o));
    for (int kv : {0, -1, 3, 8}) IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, kv, &n, pos, &r, o));
    IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &n, pos, &r, (char*)qkv + 16));   // overlap
    IS(OTAS_EINVAL, otas_norm_rotary(c, (char*)qkv + 4, 5, 2, &n, pos, &r, o));      // alignment
    IS(OTAS_EUNSUPPORTED, otas_norm_rotary(c, qkv, 1ll << 31, 2, &n, pos, &r, qkv));
    for (float eps : {0.f, -1.f, (float)NAN, INFINITY}) {
      otas_head_norm_desc x = n;
      x.eps = eps;
      IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &x, pos, &r, o));
    }
    for (int which : {0, 1}) {
      otas_head_norm_desc x = n;
      const void*& g = which ? x.k_gain : x.q_gain;
      g = (char*)gain + 8;
      IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &x, pos, &r, o));
      g = (char*)o + 16;                                                            // within out
      IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &x, pos, &r, o));
      g = (char*)o - 64 * e;
      IS(OTAS_OK, otas_norm_rotary(c, qkv, 5, 2, &x, pos, &r, o));
      x.per_head = 1;                                                               // of all heads they reach into it
      IS(OTAS_EINVAL, otas_norm_rotary(c, qkv, 5, 2, &x, pos, &r, o));
      g = nullptr;
      IS(OTAS_OK, otas_norm_rotary(c, qkv, 5, 2, &x, pos, &r, o));
    }

    const int32_t off[] = {0, 3, 3, 8}, falling[] = {0, 3, 2}, shifted[] = {1, 3}, empty[] = {0, 0};
    const otas_score_desc s = {0.f, 0.f, nullptr}, nan = {NAN, 0.f, nullptr}, negative = {0.f, -1.f, nullptr};
    IS(OTAS_OK, otas_attention_window(c, qkv, 2, off, 3, 1, 0, &s, o));
    IS(OTAS_OK, otas_attention_window(c, qkv, 2, off, 3, INT32_MAX, INT32_MAX, nullptr, o));
    IS(OTAS_OK, otas_attention_window(c, nullptr, 2, empty, 1, 5, 0, nullptr, nullptr));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, off, 3, 0, 0, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, off, 3, -1, 0, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, off, 3, 1, -1, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, off, 0, 1, 0, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 3, off, 3, 1, 0, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, falling, 2, 1, 0, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, shifted, 1, 1, 0, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, off, 3, 1, 0, &nan, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, off, 3, 1, 0, &negative, o));
    IS(OTAS_EINVAL, otas_attention_window(c, qkv, 2, off, 3, 1, 0, &s, qkv));
    IS(OTAS_EINVAL, otas_attention_window(c, nullptr, 2, off, 3, 1, 0, &s, o));
    IS(OTAS_EINVAL, otas_attention_window(c, (char*)qkv + 8, 2, off, 3, 1, 0, &s, o));
    const int32_t longer[] = {0, OTAS_MAX_LONG_SEQ + 1}, longest[] = {0, OTAS_MAX_LONG_SEQ};
    IS(OTAS_EUNSUPPORTED, otas_attention_window(c, qkv, 2, longer, 1, 1, 0, nullptr, o));
    IS(OTAS_OK, otas_attention_window(c, qkv, 2, longest, 1, 1, 0, nullptr, o));

    // the last tokens of either cache
    const otas_kv_cache k = {base + (4ull << 36), base + (5ull << 36), pos, nullptr, 600, 2, 100};
    const otas_kv_cache4 f = {base + (4ull << 36), base + (5ull << 36), base + (6ull << 36), base + (7ull << 36), 600, 2, 128};
    const int32_t slot[] = {5, 0, 599}, len[] = {100, 0, 40}, twice[] = {5, 0, 5}, outside[] = {5, 0, 600}, shorter[] = {2, 0, 40}, over[] = {129, 0, 40}, under[] = {-1, 0, 40};
    const size_t need = otas_attention_recent_workspace_bytes(c, 2, off, len, 3, 50, 4);
    CHECK(need > 0 && need % 256 == 0);
    CHECK(otas_attention_recent_workspace_bytes(nullptr, 2, off, len, 3, 50, 4) == 0 && otas_attention_recent_workspace_bytes(c, 3, off, len, 3, 50, 4) == 0);
    CHECK(otas_attention_recent_workspace_bytes(c, 2, off, len, 3, 0, 4) == 0 && otas_attention_recent_workspace_bytes(c, 2, off, len, 3, 50, -1) == 0);
    CHECK(otas_attention_recent_workspace_bytes(c, 2, off, shorter, 3, 50, 4) == 0 && otas_attention_recent_workspace_bytes(c, 2, off, under, 3, 50, 4) == 0);
    auto either = [&](bool four, const void* in, const int32_t* of, const int32_t* sl, const int32_t* ln, int B, int window, int sinks, const otas_score_desc* sc, void* work,
                      size_t bytes, void* out) {
      return four ? otas_attention_cache4(c, &f, in, of, sl, ln, B, window, sinks, sc, work, bytes, out)
                  : otas_attention_recent(c, &k, in, of, sl, ln, B, window, sinks, sc, work, bytes, out);
    };
    for (bool four : {false, true}) {
      IS(OTAS_OK, either(four, qkv, off, slot, len, 3, 50, 4, &s, ws, need, o));
      IS(OTAS_OK, either(four, qkv, off, twice, len, 3, 50, 4, nullptr, ws, need, o));
      IS(OTAS_OK, either(four, nullptr, empty, slot, len, 1, 50, 4, nullptr, nullptr, 0, nullptr));
      IS(OTAS_EINVAL, either(four, qkv, off, outside, len, 3, 50, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, shorter, 3, 50, 4, &s, ws, need, o));   // three rows of two entries
      IS(OTAS_EINVAL, either(four, qkv, off, slot, over, 3, 50, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, under, 3, 50, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, nullptr, len, 3, 50, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 0, 50, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, falling, slot, len, 2, 50, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 0, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 50, -4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 50, 4, &nan, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 50, 4, &s, nullptr, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 50, 4, &s, (char*)ws + 16, need, o));
      IS(OTAS_EINVAL, either(four, (char*)qkv + 8, off, slot, len, 3, 50, 4, &s, ws, need, o));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 50, 4, &s, ws, need, qkv));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 50, 4, &s, ws, need, (char*)k.k + 256));
      IS(OTAS_EINVAL, either(four, qkv, off, slot, len, 3, 50, 4, &s, ws, need, (char*)k.v + 256));
    }
    IS(OTAS_EINVAL, otas_attention_cache4(c, &f, qkv, off, slot, len, 3, 50, 4, &s, ws, need, (char*)f.k_scales + 256));
    IS(OTAS_EINVAL, otas_attention_cache4(c, &f, (char*)f.v_scales + 256, off, slot, len, 3, 50, 4, &s, ws, need, o));
    {   // a call of several parts refuses less room than they take, and a workspace within the cache
      const otas_kv_cache4 deep = {f.k, f.v, f.k_scales, f.v_scales, 600, 2, 65536};
      const int32_t one[] = {0, 1}, far[] = {65536};
      const size_t bytes = otas_attention_recent_workspace_bytes(c, 2, one, far, 1, INT32_MAX, 0);
      CHECK(bytes > 4096);
      IS(OTAS_OK, otas_attention_cache4(c, &deep, qkv, one, slot, far, 1, INT32_MAX, 0, &s, ws, bytes, o));
      IS(OTAS_ENOMEM, otas_attention_cache4(c, &deep, qkv, one, slot, far, 1, INT32_MAX, 0, &s, ws, 64, o));
      IS(OTAS_EINVAL, otas_attention_cache4(c, &deep, qkv, one, slot, far, 1, INT32_MAX, 0, &s, deep.v_scales, bytes, o));
      IS(OTAS_EINVAL, otas_attention_cache4(c, &deep, qkv, one, slot, far, 1, INT32_MAX, 0, &s, o, bytes, o));
    }
    // a program that keeps one workspace asks for the longest lengths
    for (int B : {1, 5, 40})
      for (int rows : {1, 3, 70}) {
        std::vector<int32_t> of(B + 1), ls(B);
        for (int q = 0; q <= B; ++q) of[q] = rows * q;
        for (int window : {1, 100, 5000, INT32_MAX}) {
          size_t before = 0;
          for (int l = rows; l < 100000; l = l * 5 / 4 + 1) {
            std::fill(ls.begin(), ls.end(), l);
            const size_t b = otas_attention_recent_workspace_bytes(c, 2, of.data(), ls.data(), B, window, 7);
            CHECK(b >= before);
            before = b;
          }
        }
      }

    // the cache in 4 bits
    const int32_t rows[] = {7, 0, 7}, roff[] = {0, 0, 2, 3}, roff2[] = {0, 29, 31, 32}, full[] = {128, 0, 40};
    int32_t out[600];
    IS(OTAS_OK, otas_cache4_append(c, &f, qkv, 8, roff, rows, slot, len, 3, out));
    CHECK(out[0] == 100 && out[1] == 2 && out[2] == 41);
    IS(OTAS_OK, otas_cache4_append(c, &f, qkv, 8, roff, nullptr, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 7, roff, rows, slot, len, 3, out));        // row 7 of 7
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 2, roff, nullptr, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 40, roff2, nullptr, slot, len, 3, out));   // 29 rows behind 100 of 128
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 8, roff, rows, twice, len, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 8, roff, rows, outside, len, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 8, roff, rows, slot, over, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 8, roff, rows, slot, under, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, nullptr, qkv, 8, roff, rows, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, nullptr, 8, roff, rows, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache4_append(c, &f, qkv, 8, roff, rows, slot, len, 3, nullptr));
    IS(OTAS_OK, otas_cache4_read(c, &f, slot, len, roff, 3, o));
    IS(OTAS_OK, otas_cache4_read(c, &f, twice, len, roff, 3, o));
    IS(OTAS_OK, otas_cache4_read(c, &f, slot, full, roff, 3, o));
    IS(OTAS_OK, otas_cache4_read(c, &f, slot, len, empty, 1, nullptr));
    IS(OTAS_EINVAL, otas_cache4_read(c, &f, slot, len, roff2, 3, o));
    IS(OTAS_EINVAL, otas_cache4_read(c, &f, outside, len, roff, 3, o));
    IS(OTAS_EINVAL, otas_cache4_read(c, &f, slot, under, roff, 3, o));
    IS(OTAS_EINVAL, otas_cache4_read(c, &f, slot, len, roff, 3, nullptr));
    IS(OTAS_EINVAL, otas_cache4_read(c, &f, slot, len, roff, 3, (char*)o + 8));
    IS(OTAS_EINVAL, otas_cache4_read(c, nullptr, slot, len, roff, 3, o));
    auto but = [&](auto change) { otas_kv_cache4 x = f; change(x); return x; };
    const otas_kv_cache4 wrong[] = {but([](auto& x) { x.kv_heads = 3; }), but([](auto& x) { x.slots = 0; }), but([](auto& x) { x.capacity = 0; }),
                                    but([](auto& x) { x.capacity = 100; }), but([](auto& x) { x.v = (char*)x.v + 8; }), but([](auto& x) { x.k_scales = nullptr; }),
                                    but([](auto& x) { x.v_scales = (char*)x.v_scales + 4; }), but([](auto& x) { x.v = x.k; }), but([](auto& x) { x.v_scales = x.k_scales; }),
                                    but([](auto& x) { x.k_scales = (char*)x.k + 4096; })};
    for (const otas_kv_cache4& x : wrong) {
      IS(OTAS_EINVAL, otas_cache4_append(c, &x, qkv, 8, roff, rows, slot, len, 3, out));
      IS(OTAS_EINVAL, otas_cache4_read(c, &x, slot, len, roff, 3, o));
      IS(OTAS_EINVAL, otas_attention_cache4(c, &x, qkv, off, slot, len, 3, 50, 4, &s, ws, need, o));
    }
    const otas_kv_cache4 huge = but([](auto& x) { x.capacity = OTAS_MAX_LONG_SEQ + 32; });
    IS(OTAS_EUNSUPPORTED, otas_cache4_append(c, &huge, qkv, 8, roff, rows, slot, len, 3, out));
    const size_t codes = (size_t)600 * 2 * 128 * 32, scales = (size_t)600 * 2 * 128 * 2;
    for (char* in : {(char*)f.k, (char*)f.v}) {
      IS(OTAS_EINVAL, otas_cache4_append(c, &f, in + codes - 256, 8, roff, rows, slot, len, 3, out));
      IS(OTAS_OK, otas_cache4_append(c, &f, in + codes, 8, roff, rows, slot, len, 3, out));
      IS(OTAS_EINVAL, otas_cache4_read(c, &f, slot, len, roff, 3, in));
    }
    for (char* in : {(char*)f.k_scales, (char*)f.v_scales}) {
      IS(OTAS_EINVAL, otas_cache4_append(c, &f, in + scales - 256, 8, roff, rows, slot, len, 3, out));
      IS(OTAS_OK, otas_cache4_read(c, &f, slot, len, roff, 3, in + scales));
    }
    {   // widths that are no multiple of 8
      const otas_model_desc d20 = {1, 160, 8, 128, dtype, 1e-6f, 1};
      otas_ctx* n20 = nullptr;
      if (otas_create(&n20, &d20, &w, nullptr) == OTAS_OK) {
        IS(OTAS_EUNSUPPORTED, otas_cache4_append(n20, &f, qkv, 8, roff, rows, slot, len, 3, out));
        IS(OTAS_EUNSUPPORTED, otas_cache4_read(n20, &f, slot, len, roff, 3, o));
        IS(OTAS_EUNSUPPORTED, otas_attention_recent(n20, &k, qkv, off, slot, len, 3, 50, 4, &s, ws, (size_t)1 << 30, o));
        CHECK(otas_destroy(n20) == OTAS_OK);
      }
    }

    // host numbers that do not fit the arguments: uploaded, refused while the stream is captured
    std::vector<int32_t> many(500), zero(500, 0), ten(500, 10), offs(501);
    for (int q = 0; q < 500; ++q) { many[q] = 599 - q; offs[q + 1] = q + 1; }
    std::vector<int32_t> wide(1001);
    for (int q = 0; q <= 1000; ++q) wide[q] = q;
    for (bool cap : {false, true}) {
      capturing = cap;
      const otas_status want = cap ? OTAS_EUNSUPPORTED : OTAS_OK;
      IS(want, otas_cache4_append(c, &f, qkv, 500, offs.data(), nullptr, many.data(), zero.data(), 500, out));
      IS(want, otas_cache4_read(c, &f, many.data(), zero.data(), offs.data(), 500, o));
      IS(want, otas_attention_window(c, qkv, 2, wide.data(), 1000, 5, 1, nullptr, o));
      for (bool four : {false, true}) IS(want, either(four, qkv, offs.data(), many.data(), ten.data(), 500, 5, 1, nullptr, ws, (size_t)1 << 30, o));
      IS(OTAS_OK, otas_norm_rotary(c, qkv, 500, 2, &n, pos, &r, o));
    }
    capturing = false;
    CHECK(otas_destroy(c) == OTAS_OK);
  }
  std::puts("window api ok");
  return 0;
}
