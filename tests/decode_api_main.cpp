// Walks the host side of the decoder's C ABI (include/otas_decode.h) with the HIP runtime and the kernel launchers stubbed out: every
// refusal, and calls at the edges of what is accepted.  Run under a sanitizer, see test_decode_api.py.
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
#include "../paper_2401_05031_amd/csrc/decode_api.hip"

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

int main() {
  // addresses that no stub touches, far enough apart
  char* const base = (char*)(uintptr_t)(1ull << 40);
  void *qkv = base, *o = base + (1ull << 36), *ws = base + (2ull << 36);
  int32_t* pos = (int32_t*)(base + (3ull << 36));
  for (int dtype : {(int)OTAS_F32, (int)OTAS_BF16}) {
    const otas_model_desc d = {1, 256, 4, 128, dtype, 1e-6f, 1};
    otas_layer_weights w;
    std::fill((const void**)&w, (const void**)(&w + 1), qkv);
    otas_ctx* c = nullptr;
    CHECK(otas_create(&c, &d, &w, nullptr) == OTAS_OK);

    otas_rotary_desc r = {64, OTAS_ROTARY_HALF, OTAS_ROTARY_PLAIN, 0, 10000.0, 0.0, 0.0, 0.0, 0.0, 1.0};
    IS(OTAS_OK, otas_rotary(c, qkv, 5, 2, pos, &r, qkv));
    IS(OTAS_OK, otas_rotary(c, qkv, 5, 2, pos, &r, o));
    IS(OTAS_OK, otas_rotary(c, qkv, 0, 2, pos, &r, o));
    IS(OTAS_EINVAL, otas_rotary(nullptr, qkv, 5, 2, pos, &r, o));
    IS(OTAS_EINVAL, otas_rotary(c, nullptr, 5, 2, pos, &r, o));
    IS(OTAS_EINVAL, otas_rotary(c, qkv, 5, 2, nullptr, &r, o));
    IS(OTAS_EINVAL, otas_rotary(c, qkv, 5, 2, pos, nullptr, o));
    IS(OTAS_EINVAL, otas_rotary(c, qkv, 5, 2, pos, &r, nullptr));
    IS(OTAS_EINVAL, otas_rotary(c, qkv, -1, 2, pos, &r, o));
    for (int kv : {0, -1, 3, 5, 8}) IS(OTAS_EINVAL, otas_rotary(c, qkv, 5, kv, pos, &r, o));
    IS(OTAS_EINVAL, otas_rotary(c, qkv, 5, 2, pos, &r, (char*)qkv + 16));      // overlap
    IS(OTAS_EINVAL, otas_rotary(c, (char*)qkv + 4, 5, 2, pos, &r, o));         // alignment
    IS(OTAS_EINVAL, otas_rotary(c, qkv, 5, 2, (int32_t*)((char*)pos + 2), &r, o));
    IS(OTAS_EUNSUPPORTED, otas_rotary(c, qkv, 1ll << 31, 2, pos, &r, qkv));
    auto bad = [&](auto change) {
      otas_rotary_desc x = r;
      change(x);
      return otas_rotary(c, qkv, 5, 2, pos, &x, o);
    };
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.rot_dim = 63; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.rot_dim = 66; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.rot_dim = -2; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.layout = 2; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.scaling = 4; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.base = 0.0; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.base = NAN; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.magnitude = 0.0; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.magnitude = 1e300; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.scaling = OTAS_ROTARY_LINEAR; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.scaling = OTAS_ROTARY_BASE; x.factor = 2.0; x.rot_dim = 2; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.scaling = OTAS_ROTARY_BY_PARTS; x.factor = 2.0; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.scaling = OTAS_ROTARY_BY_PARTS; x.factor = 2.0; x.original_length = 100.0; x.fast_turns = x.slow_turns = 1.0; }));
    IS(OTAS_EINVAL, bad([](otas_rotary_desc& x) { x.base = 1e-308; x.rot_dim = 64; x.scaling = OTAS_ROTARY_BASE; x.factor = 1e-300; }));
    IS(OTAS_OK, bad([](otas_rotary_desc& x) { x.scaling = OTAS_ROTARY_BY_PARTS; x.factor = 2.0; x.original_length = 100.0; x.fast_turns = 8.0; x.slow_turns = 1.0; }));
    IS(OTAS_OK, bad([](otas_rotary_desc& x) { x.rot_dim = 0; }));

    const int32_t off[] = {0, 3, 3, 8}, pre[] = {3, 0, 1};
    otas_score_desc s = {0.f, 0.f, nullptr};
    IS(OTAS_OK, otas_attention_masked(c, qkv, 2, off, 3, 1, pre, pos, pos, &s, o));
    IS(OTAS_OK, otas_attention_masked(c, qkv, 2, off, 3, 1, nullptr, nullptr, nullptr, nullptr, o));
    const int32_t none[] = {0, 0};
    IS(OTAS_OK, otas_attention_masked(c, qkv, 2, none, 1, 1, nullptr, nullptr, nullptr, nullptr, o));
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, off, 0, 1, nullptr, nullptr, nullptr, nullptr, o));
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 3, off, 3, 1, nullptr, nullptr, nullptr, nullptr, o));
    const int32_t falling[] = {0, 3, 2}, shifted[] = {1, 3}, pre2[] = {4, 0, 0}, pre3[] = {0, -1, 0};
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, falling, 2, 1, nullptr, nullptr, nullptr, nullptr, o));
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, shifted, 1, 1, nullptr, nullptr, nullptr, nullptr, o));
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, off, 3, 1, pre2, nullptr, nullptr, nullptr, o));
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, off, 3, 1, pre3, nullptr, nullptr, nullptr, o));
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, off, 3, 1, nullptr, nullptr, nullptr, nullptr, qkv));
    for (float v : {(float)NAN, INFINITY, -1.f}) {
      otas_score_desc t = {0.f, v, nullptr};
      IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, off, 3, 1, nullptr, nullptr, nullptr, &t, o));
    }
    otas_score_desc t = {NAN, 0.f, nullptr};
    IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, off, 3, 1, nullptr, nullptr, nullptr, &t, o));
    // factors that the kernels could not hold
    const otas_score_desc extremes[] = {{3e38f, 0.f, nullptr}, {0.f, 3e38f, nullptr}, {1.f, 1e-40f, nullptr}, {-3e38f, 0.f, nullptr}, {1e30f, 1e-20f, nullptr}};
    for (const otas_score_desc& x : extremes) IS(OTAS_EINVAL, otas_attention_masked(c, qkv, 2, off, 3, 1, nullptr, nullptr, nullptr, &x, o));
    const otas_score_desc wide[] = {{-2e38f, 0.f, nullptr}, {1e-30f, 1e30f, nullptr}, {1.f, 1e-37f, nullptr}};
    for (const otas_score_desc& x : wide) IS(OTAS_OK, otas_attention_masked(c, qkv, 2, off, 3, 1, nullptr, nullptr, nullptr, &x, o));
    const int32_t longer[] = {0, OTAS_MAX_LONG_SEQ + 1}, longest[] = {0, OTAS_MAX_LONG_SEQ};
    IS(OTAS_EUNSUPPORTED, otas_attention_masked(c, qkv, 2, longer, 1, 1, nullptr, nullptr, nullptr, nullptr, o));
    IS(OTAS_OK, otas_attention_masked(c, qkv, 2, longest, 1, 1, nullptr, nullptr, nullptr, nullptr, o));

    const otas_kv_cache k = {base + (4ull << 36), base + (5ull << 36), pos, (float*)pos, 600, 2, 100};
    auto cache_but = [&](auto change) { otas_kv_cache x = k; change(x); return x; };
    const int32_t slot[] = {5, 0, 599}, len[] = {100, 0, 40}, rows[] = {7, 0, 7}, roff[] = {0, 0, 2, 3};
    int32_t out[600];
    IS(OTAS_OK, otas_cache_append(c, &k, qkv, 8, roff, rows, pos, slot, len, 3, out));
    CHECK(out[0] == 100 && out[1] == 2 && out[2] == 41);
    IS(OTAS_OK, otas_cache_append(c, &k, qkv, 8, roff, nullptr, pos, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, &k, qkv, 7, roff, rows, pos, slot, len, 3, out));    // row 7 of 7
    IS(OTAS_EINVAL, otas_cache_append(c, &k, qkv, 2, roff, nullptr, pos, slot, len, 3, out));
    const int32_t roff2[] = {0, 1, 2, 3}, twice[] = {5, 0, 5}, outside[] = {5, 0, 600}, over[] = {100, 0, 101}, under[] = {100, -1, 0};
    IS(OTAS_EINVAL, otas_cache_append(c, &k, qkv, 8, roff2, rows, pos, slot, len, 3, out));   // slot 5 is full
    IS(OTAS_EINVAL, otas_cache_append(c, &k, qkv, 8, roff, rows, pos, twice, len, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, &k, qkv, 8, roff, rows, pos, outside, len, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, &k, qkv, 8, roff, rows, pos, slot, over, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, &k, qkv, 8, roff, rows, pos, slot, under, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, nullptr, qkv, 8, roff, rows, pos, slot, len, 3, out));
    const otas_kv_cache bad_heads = cache_but([](auto& x) { x.kv_heads = 3; }), no_slots = cache_but([](auto& x) { x.slots = 0; }),
                        odd_place = cache_but([](auto& x) { x.v = (char*)x.v + 8; }), no_mass = cache_but([](auto& x) { x.mass = nullptr; }),
                        no_pos = cache_but([](auto& x) { x.positions = nullptr; }), huge = cache_but([](auto& x) { x.capacity = OTAS_MAX_LONG_SEQ + 1; });
    IS(OTAS_EINVAL, otas_cache_append(c, &bad_heads, qkv, 8, roff, rows, pos, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, &no_slots, qkv, 8, roff, rows, pos, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, &odd_place, qkv, 8, roff, rows, pos, slot, len, 3, out));
    IS(OTAS_EINVAL, otas_cache_append(c, &no_pos, qkv, 8, roff, rows, pos, slot, len, 3, out));
    IS(OTAS_EUNSUPPORTED, otas_cache_append(c, &huge, qkv, 8, roff, rows, pos, slot, len, 3, out));
    IS(OTAS_OK, otas_cache_append(c, &no_mass, qkv, 8, roff, rows, pos, slot, len, 3, out));

    // arrays of a call within the cache; the cache's two arrays in one
    const size_t held = (size_t)600 * 2 * 100 * 64 * (dtype == OTAS_F32 ? 4 : 2);
    const otas_kv_cache one = cache_but([](auto& x) { x.v = x.k; });
    IS(OTAS_EINVAL, otas_cache_append(c, &one, qkv, 8, roff, rows, pos, slot, len, 3, out));
    for (char* in : {(char*)k.k, (char*)k.v}) {
      IS(OTAS_EINVAL, otas_cache_append(c, &k, in, 8, roff, rows, pos, slot, len, 3, out));
      IS(OTAS_EINVAL, otas_cache_append(c, &k, in + held - 256, 8, roff, rows, pos, slot, len, 3, out));
      IS(OTAS_OK, otas_cache_append(c, &k, in + held, 8, roff, rows, pos, slot, len, 3, out));
      IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, nullptr, nullptr, slot, len, 3, nullptr, 0, in + 256, (size_t)1 << 30, o));
      IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, nullptr, nullptr, slot, len, 3, nullptr, 0, ws, (size_t)1 << 30, in - 256));
      const int32_t half[] = {50, 0, 20};
      IS(OTAS_EINVAL, otas_cache_evict(c, &k, slot, len, half, 3, 0, nullptr, in, (size_t)1 << 30, out));
    }
    const otas_kv_cache endless = cache_but([](auto& x) { x.slots = INT32_MAX; x.capacity = OTAS_MAX_LONG_SEQ; });
    IS(OTAS_EINVAL, otas_cache_append(c, &endless, (char*)k.k + (1ull << 50), 8, roff, rows, pos, slot, len, 3, out));
    IS(OTAS_OK, otas_cache_append(c, &endless, qkv, 8, roff, rows, pos, slot, len, 3, out));

    const int32_t parents[] = {-1, 0, 0, -1, 0, 1, 2, 3}, chain[] = {-1, 0, 1, -1, 0, 1, 2, 3};
    size_t need = otas_attention_tree_workspace_bytes(c, 2, off, len, 3, 1);
    CHECK(need > 0 && need % 256 == 0);
    IS(OTAS_OK, otas_attention_tree(c, &k, qkv, off, parents, pos, slot, len, 3, &s, 1, ws, need, o));
    IS(OTAS_OK, otas_attention_tree(c, &k, qkv, off, chain, nullptr, slot, len, 3, nullptr, 0, ws, need, o));
    IS(OTAS_OK, otas_attention_tree(c, &k, qkv, off, nullptr, nullptr, twice, len, 3, nullptr, 0, ws, need, o));
    IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, nullptr, nullptr, twice, len, 3, nullptr, 1, ws, need, o));
    IS(OTAS_EINVAL, otas_attention_tree(c, &no_mass, qkv, off, nullptr, nullptr, slot, len, 3, nullptr, 1, ws, need, o));
    IS(OTAS_ENOMEM, otas_attention_tree(c, &k, qkv, off, parents, pos, slot, len, 3, &s, 1, ws, 64, o));
    IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, parents, pos, slot, len, 3, &s, 1, (char*)ws + 16, need, o));
    IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, parents, pos, slot, len, 3, &s, 1, ws, need, qkv));
    IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, parents, pos, slot, len, 3, &s, 1, qkv, need, o));
    IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, parents, pos, slot, over, 3, &s, 1, ws, need, o));
    otas_score_desc sloped = {0.f, 0.f, (const float*)pos};
    IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, parents, nullptr, slot, len, 3, &sloped, 1, ws, need, o));
    const int32_t self[] = {0, 0, 0, -1, 0, 1, 2, 3}, low[] = {-2, 0, 0, -1, 0, 1, 2, 3}, later[] = {-1, 0, 0, -1, 2, 1, 2, 3};
    for (const int32_t* p : {self, low, later}) IS(OTAS_EINVAL, otas_attention_tree(c, &k, qkv, off, p, pos, slot, len, 3, &s, 1, ws, need, o));
    const int32_t most[] = {0, 64}, more[] = {0, 65}, one_slot[] = {3}, one_len[] = {50};
    need = otas_attention_tree_workspace_bytes(c, 2, most, one_len, 1, 1);
    IS(OTAS_OK, otas_attention_tree(c, &k, qkv, most, nullptr, pos, one_slot, one_len, 1, &s, 1, ws, need, o));
    IS(OTAS_EUNSUPPORTED, otas_attention_tree(c, &k, qkv, more, nullptr, pos, one_slot, one_len, 1, &s, 1, ws, (size_t)1 << 34, o));
    CHECK(otas_attention_tree_workspace_bytes(c, 2, more, one_len, 1, 0) == 0 && otas_attention_tree_workspace_bytes(nullptr, 2, most, one_len, 1, 1) == 0);
    // a program that keeps one workspace asks for the longest lengths
    for (int B : {1, 5, 40}) {
      std::vector<int32_t> of(B + 1), ls(B);
      for (int q = 0; q <= B; ++q) of[q] = 3 * q;
      for (int mass : {0, 1}) {
        size_t before = 0;
        for (int l = 0; l < 100000; l = l * 5 / 4 + 1) {
          std::fill(ls.begin(), ls.end(), l);
          const size_t n = otas_attention_tree_workspace_bytes(c, 2, of.data(), ls.data(), B, mass);
          CHECK(n >= before);
          before = n;
        }
      }
    }

    const int32_t keep[] = {30, 0, 40};
    need = otas_cache_evict_workspace_bytes(c, len, keep, 3);
    CHECK(need > 0);
    IS(OTAS_OK, otas_cache_evict(c, &k, slot, len, keep, 3, 2, len, ws, need, out));
    CHECK(out[0] == 30 && out[1] == 0 && out[2] == 40);
    IS(OTAS_OK, otas_cache_evict(c, &k, slot, len, keep, 3, 0, nullptr, ws, need, out));
    IS(OTAS_ENOMEM, otas_cache_evict(c, &k, slot, len, keep, 3, 0, nullptr, ws, 64, out));
    IS(OTAS_EINVAL, otas_cache_evict(c, &k, slot, len, keep, 3, -1, nullptr, ws, need, out));
    IS(OTAS_EINVAL, otas_cache_evict(c, &k, twice, len, keep, 3, 0, nullptr, ws, need, out));
    IS(OTAS_EINVAL, otas_cache_evict(c, &no_mass, slot, len, keep, 3, 0, nullptr, ws, need, out));
    IS(OTAS_EINVAL, otas_cache_evict(c, &k, slot, len, under, 3, 0, nullptr, ws, need, out));
    CHECK(otas_cache_evict_workspace_bytes(c, len, under, 3) == 0);

    // host numbers that do not fit the arguments: uploaded, refused while the stream is captured
    std::vector<int32_t> many(500), zero(500, 0), offs(501);
    for (int q = 0; q < 500; ++q) { many[q] = 599 - q; offs[q + 1] = q + 1; }
    for (bool cap : {false, true}) {
      capturing = cap;
      const otas_status want = cap ? OTAS_EUNSUPPORTED : OTAS_OK;
      IS(want, otas_cache_append(c, &k, qkv, 500, offs.data(), nullptr, pos, many.data(), zero.data(), 500, out));
      IS(want, otas_attention_masked(c, qkv, 2, offs.data(), 500, 1, nullptr, nullptr, nullptr, nullptr, o));
      IS(want, otas_attention_tree(c, &k, qkv, offs.data(), nullptr, nullptr, many.data(), zero.data(), 500, nullptr, 0, ws, (size_t)1 << 30, o));
      std::vector<int32_t> ten(500, 10), five(500, 5);
      IS(want, otas_cache_evict(c, &k, many.data(), ten.data(), five.data(), 500, 0, nullptr, ws, (size_t)1 << 30, out));
      IS(OTAS_OK, otas_rotary(c, qkv, 500, 2, pos, &r, o));
    }
    capturing = false;
    std::vector<int32_t> big(OTAS_MAX_LONG_SEQ, 0);   // more host numbers than the plan buffer holds
    const int32_t boff[] = {0, OTAS_MAX_LONG_SEQ};
    const otas_kv_cache deep = cache_but([](auto& x) { x.capacity = OTAS_MAX_LONG_SEQ; });
    IS(OTAS_ENOMEM, otas_cache_append(c, &deep, qkv, 8, boff, big.data(), pos, one_slot, none, 1, out));
    CHECK(otas_destroy(c) == OTAS_OK);
  }
  std::puts("decode api ok");
  return 0;
}
