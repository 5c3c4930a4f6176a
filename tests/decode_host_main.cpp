// Host arithmetic of the decoder's operators (include/otas_decode.h) that no GPU is needed for: where the parts of a workspace lie, limits
// of launches, factors of a rotation.  Built as decode_api_main.cpp is, see test_decode_host.py.
#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime.h>
#ifndef __align__
#define __align__(n) __attribute__((aligned(n)))
#endif
#ifndef HIP_SYMBOL
#define HIP_SYMBOL(x) (&x)
#endif
#include "../paper_2401_05031_amd/csrc/api.hip"
#include "../paper_2401_05031_amd/csrc/decode_api.hip"

extern "C" hipError_t hipMalloc(void** p, size_t n) { *p = std::calloc(1, n); return hipSuccess; }
extern "C" hipError_t hipHostMalloc(void** p, size_t n, unsigned) { *p = std::calloc(1, n); return hipSuccess; }
extern "C" hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
extern "C" hipError_t hipHostFree(void* p) { std::free(p); return hipSuccess; }
extern "C" hipError_t hipGetSymbolAddress(void** p, const void*) { static int32_t cell[64]; *p = cell; return hipSuccess; }

#define CHECK(e) do { if (!(e)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #e); return 1; } } while (0)
#define IS(want, call) do { const otas_status got_ = (call); if (got_ != (want)) { std::fprintf(stderr, "line %d: %s -> %d\n", __LINE__, #call, (int)got_); return 1; } } while (0)

// Sums and logits of a tree begin at multiples of four floats, one behind the other and within what the caller is asked for.
static int workspace_places() {
  int uneven = 0;
  for (int dtype : {0, 1})
    for (int dh : {4, 20, 64, 80, 128})
      for (int H : {1, 3, 6, 7})
        for (int KV : {1, 3})
          for (int B : {1, 3, 40})
            for (int n : {1, 2, 9, 64})
              for (int l : {0, 1, 130, 300, 600, 1100, 5000, 70000}) {
                if (H % KV) continue;
                std::vector<int32_t> off(B + 1), len(B);
                for (int q = 0; q <= B; ++q) off[q] = n * q;
                for (int q = 0; q < B; ++q) len[q] = l * (q + 1) / B;
                const int64_t T = off[B], TH = T * H;
                const TreeShape t = tree_shape(dtype, dh, H, KV, off.data(), len.data(), B);
                CHECK(t.parts >= 1 && t.room >= t.parts);
                if (t.parts > 1) {
                  const size_t sums = tree_sums_at(t, T, H);
                  uneven += 2 * TH * (1 + t.parts) % 4 != 0;
                  CHECK(sums % 4 == 0 && sums >= (size_t)(2 * TH * (1 + t.parts)));
                  CHECK(sums + (size_t)TH * t.parts * dh <= tree_logits_at(t, T, H, dh));
                }
                CHECK(tree_logits_at(t, T, H, dh) % 4 == 0);
                for (bool mass : {false, true}) {
                  const bool logits = mass && dtype != 0 && bf16_width(dh) && t.rows == 32;
                  CHECK(tree_workspace_floats(t, dtype, T, H, dh, l, mass) >= tree_logits_at(t, T, H, dh) + (logits ? (size_t)TH * l : 0));
                }
              }
  CHECK(uneven > 100);   // the case was met
  return 0;
}

// As many workgroups as a launch may have, and one more.
static int most_workgroups() {
  char* const base = (char*)(uintptr_t)(1ull << 40);
  void *qkv = base, *ws = base + (1ull << 44);
  for (int dtype : {(int)OTAS_F32, (int)OTAS_BF16}) {
    const otas_model_desc d = {1, 64, 1, 64, dtype, 1e-6f, 1};
    otas_layer_weights w;
    std::fill((const void**)&w, (const void**)(&w + 1), qkv);
    otas_ctx* c = nullptr;
    CHECK(otas_create(&c, &d, &w, nullptr) == OTAS_OK);
    const otas_kv_cache k = {base + (1ull << 45), base + (1ull << 46), (int32_t*)qkv, (float*)qkv, 70000, 1, OTAS_MAX_LONG_SEQ};
    std::vector<int32_t> off(17), slot(16), len(16, 0), out(16);
    for (int q = 0; q < 16; ++q) { slot[q] = 15 - q; off[q + 1] = (q + 1) << 20; }
    IS(OTAS_EUNSUPPORTED, otas_cache_append(c, &k, qkv, 1 << 24, off.data(), nullptr, (int32_t*)qkv, slot.data(), len.data(), 16, out.data()));
    off[16] -= 1;
    IS(OTAS_OK, otas_cache_append(c, &k, qkv, 1 << 24, off.data(), nullptr, (int32_t*)qkv, slot.data(), len.data(), 16, out.data()));
    CHECK(out[0] == 1 << 20 && out[15] == (1 << 20) - 1);
    // an eviction's queries, and its lists of places and sources: 2 x 524288 entries a query here
    const int B = 65536;
    std::vector<int32_t> all(B), n(B, 10), five(B, 5), rest(B);
    for (int q = 0; q < B; ++q) all[q] = q;
    IS(OTAS_EUNSUPPORTED, otas_cache_evict(c, &k, all.data(), n.data(), five.data(), B, 0, nullptr, ws, (size_t)1 << 40, rest.data()));
    IS(OTAS_OK, otas_cache_evict(c, &k, all.data(), n.data(), five.data(), B - 1, 0, nullptr, ws, (size_t)1 << 40, rest.data()));
    std::fill(n.begin(), n.end(), OTAS_MAX_LONG_SEQ);
    std::fill(five.begin(), five.end(), OTAS_MAX_LONG_SEQ / 2);
    IS(OTAS_EUNSUPPORTED, otas_cache_evict(c, &k, all.data(), n.data(), five.data(), 2048, 0, nullptr, ws, (size_t)1 << 40, rest.data()));
    IS(OTAS_OK, otas_cache_evict(c, &k, all.data(), n.data(), five.data(), 2047, 0, nullptr, ws, (size_t)1 << 40, rest.data()));
    CHECK(otas_destroy(c) == OTAS_OK);
  }
  return 0;
}

// Rotations whose base or whose farthest angle is no number in 64 bits, and their like that are.
static int rotations() {
  char* const base = (char*)(uintptr_t)(1ull << 40);
  const otas_model_desc d = {1, 128, 1, 64, OTAS_F32, 1e-6f, 1};
  otas_layer_weights w;
  std::fill((const void**)&w, (const void**)(&w + 1), base);
  otas_ctx* c = nullptr;
  CHECK(otas_create(&c, &d, &w, nullptr) == OTAS_OK);
  auto turn = [&](int rot, int scaling, double b, double factor) {
    const otas_rotary_desc r = {rot, OTAS_ROTARY_HALF, scaling, 0, b, factor, 4096.0, 32.0, 1.0, 1.0};
    return otas_rotary(c, base, 5, 1, (int32_t*)base, &r, base);
  };
  IS(OTAS_EINVAL, turn(4, OTAS_ROTARY_BASE, 10000.0, 1e160));     // base 1e324: all but the first pair would stand still
  IS(OTAS_OK, turn(4, OTAS_ROTARY_BASE, 10000.0, 1e150));
  IS(OTAS_EINVAL, turn(128, OTAS_ROTARY_BASE, 1e300, 1e10));
  IS(OTAS_EINVAL, turn(4, OTAS_ROTARY_BASE, 1.0, 1e-170));        // base 0
  IS(OTAS_EINVAL, turn(4, OTAS_ROTARY_LINEAR, 1e-300, 1e-154));   // 1e304 at position 1, infinity from 1e4 on
  IS(OTAS_OK, turn(4, OTAS_ROTARY_LINEAR, 1e-300, 1.0));
  IS(OTAS_OK, turn(4, OTAS_ROTARY_PLAIN, 1e300, 0.0));
  CHECK(otas_destroy(c) == OTAS_OK);
  return 0;
}

int main() {
  if (workspace_places() || most_workgroups() || rotations()) return 1;
  std::puts("decode host ok");
  return 0;
}
