// What include/otas_decode.h says of arrays that overlap a cache, at every entry point that has one, with the HIP runtime and the kernel launchers stubbed
// out.  Run under a sanitizer, see test_cache_overlap.py.
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
#include "../paper_2401_05031_amd/csrc/window_api.hip"

extern "C" hipError_t hipMalloc(void** p, size_t n) { *p = std::calloc(1, n); return hipSuccess; }
extern "C" hipError_t hipHostMalloc(void** p, size_t n, unsigned) { *p = std::calloc(1, n); return hipSuccess; }
extern "C" hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
extern "C" hipError_t hipHostFree(void* p) { std::free(p); return hipSuccess; }
extern "C" hipError_t hipGetSymbolAddress(void** p, const void*) { static int32_t cell[64]; *p = cell; return hipSuccess; }

#define CHECK(e) do { if (!(e)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #e); return 1; } } while (0)
#define IS(want, call) do { const otas_status got_ = (call); if (got_ != (want)) { std::fprintf(stderr, "line %d: %s -> %d\n", __LINE__, #call, (int)got_); return 1; } } while (0)

int main(int, char** argv) {
  const bool tree = argv[1][0] == 't';
  char* const base = (char*)(uintptr_t)(1ull << 40);
  char *qkv = base, *o = base + (1ull << 36), *ws = base + (2ull << 36);
  int32_t* pos = (int32_t*)(base + (3ull << 36));
  for (int dtype : {(int)OTAS_F32, (int)OTAS_BF16}) {
    const size_t e = dtype == OTAS_F32 ? 4 : 2;
    const otas_model_desc d = {1, 256, 4, 128, dtype, 1e-6f, 1};
    otas_layer_weights w;
    std::fill((const void**)&w, (const void**)(&w + 1), qkv);
    otas_ctx* c = nullptr;
    CHECK(otas_create(&c, &d, &w, nullptr) == OTAS_OK);
    const otas_kv_cache k = {base + (4ull << 36), base + (5ull << 36), pos, nullptr, 600, 2, 100};
    const otas_kv_cache4 f = {base + (4ull << 36), base + (5ull << 36), base + (6ull << 36), base + (7ull << 36), 600, 2, 128};
    const int32_t off[] = {0, 3, 3, 8}, slot[] = {5, 0, 599}, len[] = {100, 0, 40}, empty[] = {0, 0};
    const size_t bytes = (size_t)600 * 2 * 100 * 64 * e, row = (size_t)8 * 64 * e, room = (size_t)1 << 30;
    auto call = [&](int which, const void* in, const int32_t* offsets, int B, void* out) -> otas_status {
      if (which == 0) return otas_attention_tree(c, &k, in, offsets, nullptr, nullptr, slot, len, B, nullptr, 0, ws, room, out);
      if (which == 1) return otas_attention_recent(c, &k, in, offsets, slot, len, B, 50, 4, nullptr, ws, room, out);
      return otas_attention_cache4(c, &f, in, offsets, slot, len, B, 50, 4, nullptr, ws, room, out);
    };
    for (int which = tree ? 0 : 1; which < (tree ? 1 : 3); ++which) {
      IS(OTAS_OK, call(which, qkv, off, 3, o));
      IS(OTAS_OK, call(which, nullptr, empty, 1, nullptr));
      for (char* in : {(char*)k.k, (char*)k.v}) {
        const size_t size = which == 2 ? (size_t)600 * 2 * 128 * 32 : bytes;
        IS(OTAS_EINVAL, call(which, in, off, 3, o));
        IS(OTAS_EINVAL, call(which, in + 4096, off, 3, o));
        IS(OTAS_EINVAL, call(which, in + size - 16, off, 3, o));
        IS(OTAS_OK, call(which, in + size, off, 3, o));                    // right behind it
        IS(OTAS_EINVAL, call(which, in - 8 * row + 16, off, 3, o));        // its last bytes
        IS(OTAS_OK, call(which, in - 8 * row, off, 3, o));                 // right before it
        IS(OTAS_EINVAL, call(which, qkv, off, 3, in));
        for (int at : {0, 4096}) IS(OTAS_OK, call(which, in + at, empty, 1, in + 2 * at));   // no rows, no bytes
      }
    }
    CHECK(otas_destroy(c) == OTAS_OK);
  }
  std::puts("cache overlap ok");
  return 0;
}
