// Drives the host side of the calls on 8-bit pages -- everything that runs before a GPU call -- in a build whose host code is
// instrumented with AddressSanitizer and UndefinedBehaviorSanitizer (tests/test_pages_sanitizers.py).  Device pointers are fake and
// never dereferenced: every call fails its validation or has nothing to launch.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <vector>

#include "ifkv.h"

static int g_failures = 0;
#define EXPECT(cond)                                                  \
  do {                                                                \
    if (!(cond)) {                                                    \
      std::printf("line %d: expectation failed: %s\n", __LINE__, #cond); \
      ++g_failures;                                                   \
    }                                                                 \
  } while (0)

static uint32_t lcg(uint32_t &s) { return s = s * 1664525u + 1013904223u; }

int main() {
  const int64_t limits[] = {0, 1, 2, 63, 64, 65, 4096, INT32_MAX, int64_t(INT32_MAX) + 1, INT64_MAX, -1, INT64_MIN};
  uint32_t seed = 7;
  for (int dtype : {IFKV_BF16, IFKV_F32})
    for (int d : {64, 128}) {
      ifkv_layer_desc desc;
      std::memset(&desc, 0, sizeof desc);
      desc.dtype = dtype, desc.n_q_heads = 32, desc.n_kv_heads = 8, desc.head_dim = d, desc.rope_theta = 5e5;
      desc.max_ctx = 4096, desc.max_prompt = 64;
      ifkv_ctx *c = nullptr;
      EXPECT(ifkv_create(&c, &desc, nullptr) == IFKV_OK);
      char *f = reinterpret_cast<char *>(4096);
      int32_t *fi = reinterpret_cast<int32_t *>(4096);
      ifkv_page_cache pages = {f, f, reinterpret_cast<float *>(f), reinterpret_cast<float *>(f), 1000};

      // lists of copies: each has one fault, wherever it stands; the lists end where their memory ends
      for (int turn = 0; turn < 300; ++turn) {
        const int n = 1 + lcg(seed) % 499;
        std::vector<int32_t> src(n), dst(n);
        for (int i = 0; i < n; ++i) dst[i] = 2 * i, src[i] = 2 * (lcg(seed) % 499) + 1;
        const int at = lcg(seed) % n, other = lcg(seed) % n;
        switch (turn % 6) {
          case 0: src[at] = -1; break;
          case 1: src[at] = 1000; break;
          case 2: dst[at] = INT32_MIN; break;
          case 3: dst[at] = INT32_MAX; break;
          case 4: src[at] = dst[other]; break;
          default:
            if (at == other) dst[at] = -5;
            else dst[at] = dst[other];
        }
        EXPECT(ifkv_copy_pages(c, &pages, n, src.data(), dst.data()) == IFKV_EINVAL);
      }
      // sizes at the ends of their types: refused, or nothing to do
      for (int64_t a : limits)
        for (int64_t b : limits) {
          const int32_t a32 = static_cast<int32_t>(a), b32 = static_cast<int32_t>(b);
          ifkv_page_cache none = {nullptr, nullptr, nullptr, nullptr, a};
          EXPECT(ifkv_copy_pages(c, &none, b == 0 ? 1 : b, nullptr, nullptr) != IFKV_OK);
          EXPECT(ifkv_store_pages(c, &pages, fi, a32, b32, nullptr, fi, fi, b, f, f, 0, 0) != IFKV_OK || a32 == 0 || b == 0);
          EXPECT(ifkv_store_pages(c, &pages, fi, 1, 1, nullptr, fi, fi, 3, f, f, a, b) != IFKV_OK);
          EXPECT(ifkv_attend_pages(c, &pages, fi, a32, 3, fi, b32, f, a, fi, b, nullptr, nullptr) != IFKV_OK || a32 == 0 || b == 0);
          EXPECT(ifkv_attend_pages(c, &none, fi, 2, b32, fi, a32, nullptr, b, fi, 2, f, nullptr) != IFKV_OK);
          std::vector<int32_t> axes(d / 2, 0);
          EXPECT(ifkv_rope_rows_axes(c, nullptr, fi, a32, axes.data(), b == 0 ? 1 : b, 40, a) != IFKV_OK);
          EXPECT(ifkv_rope_rows_axes(c, nullptr, fi, 1, axes.data(), 4, a32, b) != IFKV_OK);
          axes[lcg(seed) % axes.size()] = 1 + lcg(seed) % 100;
          EXPECT(ifkv_rope_rows_axes(c, f, fi, 1, axes.data(), 4, 40, 0) == IFKV_EINVAL);
        }
      ifkv_destroy(c);
    }
  if (g_failures == 0) std::printf("calls on pages under the sanitizers: ok\n");
  return g_failures != 0;
}
