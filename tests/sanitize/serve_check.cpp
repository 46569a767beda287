// Sanitizer driver for the host code of the operators that serve from the 4-bit cache (test
// infrastructure): linked with host-sanitized builds of kia_serve_abi.hip and kia_abi.hip and
// run by tests/test_serve_sanitizers_host.py on a machine without a GPU. Sizes of workspaces
// over many shapes, and calls that every argument check refuses on the host before any HIP call
// but the count of compute units.
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include "kia.h"

static int fails = 0;
#define CHECK(c)                                                   \
  do {                                                             \
    if (!(c)) {                                                    \
      fprintf(stderr, "check failed line %d: %s\n", __LINE__, #c); \
      ++fails;                                                     \
    }                                                              \
  } while (0)

int main() {
  alignas(256) static char buf[256];
  int32_t *ints = reinterpret_cast<int32_t *>(buf);
  const int most = INT_MAX;
  for (int page : {16, 64, 256, 17, 0})
    for (int width : {1, 63, 8192, 1 << 20, most / 16, most, 0, -1})
      for (int B : {1, 33, 1 << 14, most})
        for (int G : {1, 7, 128, most})
          for (int T : {1, 5, 1 << 10, most})
            for (int d : {32, 64, 128, 48}) {
              size_t n = 1;
              int rc = kia_cache4_select_ws_bytes(page, width, B, G, 1, T, d, &n);
              CHECK((rc == KIA_OK) == (n > 0));
              for (int count : {1, 999, 200000, 200001, most, -1}) {
                rc = kia_cache4_pages_ws_bytes(page, width, count, B, G, 1, T, d, &n);
                CHECK((rc == KIA_OK) == (n > 0));
              }
              for (int shared : {32, 256, 1 << 20, most, 0}) {
                rc = kia_cache4_shared_ws_bytes(page, width, shared, B, G, 1, T, d, &n);
                CHECK((rc == KIA_OK) == (n > 0));
              }
            }

  // refusals
  kia_view ok = {buf, 64 * 8 * 2, 64 * 8, 64}, bad = {buf, 0, 0, 3}, off = {buf + 2, 1024, 512, 64};
  for (int i = 0; i < 4; ++i)
    for (const kia_view *x : {(const kia_view *)&bad, (const kia_view *)&off, (const kia_view *)nullptr}) {
      const kia_view *v[4];
      for (int k = 0; k < 4; ++k) v[k] = k == i ? x : &ok;
      CHECK(kia_cache4_append(v[0], v[1], v[2], v[3], buf, buf, 1, 16, ints, 1, ints, nullptr, (const double *)buf,
                              1.f, 0, 1, 2, 2, 8, 64, 64, KIA_BF16, nullptr) != KIA_OK);
      if (i < 2) {
        CHECK(kia_cache4_attn_pages(v[0], v[1], buf, 1, 16, ints, 1, ints, ints, 1, buf, 1, 2, 2, 8, 64, 4, 1, 8.f, 1,
                                    KIA_BF16, nullptr) != KIA_OK);
        CHECK(kia_cache4_attn_shared(v[0], v[1], buf, 1, 16, ints, 2, ints, 32, buf, 1, 2, 2, 8, 64, 4, 1, 8.f, 1,
                                     KIA_BF16, nullptr) != KIA_OK);
      }
      if (i < 1)
        CHECK(kia_cache4_select(v[0], buf, 1, 16, ints, 1, ints, buf, ints, 2, 1, 1, 1, 2, 2, 8, 64, KIA_BF16,
                                nullptr) != KIA_OK);
    }
  for (int starts : {0, 1})
    CHECK(kia_cache4_bounds(buf, buf, 1, 16, ints, 1, starts ? ints : nullptr, starts ? nullptr : ints, 1, 2, 64,
                            nullptr) == KIA_ERR_NULL);
  CHECK(kia_cache4_append(&ok, &ok, &ok, &ok, buf, buf, 1, 16, ints, 1, ints, nullptr, (const double *)buf, 1.f, 0, 1,
                          2, 2, INT_MAX, 64, 64, KIA_BF16, nullptr) == KIA_ERR_SHAPE);
  CHECK(kia_cache4_select(&ok, buf, 1, 16, ints, 1, ints, buf, ints, INT_MAX, INT_MAX, INT_MAX, 1, 2, 2, 8, 64,
                          KIA_BF16, nullptr) == KIA_ERR_SHAPE);
  if (fails) return 1;
  printf("serve host sanitizer run: ok\n");
  return 0;
}
