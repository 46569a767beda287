// Sanitizer driver for the host code of the operators around the attention (test
// infrastructure): linked with host-sanitized builds of kia_around_abi.hip and kia_abi.hip
// and run by tests/test_around_sanitizers_host.py on a machine without a GPU. Sizes of
// workspaces over many shapes, and calls that every argument check refuses on the
// host before any HIP call but the count of compute units.
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
  float *f = reinterpret_cast<float *>(buf);
  // workspaces: every size that the checks let through, small and at the limits
  const int T[] = {1, 63, 64, 65, 1000, 65536, 1 << 20, 1 << 24, (1 << 24) + 1, 0, INT_MAX};
  const int W[] = {1, 63, 512, 1 << 20, INT_MAX, 0};
  const int S[] = {0, 1, 64, 1 << 20, INT_MAX, -1};
  for (int t : T)
    for (int w : W)
      for (int s : S)
        for (int H : {1, 8, 64})
          for (int d : {16, 64, 128}) {
            size_t n = 1;
            const int rc = kia_window_ws_bytes(2, H, H < 8 ? H : H / 8, t, d, w, s, &n);
            const bool ok = t >= 1 && t <= 1 << 24 && w >= 1 && s >= 0;
            CHECK((rc == KIA_OK) == ok && (n > 0) == ok);
            if (ok) CHECK(n >= (size_t)2 * H * t * 4 && n < (size_t)2 * H * t * 4 + (1u << 29));
            size_t m = 1;
            const int rc2 = kia_cache4_ws_bytes(64, t < 1 ? t : t / 64 + 1, 3, H, H < 8 ? H : H / 8,
                                                1 + (w & 3), d, w == INT_MAX ? 0 : w, s, &m);
            CHECK((rc2 == KIA_OK) == (m > 0));
          }
  size_t n = 1;
  CHECK(kia_cache4_bytes(1 << 20, 256, 128, 128, &n) == KIA_OK &&
        n == (size_t)(1 << 20) * 2 * 128 * 256 * 68);
  CHECK(kia_cache4_bytes(1, 17, 1, 64, &n) == KIA_ERR_CACHE && n == 0);

  // refusals
  kia_view ok = {buf, 64 * 8 * 2, 64 * 8, 64}, bad = {buf, 0, 0, 3}, off = {buf + 2, 1024, 512, 64};
  for (int i = 0; i < 8; ++i) {
    const kia_view *v[8];
    for (const kia_view *x : {(const kia_view *)&bad, (const kia_view *)&off, (const kia_view *)nullptr}) {
      for (int k = 0; k < 8; ++k) v[k] = k == i ? x : &ok;
      CHECK(kia_window_bwd(v[0], v[1], v[2], v[3], v[4], f, nullptr, buf, v[5], v[6], v[7], 1, 2, 2,
                           8, 64, 4, 0, KIA_BF16, nullptr) != KIA_OK);
      if (i < 4) {
        CHECK(kia_window_fwd(v[0], v[1], v[2], v[3], f, nullptr, 1, 2, 2, 8, 64, 4, 0, KIA_BF16,
                             nullptr) != KIA_OK);
        CHECK(kia_rotary(v[0], v[1], v[2], v[3], nullptr, 0, 0, (const double *)buf, 1.f, 0, 0, 1, 2,
                         2, 8, 64, 64, KIA_BF16, nullptr) != KIA_OK);
      }
      if (i < 2) {
        CHECK(kia_cache4_write(v[0], v[1], buf, 1, 16, ints, 1, ints, nullptr, 1, 2, 8, 64, KIA_BF16,
                               nullptr) != KIA_OK);
        CHECK(kia_cache4_read(buf, 1, 16, ints, 1, ints, nullptr, v[0], v[1], 1, 2, 8, 64, KIA_BF16,
                              nullptr) != KIA_OK);
        CHECK(kia_cache4_attn(v[0], v[1], buf, 1, 16, ints, 1, ints, buf, 1, 2, 2, 8, 64, 4, 1, 8.f,
                              1, 0, 0, KIA_BF16, nullptr) != KIA_OK);
      }
    }
  }
  CHECK(kia_rotary(&ok, &ok, nullptr, nullptr, nullptr, 0, INT_MAX, (const double *)buf, 1.f, 0, 0, 1,
                   2, 0, 8, 64, 64, KIA_BF16, nullptr) == KIA_ERR_SHAPE);
  CHECK(kia_cache4_attn(&ok, &ok, buf, 1, 16, ints, 1, ints, buf, 1, 3, 2, 8, 64, 4, 1, 8.f, 1, 0, 0,
                        KIA_BF16, nullptr) == KIA_ERR_HEADS);
  if (fails) return 1;
  printf("around host sanitizer run: ok\n");
  return 0;
}
