// kia_checks.hpp -- argument checks that the entry points of the operators around the
// attention share. Host side only.
#pragma once

#include <limits.h>
#include <math.h>

#include <algorithm>

#include "kia_around.hpp"

namespace kia {

inline bool al16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? KIA_OK : KIA_ERR_HIP; }
inline int bytes_of(int dtype) { return dtype == KIA_F32 ? 4 : 2; }
// A launch counts its threads, 256 a workgroup, in 32 bits.
inline bool too_many(double groups) { return groups >= 1 << 24; }

inline int check_common(int B, int H, int Hkv, int T, int d, int dtype, bool small_heads) {
  if (B < 1 || H < 1 || Hkv < 1 || T < 1) return KIA_ERR_SHAPE;
  if (d != 32 && d != 64 && d != 128 && !(small_heads && d == 16)) return KIA_ERR_HEADDIM;
  if (dtype != KIA_F32 && dtype != KIA_BF16) return KIA_ERR_ENUM;
  return KIA_OK;
}

// One view: 16-byte aligned rows that do not overlap. (Strides of dimensions of size 1
// are not looked at: the kernels never multiply them by more than 0.)
inline int check_view(const kia_view *v, int B, int H, int T, int d, int dtype) {
  if (!v || !v->data) return KIA_ERR_NULL;
  if (!al16(v->data)) return KIA_ERR_ALIGN;
  const int64_t unit = 16 / bytes_of(dtype);
  if (T > 1 && (v->st < d || v->st > (1 << 22) || v->st % unit)) return KIA_ERR_VIEW;
  if ((H > 1 && (v->sh < 0 || v->sh % unit)) || (B > 1 && (v->sb < 0 || v->sb % unit)))
    return KIA_ERR_VIEW;
  return KIA_OK;
}
inline View view_of(const kia_view *v, int B, int H, int T) {
  View w;
  w.p = v->data;
  w.sb = B > 1 ? v->sb : 0;
  w.sh = H > 1 ? v->sh : 0;
  w.st = T > 1 ? v->st : 0;
  return w;
}

inline int page_log(int page) {
  for (int l = 4; l <= 8; ++l)
    if (page == 1 << l) return l;
  return -1;
}

inline int check_cache(const void *cache, int pages, int page, const int32_t *table, int width, int B,
                int H, int Hkv, int T, int d, int dtype) {
  int rc = check_common(B, H, Hkv, T, d, dtype, false);
  if (rc) return rc;
  if (page_log(page) < 0) return KIA_ERR_CACHE;
  if (pages < 1 || width < 1 || (int64_t)width * page > INT_MAX) return KIA_ERR_SHAPE;
  if (!cache || !table) return KIA_ERR_NULL;
  if (!al16(cache) || (uintptr_t)table & 3u) return KIA_ERR_ALIGN;
  return KIA_OK;
}

inline int check_cached(int H, int Hkv, int K, int calib, float tau, int recon, int window, int sinks) {
  if (H % Hkv) return KIA_ERR_HEADS;
  if (recon < KIA_RECON_LERP || recon > KIA_RECON_SOFTMAX) return KIA_ERR_ENUM;
  if (recon != KIA_RECON_SOFTMAX) {
    if (K < 1 || K > 64) return KIA_ERR_K;
    if (calib < KIA_CALIB_MINMAX || calib > KIA_CALIB_RESOLVED) return KIA_ERR_ENUM;
    if (calib != KIA_CALIB_MINMAX && !(tau > 0.f && isfinite(tau))) return KIA_ERR_TAU;
  }
  if (window < 0 || sinks < 0) return KIA_ERR_SHAPE;
  return KIA_OK;
}

}  // namespace kia
