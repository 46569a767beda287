// kia_around_abi.hip -- extern "C" entry points of the operators around K-interval
// attention (declared in include/kia.h). Host side only: argument checks before any
// launch, workspace sizes, launch shapes, launches on the caller's stream.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "kia_around.hpp"
#include "kia_host.hpp"

namespace {

using namespace kia;

bool al16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
int launched() { return hipGetLastError() == hipSuccess ? KIA_OK : KIA_ERR_HIP; }
int bytes_of(int dtype) { return dtype == KIA_F32 ? 4 : 2; }
// A launch counts its threads, 256 a workgroup, in 32 bits.
bool too_many(double groups) { return groups >= 1 << 24; }

int check_common(int B, int H, int Hkv, int T, int d, int dtype, bool small_heads) {
  if (B < 1 || H < 1 || Hkv < 1 || T < 1) return KIA_ERR_SHAPE;
  if (d != 32 && d != 64 && d != 128 && !(small_heads && d == 16)) return KIA_ERR_HEADDIM;
  if (dtype != KIA_F32 && dtype != KIA_BF16) return KIA_ERR_ENUM;
  return KIA_OK;
}

// One view: 16-byte aligned rows that do not overlap. (Strides of dimensions of size 1
// are not looked at: the kernels never multiply them by more than 0.)
int check_view(const kia_view *v, int B, int H, int T, int d, int dtype) {
  if (!v || !v->data) return KIA_ERR_NULL;
  if (!al16(v->data)) return KIA_ERR_ALIGN;
  const int64_t unit = 16 / bytes_of(dtype);
  if (T > 1 && (v->st < d || v->st > (1 << 22) || v->st % unit)) return KIA_ERR_VIEW;
  if ((H > 1 && (v->sh < 0 || v->sh % unit)) || (B > 1 && (v->sb < 0 || v->sb % unit)))
    return KIA_ERR_VIEW;
  return KIA_OK;
}
View view_of(const kia_view *v, int B, int H, int T) {
  View w;
  w.p = v->data;
  w.sb = B > 1 ? v->sb : 0;
  w.sh = H > 1 ? v->sh : 0;
  w.st = T > 1 ? v->st : 0;
  return w;
}

}  // namespace

// ---- rotary positions -----------------------------------------------------------
extern "C" int kia_rotary(const kia_view *q, const kia_view *q_out, const kia_view *k,
                          const kia_view *k_out, const int32_t *positions, int64_t positions_sb,
                          int first, const double *freq, float factor, int layout, int back, int B,
                          int H, int Hkv, int T, int d, int rot, int dtype, void *stream) {
  const bool keys = k || k_out;
  int rc = check_common(B, H, keys ? Hkv : 1, T, d, dtype, true);
  if (rc) return rc;
  if (rot < 2 || rot > d || rot % 2) return KIA_ERR_HEADDIM;
  if ((layout != KIA_ROTARY_HALF && layout != KIA_ROTARY_NEIGHBOURS) || (back != 0 && back != 1))
    return KIA_ERR_ENUM;
  if (!freq) return KIA_ERR_NULL;
  if ((uintptr_t)freq & 7u || (uintptr_t)positions & 3u) return KIA_ERR_ALIGN;
  if (positions_sb < 0 || (int64_t)first + T > INT_MAX) return KIA_ERR_SHAPE;
  if ((int64_t)B * T > INT_MAX || (int64_t)H + (keys ? Hkv : 0) > 65535) return KIA_ERR_SHAPE;
  int vw = 0;
  const int tokens = rotary_tokens(T, d, rot, dtype, vw);
  if (too_many((double)B * ((T + tokens - 1) / tokens))) return KIA_ERR_SHAPE;
  const kia_view *v[4] = {q, q_out, k, k_out};
  for (int i = 0; i < (keys ? 4 : 2); ++i) {
    rc = check_view(v[i], B, i < 2 ? H : Hkv, T, d, dtype);
    if (rc) return rc;
  }
  RotArgs a{};
  auto side = [&](RotSide &s, const kia_view *x, const kia_view *y, int heads) {
    const View u = view_of(x, B, heads, T), w = view_of(y, B, heads, T);
    s = RotSide{u.p, w.p, u.sb, u.sh, u.st, w.sb, w.sh, w.st};
  };
  side(a.q, q, q_out, H);
  if (keys) side(a.k, k, k_out, Hkv);
  a.pos = positions;
  a.pos_sb = positions_sb;
  a.freq = freq;
  a.factor = factor;
  a.first = first;
  a.layout = layout;
  a.back = back;
  a.B = B, a.H = H, a.Hkv = keys ? Hkv : 0, a.T = T, a.d = d, a.rot = rot;
  hipStream_t s = static_cast<hipStream_t>(stream);
  timed_call("kia_rotary", s, [&] { launch_rotary(a, dtype, host_cus(), s); });
  return launched();
}

// ---- attention with a sliding window ----------------------------------------------
namespace {

int check_window(int B, int H, int Hkv, int T, int d, int window, int sinks, int dtype) {
  int rc = check_common(B, H, Hkv, T, d, dtype, true);
  if (rc) return rc;
  if (H % Hkv) return KIA_ERR_HEADS;
  if (T > 1 << 24 || window < 1 || sinks < 0) return KIA_ERR_SHAPE;
  if ((double)B * H * ((T + 31) / 32) > 1 << 27) return KIA_ERR_SHAPE;
  return KIA_OK;
}

// (The key blocks' parts are less than 2816 more than the blocks: a part has `fine` tiles at
// least, all blocks together at most 512 times `most`, and most / fine is at most 11 / 2, by
// the division rounded down. So less than 2816 blocks have several parts, and their sums less
// than 45056 workgroups.)
bool window_too_many(int B, int H, int T) { return too_many((double)B * H * ((T + 63) / 64) + 4096); }

WinArgs window_args(int B, int H, int Hkv, int T, int d, int window, int sinks, int dtype) {
  WinArgs a{};
  a.B = B, a.H = H, a.Hkv = Hkv, a.T = T;
  a.window = std::min(window, T);
  // (first tokens that the window holds everywhere change nothing)
  a.sinks = a.window == T ? 0 : std::min(sinks, T);
  a.scale = (float)(1.0 / sqrt((double)d));
  // The key blocks' lists of query tiles, in parts of at most all tiles over the workgroups
  // that the chip holds (two a CU, of d = 128 in fp32 one), and of two tiles at least (four
  // of d = 128 in bf16; its sums cost as much to add). Blocks of first tokens, which every
  // query sees, are cut about four times finer (five and a half at most), so that they fill
  // the gaps that the others leave. (The places are those of the whole chip and not of the
  // device at hand: the workspace, whose size goes by the parts, is then the same on all.) Measured, dK and dV and the sum (us) with 8 / 4 / 2 tiles at least, windows of 256:
  //   d = 64, T = 1024, 12 heads, fp32            53 + 6 / 43 + 7 / 35 + 8
  //   d = 64, T = 500, 16 heads over 4, bf16      24 + 6 / 16 + 6 / 13 + 6
  //   d = 128, T = 1024, 16 heads over 4, bf16    34 + 7 / 27 + 8 / 29 + 10
  //   d = 128, T = 685, 21 heads over 3, window 7, fp32   86 + 6 / 54 + 6 / 35 + 7
  const int G = H / Hkv, nkb = (T + WIN_KB - 1) / WIN_KB;
  const int least = d == 128 && dtype == KIA_BF16 ? 4 : 2;
  const int slots = d == 128 && dtype == KIA_F32 ? 256 : 512;
  a.sink_blocks = (a.sinks + WIN_KB - 1) / WIN_KB;
  const int64_t all = (T + WIN_QT - 1) / WIN_QT;
  const int64_t near = std::min<int64_t>(all, (WIN_KB - 1 + (int64_t)a.window + WIN_QT - 1) / WIN_QT);
  const int64_t total = (int64_t)B * Hkv * G * (a.sink_blocks * all + (nkb - a.sink_blocks) * near);
  const int64_t most = std::max<int64_t>(least, (total + slots - 1) / slots);
  a.parts_b = nkb > a.sink_blocks ? (int)((G * near + most - 1) / most) : 1;
  const int64_t fine = std::max<int64_t>({least, G * near / (4 * a.parts_b), most / 4});
  a.parts_a = a.sink_blocks ? (int)((G * all + fine - 1) / fine) : 1;
  return a;
}

size_t window_ws(const WinArgs &a, int d) {
  const size_t delta = ((size_t)a.B * a.H * a.T * 4 + 255) / 256 * 256;
  const int nkb = (a.T + WIN_KB - 1) / WIN_KB;
  return delta + (size_t)a.B * a.Hkv * win_slots(nkb, a.sink_blocks, a.parts_a, a.parts_b) * 2 *
                     WIN_KB * d * 4;
}

}  // namespace

extern "C" int kia_window_ws_bytes(int B, int H, int Hkv, int T, int d, int window, int sinks,
                                   size_t *bytes) {
  if (!bytes) return KIA_ERR_NULL;
  *bytes = 0;
  const int rc = check_window(B, H, Hkv, T, d, window, sinks, KIA_F32);
  if (rc) return rc;
  // (for either type)
  for (int dtype : {KIA_F32, KIA_BF16})
    *bytes = std::max(*bytes, window_ws(window_args(B, H, Hkv, T, d, window, sinks, dtype), d));
  return KIA_OK;
}

extern "C" int kia_window_fwd(const kia_view *q, const kia_view *k, const kia_view *v,
                              const kia_view *o, float *lse, const int32_t *lengths, int B, int H,
                              int Hkv, int T, int d, int window, int sinks, int dtype,
                              void *stream) {
  int rc = check_window(B, H, Hkv, T, d, window, sinks, dtype);
  if (rc) return rc;
  if (window_too_many(B, H, T)) return KIA_ERR_SHAPE;
  const kia_view *x[4] = {q, k, v, o};
  for (int i = 0; i < 4; ++i) {
    rc = check_view(x[i], B, i == 1 || i == 2 ? Hkv : H, T, d, dtype);
    if (rc) return rc;
  }
  if (!lse) return KIA_ERR_NULL;
  if (!al16(lse) || (uintptr_t)lengths & 3u) return KIA_ERR_ALIGN;
  WinArgs a = window_args(B, H, Hkv, T, d, window, sinks, dtype);
  a.q = view_of(q, B, H, T), a.o = view_of(o, B, H, T);
  a.k = view_of(k, B, Hkv, T), a.v = view_of(v, B, Hkv, T);
  a.lse = lse;
  a.lengths = lengths;
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (d) {
    case 16: launch_win_fwd<16>(a, dtype, host_cus(), s); break;
    case 32: launch_win_fwd<32>(a, dtype, host_cus(), s); break;
    case 64: launch_win_fwd<64>(a, dtype, host_cus(), s); break;
    default: launch_win_fwd<128>(a, dtype, host_cus(), s); break;
  }
  return launched();
}

extern "C" int kia_window_bwd(const kia_view *q, const kia_view *k, const kia_view *v,
                              const kia_view *o, const kia_view *dO, const float *lse,
                              const int32_t *lengths, void *ws, const kia_view *dq,
                              const kia_view *dk, const kia_view *dv, int B, int H, int Hkv, int T,
                              int d, int window, int sinks, int dtype, void *stream) {
  int rc = check_window(B, H, Hkv, T, d, window, sinks, dtype);
  if (rc) return rc;
  if (window_too_many(B, H, T)) return KIA_ERR_SHAPE;
  const kia_view *x[8] = {q, o, dO, dq, k, v, dk, dv};
  for (int i = 0; i < 8; ++i) {
    rc = check_view(x[i], B, i < 4 ? H : Hkv, T, d, dtype);
    if (rc) return rc;
  }
  if (!lse || !ws) return KIA_ERR_NULL;
  if (!al16(lse) || (uintptr_t)lengths & 3u || (uintptr_t)ws & 255u) return KIA_ERR_ALIGN;
  WinArgs a = window_args(B, H, Hkv, T, d, window, sinks, dtype);
  a.q = view_of(q, B, H, T), a.o = view_of(o, B, H, T), a.dO = view_of(dO, B, H, T);
  a.dq = view_of(dq, B, H, T);
  a.k = view_of(k, B, Hkv, T), a.v = view_of(v, B, Hkv, T);
  a.dk = view_of(dk, B, Hkv, T), a.dv = view_of(dv, B, Hkv, T);
  a.lse = const_cast<float *>(lse);
  a.lengths = lengths;
  a.delta = static_cast<float *>(ws);
  a.part = a.delta + ((size_t)B * H * T + 63) / 64 * 64;
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (d) {
    case 16: launch_win_bwd<16>(a, dtype, host_cus(), s); break;
    case 32: launch_win_bwd<32>(a, dtype, host_cus(), s); break;
    case 64: launch_win_bwd<64>(a, dtype, host_cus(), s); break;
    default: launch_win_bwd<128>(a, dtype, host_cus(), s); break;
  }
  return launched();
}

// ---- the 4-bit cache ---------------------------------------------------------------
namespace {

int page_log(int page) {
  for (int l = 4; l <= 8; ++l)
    if (page == 1 << l) return l;
  return -1;
}

int check_cache(const void *cache, int pages, int page, const int32_t *table, int width, int B,
                int H, int Hkv, int T, int d, int dtype) {
  int rc = check_common(B, H, Hkv, T, d, dtype, false);
  if (rc) return rc;
  if (page_log(page) < 0) return KIA_ERR_CACHE;
  if (pages < 1 || width < 1 || (int64_t)width * page > INT_MAX) return KIA_ERR_SHAPE;
  if (!cache || !table) return KIA_ERR_NULL;
  if (!al16(cache) || (uintptr_t)table & 3u) return KIA_ERR_ALIGN;
  return KIA_OK;
}

int cache_copy(bool write, const kia_view *k, const kia_view *v, void *cache, int pages, int page,
               const int32_t *table, int width, const int32_t *starts, const int32_t *counts, int B,
               int Hkv, int T, int d, int dtype, void *stream) {
  int rc = check_cache(cache, pages, page, table, width, B, Hkv, Hkv, T, d, dtype);
  if (rc) return rc;
  for (const kia_view *x : {k, v}) {
    rc = check_view(x, B, Hkv, T, d, dtype);
    if (rc) return rc;
  }
  if (!starts) return KIA_ERR_NULL;
  if ((uintptr_t)starts & 3u || (uintptr_t)counts & 3u) return KIA_ERR_ALIGN;
  const int cus = host_cus(), per = cache_tokens(B, Hkv, T, d, cus);
  if (too_many(2.0 * B * Hkv * ((T + per - 1) / per))) return KIA_ERR_SHAPE;
  CacheArgs a{};
  a.cache = static_cast<uint8_t *>(cache);
  a.table = table, a.starts = starts, a.counts = counts;
  a.k = view_of(k, B, Hkv, T), a.v = view_of(v, B, Hkv, T);
  a.pages = pages, a.lpage = page_log(page), a.width = width;
  a.B = B, a.Hkv = Hkv, a.T = T;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (write) timed_call("kia_cache4_write", s, [&] { launch_cache_write(a, d, dtype, cus, s); });
  else timed_call("kia_cache4_read", s, [&] { launch_cache_read(a, d, dtype, cus, s); });
  return launched();
}

// The launch shape: row tiles of 16, and the parts that their keys are cut into, all
// resident at once: three workgroups a CU in bf16, two in fp32 (registers). More parts
// cost more joining than the balance gains (32 sequences of 16 000 keys, 16 heads of 128
// over 4, softmax, bf16: 67 / 59 / 69 us with two / three / six a CU; fp32, 16 sequences: 42
// / 48 with two / three). A part has 128 keys at least, 32 for each wave; up to 256 keys one part, and no
// join (a call alone of 200 keys: bf16 24 us, 28 in two parts, fp32 32 and 34; of 400: 25
// and 28, 35 and 34).
void cached_shape(CachedArgs &a, int dtype, int cus) {
  a.tiles = (a.T * (a.H / a.Hkv) + 15) / 16;
  const int64_t keys = (int64_t)a.width << a.lpage;
  const int64_t most = a.window == INT_MAX
                           ? keys
                           : std::min(keys, (int64_t)a.window + a.T + a.sinks + 64);
  const int64_t groups = (int64_t)a.Hkv * a.tiles, parts = (most + 127) / 128;
  const int64_t want = std::max<int64_t>(1, (dtype == KIA_F32 ? 2 : 3) * cus / groups);
  a.shares = most <= 256 ? 1 : (int)std::min<int64_t>({want, parts * a.B, 255});
}

int check_cached(int H, int Hkv, int K, int calib, float tau, int recon, int window, int sinks) {
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

int cached_args(CachedArgs &a, int pages, int page, int width, int B, int H, int Hkv, int T,
                int window, int sinks, int dtype) {
  a.pages = pages, a.lpage = page_log(page), a.width = width;
  a.B = B, a.H = H, a.Hkv = Hkv, a.T = T;
  a.window = window > 0 ? window : INT_MAX;
  a.sinks = window > 0 ? sinks : 0;
  if ((double)T * (H / Hkv) >= 1 << 24) return KIA_ERR_SHAPE;
  cached_shape(a, dtype, host_cus());
  if (too_many((double)(a.shares + B) * Hkv * a.tiles)) return KIA_ERR_SHAPE;
  if (a.shares > 1 && too_many((double)B * H * T)) return KIA_ERR_SHAPE;  // (the join's)
  return KIA_OK;
}

}  // namespace

extern "C" int kia_cache4_bytes(int pages, int page, int Hkv, int d, size_t *bytes) {
  if (!bytes) return KIA_ERR_NULL;
  *bytes = 0;
  if (page_log(page) < 0) return KIA_ERR_CACHE;
  const int rc = check_common(1, Hkv, Hkv, 1, d, KIA_F32, false);
  if (rc) return rc;
  if (pages < 1) return KIA_ERR_SHAPE;
  *bytes = (size_t)pages * 2 * Hkv * page * (d / 2 + d / 32);
  return KIA_OK;
}

extern "C" int kia_cache4_write(const kia_view *k, const kia_view *v, void *cache, int pages,
                                int page, const int32_t *table, int width, const int32_t *starts,
                                const int32_t *counts, int B, int Hkv, int T, int d, int dtype,
                                void *stream) {
  return cache_copy(true, k, v, cache, pages, page, table, width, starts, counts, B, Hkv, T, d,
                    dtype, stream);
}

extern "C" int kia_cache4_read(const void *cache, int pages, int page, const int32_t *table,
                               int width, const int32_t *starts, const int32_t *counts,
                               const kia_view *k, const kia_view *v, int B, int Hkv, int T, int d,
                               int dtype, void *stream) {
  return cache_copy(false, k, v, const_cast<void *>(cache), pages, page, table, width, starts,
                    counts, B, Hkv, T, d, dtype, stream);
}

extern "C" int kia_cache4_ws_bytes(int page, int width, int B, int H, int Hkv, int T, int d,
                                   int window, int sinks, size_t *bytes) {
  if (!bytes) return KIA_ERR_NULL;
  *bytes = 0;
  int rc = check_common(B, H, Hkv, T, d, KIA_F32, false);
  if (rc) return rc;
  if (H % Hkv) return KIA_ERR_HEADS;
  if (page_log(page) < 0) return KIA_ERR_CACHE;
  if (width < 1 || (int64_t)width * page > INT_MAX || window < 0 || sinks < 0) return KIA_ERR_SHAPE;
  CachedArgs a{};
  // (bf16 takes the more parts)
  rc = cached_args(a, 1, page, width, B, H, Hkv, T, window, sinks, KIA_BF16);
  if (rc) return rc;
  *bytes = cached_layout(a, d).total * 4;
  return KIA_OK;
}

extern "C" int kia_cache4_attn(const kia_view *q, const kia_view *o, const void *cache, int pages,
                               int page, const int32_t *table, int width, const int32_t *lengths,
                               void *ws, int B, int H, int Hkv, int T, int d, int K, int calib,
                               float tau, int recon, int window, int sinks, int dtype,
                               void *stream) {
  int rc = check_cache(cache, pages, page, table, width, B, H, Hkv, T, d, dtype);
  if (!rc) rc = check_cached(H, Hkv, K, calib, tau, recon, window, sinks);
  if (!rc) rc = check_view(q, B, H, T, d, dtype);
  if (!rc) rc = check_view(o, B, H, T, d, dtype);
  if (rc) return rc;
  if (!lengths || !ws) return KIA_ERR_NULL;
  if ((uintptr_t)lengths & 3u || (uintptr_t)ws & 255u) return KIA_ERR_ALIGN;
  CachedArgs a{};
  rc = cached_args(a, pages, page, width, B, H, Hkv, T, window, sinks, dtype);
  if (rc) return rc;
  a.cache = static_cast<const uint8_t *>(cache);
  a.table = table, a.lengths = lengths;
  a.q = view_of(q, B, H, T), a.o = view_of(o, B, H, T);
  const CachedLayout l = cached_layout(a, d);
  float *w = static_cast<float *>(ws);
  a.ext = w + l.ext, a.stat = w + l.stat, a.part = w + l.part;
  a.K = K, a.calib = calib, a.recon = recon, a.tau = tau;
  a.scale = (float)(1.0 / sqrt((double)d));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d == 32) launch_cached<32>(a, dtype, s);
  else if (d == 64) launch_cached<64>(a, dtype, s);
  else launch_cached<128>(a, dtype, s);
  return launched();
}
