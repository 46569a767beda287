// kia_serve_abi.hip -- extern "C" entry points of the operators that serve many and long
// texts from the 4-bit cache (declared in include/kia.h). Host side only: argument checks
// before any launch, workspace sizes, launch shapes, launches on the caller's stream.
#include "kia_checks.hpp"
#include "kia_host.hpp"

using namespace kia;

// ---- appended tokens and the bounds of pages -----------------------------------------
extern "C" int kia_cache4_append(const kia_view *q, const kia_view *q_out, const kia_view *k,
                                 const kia_view *v, void *cache, void *bounds, int pages, int page,
                                 const int32_t *table, int width, const int32_t *starts,
                                 const int32_t *counts, const double *freq, float factor, int layout, int B,
                                 int H, int Hkv, int T, int d, int rot, int dtype, void *stream) {
  int rc = check_cache(cache, pages, page, table, width, B, H, Hkv, T, d, dtype);
  if (rc) return rc;
  if (rot < 2 || rot > d || rot % 2) return KIA_ERR_HEADDIM;
  if (layout != KIA_ROTARY_HALF && layout != KIA_ROTARY_NEIGHBOURS) return KIA_ERR_ENUM;
  if (T > 1 << 24 || (int64_t)H + 2 * (int64_t)Hkv > 65535) return KIA_ERR_SHAPE;
  const kia_view *x[4] = {q, q_out, k, v};
  for (int i = 0; i < 4; ++i) {
    rc = check_view(x[i], B, i < 2 ? H : Hkv, T, d, dtype);
    if (rc) return rc;
  }
  if (!starts || !freq) return KIA_ERR_NULL;
  if ((uintptr_t)starts & 3u || (uintptr_t)counts & 3u || (uintptr_t)freq & 7u || !al16(bounds))
    return KIA_ERR_ALIGN;
  AppendArgs a{};
  a.c.pages = pages, a.c.lpage = page_log(page), a.c.width = width;
  a.c.B = B, a.c.Hkv = Hkv, a.c.T = T;
  a.spans = append_spans(T, a.c.lpage);
  // (workgroups of up to 512 threads)
  if (too_many(2.0 * B * a.spans)) return KIA_ERR_SHAPE;
  a.c.cache = static_cast<uint8_t *>(cache);
  a.c.table = table, a.c.starts = starts, a.c.counts = counts;
  a.c.k = view_of(k, B, Hkv, T), a.c.v = view_of(v, B, Hkv, T);
  a.q = view_of(q, B, H, T), a.qo = view_of(q_out, B, H, T);
  a.bounds = static_cast<uint32_t *>(bounds);
  a.freq = freq, a.factor = factor, a.layout = layout, a.rot = rot, a.H = H;
  hipStream_t s = static_cast<hipStream_t>(stream);
  timed_call("kia_cache4_append", s, [&] { launch_append(a, d, dtype, host_cus(), s); });
  return launched();
}

extern "C" int kia_cache4_bounds(const void *cache, void *bounds, int pages, int page, const int32_t *table,
                                 int width, const int32_t *starts, const int32_t *ends, int B, int Hkv,
                                 int d, void *stream) {
  const int rc = check_cache(cache, pages, page, table, width, B, Hkv, Hkv, 1, d, KIA_BF16);
  if (rc) return rc;
  if (!bounds || !starts || !ends) return KIA_ERR_NULL;
  if ((uintptr_t)starts & 3u || (uintptr_t)ends & 3u || !al16(bounds)) return KIA_ERR_ALIGN;
  AppendArgs a{};
  a.c.pages = pages, a.c.lpage = page_log(page), a.c.width = width;
  a.c.B = B, a.c.Hkv = Hkv;
  const int64_t span = std::max(page, 64);
  a.spans = (int)(((int64_t)width * page + span - 1) / span);
  if (too_many(2.0 * B * Hkv * a.spans)) return KIA_ERR_SHAPE;
  a.c.cache = static_cast<uint8_t *>(const_cast<void *>(cache));
  a.c.table = table, a.c.starts = starts, a.c.counts = ends;
  a.bounds = static_cast<uint32_t *>(bounds);
  hipStream_t s = static_cast<hipStream_t>(stream);
  timed_call("kia_cache4_bounds", s, [&] { launch_bounds(a, d, s); });
  return launched();
}

// ---- selected pages --------------------------------------------------------------------
namespace {

int check_select(int page, int width, int B, int H, int Hkv, int T, int d, int count) {
  const int rc = check_common(B, H, Hkv, T, d, KIA_BF16, false);
  if (rc) return rc;
  if (H % Hkv) return KIA_ERR_HEADS;
  if (page_log(page) < 0) return KIA_ERR_CACHE;
  if (width < 1 || (int64_t)width * page > INT_MAX || count < 1) return KIA_ERR_SHAPE;
  if ((int64_t)(H / Hkv) * d * 4 > 32768) return KIA_ERR_SHAPE;  // (a token's rows in LDS)
  // (batches of 64 pages; selections of up to 1024 threads)
  if (too_many((double)B * Hkv * T * std::max(4, (width + 63) / 64))) return KIA_ERR_SHAPE;
  return KIA_OK;
}

}  // namespace

extern "C" int kia_cache4_select_ws_bytes(int page, int width, int B, int H, int Hkv, int T, int d,
                                          size_t *bytes) {
  if (!bytes) return KIA_ERR_NULL;
  *bytes = 0;
  const int rc = check_select(page, width, B, H, Hkv, T, d, 1);
  if (rc) return rc;
  *bytes = (size_t)B * Hkv * T * select_space(width);
  return KIA_OK;
}

extern "C" int kia_cache4_select(const kia_view *q, const void *bounds, int pages, int page,
                                 const int32_t *table, int width, const int32_t *lengths, void *ws,
                                 int32_t *list, int count, int first, int last, int B, int H, int Hkv,
                                 int T, int d, int dtype, void *stream) {
  int rc = check_cache(bounds, pages, page, table, width, B, H, Hkv, T, d, dtype);
  if (!rc) rc = check_select(page, width, B, H, Hkv, T, d, count);
  if (!rc) rc = check_view(q, B, H, T, d, dtype);
  if (rc) return rc;
  if (first < 0 || last < 1 || (int64_t)first + last > count) return KIA_ERR_SHAPE;
  if (!lengths || !ws || !list) return KIA_ERR_NULL;
  if ((uintptr_t)lengths & 3u || (uintptr_t)list & 3u || (uintptr_t)ws & 255u) return KIA_ERR_ALIGN;
  SelectArgs a{};
  a.bounds = static_cast<const uint32_t *>(bounds);
  a.table = table, a.lengths = lengths;
  a.q = view_of(q, B, H, T);
  a.ws = ws;
  a.list = list;
  a.pages = pages, a.lpage = page_log(page), a.width = width;
  a.B = B, a.H = H, a.Hkv = Hkv, a.T = T;
  a.count = count, a.first = first, a.last = last;
  // A workgroup pulls some 30 GB/s of bounds: it ranks up to 100 KB of them itself, or where
  // there is one for every CU. Else workgroups of a launch of their own, two for a CU, do.
  const int64_t tokens = (int64_t)B * Hkv * T;
  a.own = width <= SELECT_OWN && ((int64_t)width * d <= 25600 || tokens >= host_cus());
  a.batch = 64;
  while (a.batch < 1024 && tokens * ((width + a.batch - 1) / a.batch) > 2 * host_cus()) a.batch *= 2;
  launch_select(a, d, dtype, static_cast<hipStream_t>(stream));
  return launched();
}

// ---- attention over selected pages, and behind shared tokens -----------------------------
namespace {

struct Operator {
  int K, calib, recon;
  float tau;
};

// What both calls check, and fill, alike.
int served_args(CachedArgs &a, const kia_view *q, const kia_view *o, const void *cache, int pages, int page,
                const int32_t *table, int width, const int32_t *lengths, void *ws, int B, int H, int Hkv, int T,
                int d, Operator op, int dtype) {
  int rc = check_cache(cache, pages, page, table, width, B, H, Hkv, T, d, dtype);
  if (!rc) rc = check_cached(H, Hkv, op.K, op.calib, op.tau, op.recon, 0, 0);
  if (!rc) rc = check_view(q, B, H, T, d, dtype);
  if (!rc) rc = check_view(o, B, H, T, d, dtype);
  if (rc) return rc;
  if (!lengths || !ws) return KIA_ERR_NULL;
  if ((uintptr_t)lengths & 3u || (uintptr_t)ws & 255u) return KIA_ERR_ALIGN;
  a.cache = static_cast<const uint8_t *>(cache);
  a.table = table, a.lengths = lengths;
  a.q = view_of(q, B, H, T), a.o = view_of(o, B, H, T);
  a.pages = pages;
  a.K = op.K, a.calib = op.calib, a.recon = op.recon, a.tau = op.tau;
  a.scale = (float)(1.0 / sqrt((double)d));
  return KIA_OK;
}

int check_sizes(CachedArgs &a, int page, int width, int B, int H, int Hkv, int T, int d) {
  const int rc = check_common(B, H, Hkv, T, d, KIA_BF16, false);
  if (rc) return rc;
  if (H % Hkv) return KIA_ERR_HEADS;
  if (page_log(page) < 0) return KIA_ERR_CACHE;
  if (width < 1 || (int64_t)width * page > INT_MAX) return KIA_ERR_SHAPE;
  if ((double)B * H * T >= 1 << 24) return KIA_ERR_SHAPE;  // (the join's workgroups)
  a.lpage = page_log(page), a.width = width;
  a.B = B, a.H = H, a.Hkv = Hkv, a.T = T;
  a.window = INT_MAX, a.sinks = 0;
  return KIA_OK;
}

// Extrema, maxima and sums, and rows of `n` parts' rows, from `at` on (ws nullptr: their size).
size_t lay(size_t at, size_t n, int d, float *ws, float *&ext, float *&stat, float *&part) {
  if (ws) ext = ws + at, stat = ext + 2 * n, part = stat + 2 * n;
  return at + (4 + (size_t)d) * n;
}

// Workgroups that the chip holds at once, about (see cached_shape of kia_around_abi.hip): heads of 128
// in their softmax and, with up to four heads a group, their weights; with more a group in bf16 some
// weights' forms have two. Smaller heads and the extrema have up to eight.
int64_t resident(int dtype) { return (int64_t)(dtype == KIA_F32 ? 2 : 3) * host_cus(); }

// Selected pages: every token's list in as many parts as fill the chip, of 128 keys at least
// and of LISTED_MOST pages at most.
int pages_shape(CachedArgs &a, int page, int width, int B, int H, int Hkv, int T, int d, int count, int dtype) {
  const int rc = check_sizes(a, page, width, B, H, Hkv, T, d);
  if (rc) return rc;
  const int64_t keys = (int64_t)count * page;
  if (count < 1 || keys > INT_MAX || count > 200000) return KIA_ERR_SHAPE;
  a.count = count;
  a.tiles = (H / Hkv + 15) / 16;
  const int64_t groups = (int64_t)B * T * Hkv * a.tiles, want = std::max<int64_t>(1, resident(dtype) / groups);
  const int64_t most = std::min<int64_t>((keys + 127) / 128, 255);
  a.parts = keys <= 256 ? 1 : (int)std::max<int64_t>(std::min(want, most), count / 1000 + 1);
  if (too_many((double)groups * a.parts)) return KIA_ERR_SHAPE;
  a.shares = B * T * a.parts;
  return KIA_OK;
}
size_t pages_lay(CachedArgs &a, int d, float *ws) {
  return lay(0, (size_t)a.shares * a.Hkv * a.tiles * 16, d, ws, a.ext, a.stat, a.part);
}

// Shared tokens: the rows of all sequences over them in parts that fill the chip, and each
// sequence's over what lies behind: as many parts for each, or, where the table has room for texts
// that pass the shared tokens by more than SPREAD_FROM, about as many in all by the lengths (256
// sequences behind 8192 tokens, 200 of their own and one 100 000, softmax: 63 us, with its own in one part
// 657, without shared tokens 214; one 30 000: 54 and 214; one 4000: as many parts for each 52, by lengths
// 49). Where all are short in such a table finding the parts costs 0 to 6 us: 41 -> 45 for those 256, 21 ->
// 25 for 64 of up to 1000; of thousands a tenth (2048 behind 2048: 154 -> 171).
constexpr int SPREAD_FROM = 4096;
int shared_shape(CachedArgs &a, int page, int width, int B, int H, int Hkv, int T, int d, int shared, int dtype) {
  const int rc = check_sizes(a, page, width, B, H, Hkv, T, d);
  if (rc) return rc;
  const int64_t keys = (int64_t)width * page;
  if (shared < 1 || shared % std::max(page, 32) || shared > keys) return KIA_ERR_SHAPE;
  a.shared = shared;
  const int G = H / Hkv;
  a.tiles = (T * G + 15) / 16;
  // Two workgroups a CU run at once (of two row tiles in heads of 128; smaller heads and the extrema
  // have two to eight): those over the shared tokens get their part of the work's
  // worth of that (a chunk of two row tiles costs 1.6 times one of one), half of it at least
  // (64 sequences behind 8192 tokens, 1000 of their own at most: with all of it 29.5 us, so 25).
  const int64_t groups = (int64_t)B * Hkv * a.tiles, own = keys - shared, cus = host_cus();
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>({2 * cus / groups, (own + 255) / 256, 64}));
  // (a begun part a sequence is half of one; of many sequences no more than run at once beside theirs)
  if (own > SPREAD_FROM)
    a.spread = (int)std::max<int64_t>(1, std::min<int64_t>(B * a.parts - B / 2, 2 * cus / ((int64_t)Hkv * a.tiles)));
  a.shares = a.spread ? a.spread + B : B * a.parts;
  a.pre.tiles = (int)(((int64_t)B * T * G + 15) / 16);
  const int rt = prefix_tiles(a.pre.tiles, d, dtype);
  const int64_t blocks = (int64_t)Hkv * ((a.pre.tiles + rt - 1) / rt);
  const double work = 0.8 * Hkv * a.pre.tiles * shared, rest = (double)groups * own;
  const int64_t slots = (int64_t)(2.0 * cus * std::max(0.5, work / (work + rest)));
  a.pre.parts = (int)std::max<int64_t>(
      1, std::min<int64_t>({(slots + blocks / 2) / blocks, ((int64_t)shared + 127) / 128, 128}));
  if (too_many((double)a.shares * Hkv * a.tiles + (double)blocks * a.pre.parts)) return KIA_ERR_SHAPE;
  a.pre.blocks = (unsigned)(blocks * a.pre.parts);
  // (a join of up to 256 parts by a workgroup, or of not too many by a few lanes)
  a.most = (int64_t)B * H * T >= MANY_ROWS && a.parts + a.pre.parts <= FEW_PARTS ? 24 : 127;
  return KIA_OK;
}
size_t shared_lay(CachedArgs &a, int d, float *ws) {
  const size_t at = lay(0, (size_t)a.shares * a.Hkv * a.tiles * 16, d, ws, a.ext, a.stat, a.part);
  const size_t end = lay(at, (size_t)a.Hkv * a.pre.tiles * 16 * a.pre.parts, d, ws, a.pre.ext, a.pre.stat, a.pre.part);
  if (!a.spread) return end;
  const size_t entries = a.B > PLANNED_FROM ? (size_t)a.tiles * a.shares : 0;
  if (ws && entries) a.plan = reinterpret_cast<int4 *>(ws + end);
  if (ws) a.own = reinterpret_cast<int2 *>(ws + end + 4 * entries);
  return end + 4 * entries + 2 * (size_t)a.tiles * a.B;
}

}  // namespace

extern "C" int kia_cache4_pages_ws_bytes(int page, int width, int count, int B, int H, int Hkv, int T, int d,
                                         size_t *bytes) {
  if (!bytes) return KIA_ERR_NULL;
  *bytes = 0;
  for (int dtype : {KIA_F32, KIA_BF16}) {
    CachedArgs a{};
    const int rc = pages_shape(a, page, width, B, H, Hkv, T, d, count, dtype);
    if (rc) return rc;
    *bytes = std::max(*bytes, pages_lay(a, d, nullptr) * 4);
  }
  return KIA_OK;
}

extern "C" int kia_cache4_attn_pages(const kia_view *q, const kia_view *o, const void *cache, int pages, int page,
                                     const int32_t *table, int width, const int32_t *lengths, const int32_t *list,
                                     int count, void *ws, int B, int H, int Hkv, int T, int d, int K, int calib,
                                     float tau, int recon, int dtype, void *stream) {
  CachedArgs a{};
  int rc = served_args(a, q, o, cache, pages, page, table, width, lengths, ws, B, H, Hkv, T, d,
                       Operator{K, calib, recon, tau}, dtype);
  if (!rc) rc = pages_shape(a, page, width, B, H, Hkv, T, d, count, dtype);
  if (rc) return rc;
  if (!list) return KIA_ERR_NULL;
  if ((uintptr_t)list & 3u) return KIA_ERR_ALIGN;
  a.list = list;
  pages_lay(a, d, static_cast<float *>(ws));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d == 32) launch_listed<32>(a, dtype, s);
  else if (d == 64) launch_listed<64>(a, dtype, s);
  else launch_listed<128>(a, dtype, s);
  return launched();
}

extern "C" int kia_cache4_shared_ws_bytes(int page, int width, int shared, int B, int H, int Hkv, int T, int d,
                                          size_t *bytes) {
  if (!bytes) return KIA_ERR_NULL;
  *bytes = 0;
  for (int dtype : {KIA_F32, KIA_BF16}) {
    CachedArgs a{};
    const int rc = shared_shape(a, page, width, B, H, Hkv, T, d, shared, dtype);
    if (rc) return rc;
    *bytes = std::max(*bytes, shared_lay(a, d, nullptr) * 4);
  }
  return KIA_OK;
}

extern "C" int kia_cache4_attn_shared(const kia_view *q, const kia_view *o, const void *cache, int pages, int page,
                                      const int32_t *table, int width, const int32_t *lengths, int shared, void *ws,
                                      int B, int H, int Hkv, int T, int d, int K, int calib, float tau, int recon,
                                      int dtype, void *stream) {
  CachedArgs a{};
  int rc = served_args(a, q, o, cache, pages, page, table, width, lengths, ws, B, H, Hkv, T, d,
                       Operator{K, calib, recon, tau}, dtype);
  if (!rc) rc = shared_shape(a, page, width, B, H, Hkv, T, d, shared, dtype);
  if (rc) return rc;
  shared_lay(a, d, static_cast<float *>(ws));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d == 32) launch_shared<32>(a, dtype, s);
  else if (d == 64) launch_shared<64>(a, dtype, s);
  else launch_shared<128>(a, dtype, s);
  return launched();
}
