// kia_around.hpp -- arguments and launchers of the operators around K-interval
// attention: rotary positions, attention with a sliding window, the 4-bit cache.
#pragma once

#include <algorithm>

#include "kia.h"
#include "kia_device.hpp"

namespace kia {

// A [B, heads, T, d] tensor whose rows are contiguous (strides in elements).
struct View {
  void *p = nullptr;
  int64_t sb = 0, sh = 0, st = 0;
};
template <typename TI> __device__ __forceinline__ TI *slice_of(const View &v, int b, int h) {
  return static_cast<TI *>(v.p) + b * v.sb + h * v.sh;
}

// A value of all 64 lanes, by rotations of 16 and then from lane to scalar.
template <int CTRL> __device__ __forceinline__ uint32_t rotated(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
}
template <class F> __device__ __forceinline__ uint32_t over16(uint32_t x, F f) {
  x = f(x, rotated<0x128>(x));  // row_ror 8, 4, 2, 1
  x = f(x, rotated<0x124>(x));
  x = f(x, rotated<0x122>(x));
  return f(x, rotated<0x121>(x));
}
template <class F> __device__ __forceinline__ uint32_t over64(uint32_t x, F f) {
  x = over16(x, f);
  const uint32_t y[4] = {(uint32_t)__builtin_amdgcn_readlane((int)x, 0), (uint32_t)__builtin_amdgcn_readlane((int)x, 16),
                         (uint32_t)__builtin_amdgcn_readlane((int)x, 32), (uint32_t)__builtin_amdgcn_readlane((int)x, 48)};
  return f(f(y[0], y[1]), f(y[2], y[3]));
}
struct Sum { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a + b; } };
// The sum of the lanes before a lane, and its own.
__device__ __forceinline__ uint32_t sum_to(uint32_t x) {
  x += rotated<0x111>(x);  // row_shr 1, 2, 4, 8 (zeros come in)
  x += rotated<0x112>(x);
  x += rotated<0x114>(x);
  x += rotated<0x118>(x);
  const uint32_t a = __builtin_amdgcn_readlane((int)x, 15), b = __builtin_amdgcn_readlane((int)x, 31),
                 c = __builtin_amdgcn_readlane((int)x, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return x + (row > 0 ? a : 0) + (row > 1 ? b : 0) + (row > 2 ? c : 0);
}

// ---- rotary positions (kia_rotary.hip) ----------------------------------------
struct RotSide {
  const void *x;
  void *y;
  int64_t xb, xh, xt, yb, yh, yt;
};
struct RotArgs {
  RotSide q, k;  // Hkv = 0: no keys
  const int *pos;  // or nullptr: first + t
  int64_t pos_sb;
  const double *freq;
  float factor;
  int first, layout, back, B, H, Hkv, T, d, rot;
  int tokens, per;  // tokens of a workgroup, rounds of heads of a share (the launcher's)
};
// Sine and cosine of the angle p * freq, to a quarter turn in 64 bits and from there in 32.
__device__ __forceinline__ void turn_of(double p, double freq, float &s, float &c) {
  // quarter turns: q whole ones and a rest of at most a half
  const double x = p * freq * 0.63661977236758134308;
  const double q = rint(x);
  sincospif(0.5f * (float)(x - q), &s, &c);
  // (a large q is a multiple of 4 plus these bits whatever its size)
  const int k = (int)(q - 4.0 * floor(q * 0.25));
  if (k & 1) { const float y = s; s = c; c = -y; }
  if (k & 2) { s = -s; c = -c; }
}
// Tokens of a workgroup, and the channels of an access (vw): the widest whose pairs fill
// whole chunks (16 bytes for most plans; a rotated part of 2 mod 4 channels takes
// single values).
constexpr int ROT_NT = 256;
inline int rotary_tokens(int T, int d, int rot, int dtype, int &vw) {
  vw = dtype == KIA_F32 ? 4 : 8;
  while (rot / 2 % vw) vw /= 2;
  int tokens = 1;
  while (2 * tokens <= T && tokens < 8 && 2 * tokens * (d / (2 * vw)) <= ROT_NT) tokens *= 2;
  return tokens;
}
void launch_rotary(RotArgs a, int dtype, int cus, hipStream_t s);

// ---- attention with a sliding window (kia_window.hip) ---------------------------
struct WinArgs {
  View q, k, v, o, dO, dq, dk, dv;
  float *lse, *delta, *part;
  const int *lengths;
  int B, H, Hkv, T, window, sinks;
  float scale;
  // the key blocks' query ranges: blocks that hold first tokens, and the parts that
  // each block of either kind is cut into
  int sink_blocks, parts_a, parts_b;
};
constexpr int WIN_KB = 64;  // keys of a block of the key gradients
constexpr int WIN_QT = 64;  // queries of one step there

// Partial sums that the key blocks of one key head leave (blocks of one part leave none).
__host__ __device__ inline int win_slots(int nkb, int sb, int pa, int pb) {
  return (pa > 1 ? sb * pa : 0) + (pb > 1 ? (nkb - sb) * pb : 0);
}
template <int D> void launch_win_fwd(const WinArgs &a, int dtype, int cus, hipStream_t s);
template <int D> void launch_win_bwd(const WinArgs &a, int dtype, int cus, hipStream_t s);

// ---- the 4-bit cache (kia_cache.hip) --------------------------------------------
struct CacheArgs {
  uint8_t *cache;
  const int *table, *starts, *counts;  // counts: new tokens of each sequence, or nullptr
  View k, v;                           // the tokens to hold, or where to read them to
  int pages, lpage, width, B, Hkv, T;  // lpage: log2 of the tokens of a page
};
// Tokens of a head that a workgroup writes or reads: four a thread where that still leaves
// eight workgroups a CU.
inline int cache_tokens(int B, int Hkv, int T, int d, int cus) {
  const int one = 256 * 8 / d;
  return 2.0 * B * Hkv * T / (4 * one) >= 8.0 * cus ? 4 * one : one;
}
void launch_cache_write(const CacheArgs &a, int d, int dtype, int cus, hipStream_t s);
void launch_cache_read(const CacheArgs &a, int d, int dtype, int cus, hipStream_t s);

// ---- appended tokens and the bounds of pages (kia_append.hip) -----------------------
struct AppendArgs {
  CacheArgs c;
  View q, qo;
  uint32_t *bounds;  // [pages][Hkv][2][d] bf16, or nullptr
  const double *freq;
  float factor;
  int layout, rot, H;
  int spans;  // of a sequence's new tokens: 64 positions or a page, whichever is more
  int kshares, vshares;  // shares of the key heads' keys and values (the launcher's)
};
inline int append_spans(int T, int lpage) {
  const int l = lpage > 6 ? lpage : 6;
  return ((T - 1 + (1 << l) - 1) >> l) + 1;
}
void launch_append(AppendArgs a, int d, int dtype, int cus, hipStream_t s);
void launch_bounds(const AppendArgs &a, int d, hipStream_t s);

// ---- selected pages (kia_select.hip) ------------------------------------------------
struct SelectArgs {
  const uint32_t *bounds;
  const int *table, *lengths;
  View q;
  void *ws;   // select_space(width) bytes for each of [B][Hkv][T]
  int *list;  // [B][Hkv][T][count]
  int pages, lpage, width, B, H, Hkv, T;
  int count, first, last;
  bool own;   // a workgroup ranks the pages that it selects from
  int batch;  // else: pages that one ranks, 64 at least
};
constexpr int SELECT_OWN = 1024;  // pages that it can
__host__ __device__ inline size_t select_space(int width) {
  return ((size_t)width * 12 + ((size_t)width + 63) / 64 * 16 + 7) / 8 * 8;
}
void launch_select(const SelectArgs &a, int d, int dtype, hipStream_t s);

// ---- attention over the cache (kia_cached.hip) ----------------------------------------
// The rows of all sequences over the tokens that they share: b T G + t G + g is the row of
// token t and head g of the group, in 16-row tiles.
struct Prefix {
  float *ext, *stat, *part;  // as CachedArgs'
  int tiles, parts;
  unsigned blocks;  // workgroups
  __host__ __device__ int64_t slot(int hk, unsigned row) const {
    return (((int64_t)hk * tiles + row / 16) * parts) * 16 + row % 16;
  }
};
// Row tiles that a wave takes.
inline int prefix_tiles(int tiles, int d, int dtype) {
  return tiles == 1 || (d == 128 && dtype == KIA_F32) ? 1 : 2;
}
struct CachedArgs {
  const uint8_t *cache;
  const int *table, *lengths;
  View q, o;
  float *ext, *stat, *part;  // workspace (cached_layout)
  int pages, lpage, width, B, H, Hkv, T;
  int window, sinks;  // window: INT_MAX where there is none
  int K, calib, recon;
  float tau, scale;
  int tiles, shares;  // 16-row tiles of a key head's rows, parts of its keys (< 256)
  // Over listed pages, and over what lies behind shared tokens: `tiles` of a token's, or a
  // sequence's, rows, `parts` for each, `shares` in all for a row tile. With `spread` (about
  // so many in all) the sequences have parts by their lengths, up to `most`, and `parts` is the
  // usual number. Which, is found by every workgroup, or of more than PLANNED_FROM sequences by a
  // launch before the others:
  int parts, spread, most;
  int4 *plan;  // [tiles][shares]: a part's sequence (-1: none), that one's first part, parts and keys
  int2 *own;   // [tiles][B]: a sequence's first part, and parts
  const int *list;  // [B][Hkv][T][count]
  int count;
  int shared;  // tokens
  Prefix pre;
};
// Entries of a list that one part takes, at most.
constexpr int LISTED_MOST = 1024;
// A row's parts are joined by a workgroup, or, where up to FEW_PARTS are usual and there are many
// rows, by D / 4 lanes.
constexpr int FEW_PARTS = 8, MANY_ROWS = 2048;
// (A launch takes 3 to 4 us and a walk over 64 sequences' lengths 1 to 2, but of all workgroups: 16
// sequences behind 2048 tokens, up to 4000 of their own, 21 us planned and 18 by each; 256 behind 2048, 200
// of their own, LERP, 45 and 49; 1024, softmax, 88 and 150.)
constexpr int PLANNED_FROM = 64;
// Floats of the workspace: the parts' extrema, their maxima and sums, their rows.
struct CachedLayout {
  size_t ext, stat, part, total;
};
inline CachedLayout cached_layout(const CachedArgs &a, int d) {
  const size_t n = (size_t)(a.shares + a.B) * a.Hkv * a.tiles * 16;
  CachedLayout l;
  l.ext = 0;
  l.stat = 2 * n;
  l.part = 4 * n;
  l.total = 4 * n + n * d;
  return l;
}
template <int D> void launch_cached(const CachedArgs &a, int dtype, hipStream_t s);
template <int D> void launch_listed(const CachedArgs &a, int dtype, hipStream_t s);
template <int D> void launch_shared(const CachedArgs &a, int dtype, hipStream_t s);

}  // namespace kia
