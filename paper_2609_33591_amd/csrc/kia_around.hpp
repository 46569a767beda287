// kia_around.hpp -- arguments and launchers of the operators around K-interval
// attention: rotary positions, attention with a sliding window, the 4-bit cache.
#pragma once

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
};
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

}  // namespace kia
