// kia_cached.hpp -- what the kernels that attend over the 4-bit cache share: a lane's share
// of 32 keys and values, their bf16 operands, and the interval weights of its scores.
#pragma once

#include <limits.h>

#include "kia_cache.hpp"

namespace kia {

// 32 keys at a time: two tiles of 16 and the next two on their way leave room for three
// workgroups a CU in bf16 (162 registers; with 64 keys 217, two workgroups, and the
// interval weights of 32 x 16 500 keys took 101 us against 88).
constexpr int TILES = 2, CHUNK = 16 * TILES, NWAVE = 4;
enum { PASS_SOFTMAX, PASS_EXTREMA, PASS_GRID };

__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Where part p of `parts` begins: count * p / parts, without a product of more than 32 bits
// (p <= parts < 2^15).
__device__ __forceinline__ int share_of(int count, unsigned p, unsigned parts) {
  const unsigned q = (unsigned)count / parts, rest = (unsigned)count % parts;
  return (int)(q * p + rest * p / parts);
}

// One lane's share of a chunk: codes and scales of its keys and values.
template <int D, bool VALUES> struct Stage4 {
  static constexpr int N = D / 32;  // words of codes of a 16-key tile
  uint32_t k[TILES][N], v[VALUES ? TILES : 1][N], vs[VALUES ? TILES : 1];
  uint8_t ks[TILES];
  int at[TILES];  // the tiles' first keys
  int ok;         // bit t: the tile's page is one of the cache's
  // the values of token e (of the lane's four) of tile i as zeros
  __device__ __forceinline__ void clear(int i, int e) {
    vs[i] &= ~(0xffu << (8 * e));
    if constexpr (D == 128) v[i][e] = 0;
    else if constexpr (D == 64) v[i][e / 2] &= ~(0xffffu << (16 * (e % 2)));
    else v[i][0] &= ~(0xffu << (8 * e));
  }
};
template <int N> __device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const u32x4 x = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
  } else if constexpr (N == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
    w[0] = x[0], w[1] = x[1];
  } else {
    w[0] = *reinterpret_cast<const uint32_t *>(p);
  }
}

// Eight channels of a query as operands: channel block c of its NP pieces.
template <typename TI, int NP, int N>
__device__ __forceinline__ void load_query(const TI *p, bf16x8 (&q)[NP][N], int c) {
  if constexpr (NP == 1) {
    q[0][c] = as_op(*reinterpret_cast<const u32x4 *>(p));
  } else {
    float x[8];
    load8(p, x);
    bf16x8 y[3];
    to_pieces<3>(x, y);
#pragma unroll
    for (int i = 0; i < 3; ++i) q[i][c] = y[i];
  }
}

// An entry of a table at an index that all lanes have, by a scalar load: a vector load would have
// the loop wait for what it asked for before, the next keys among it.
__device__ __forceinline__ int entry_of(const int *table, int64_t i) {
  return ((const __attribute__((address_space(4))) int *)table)[i];
}

// Where a lane's share of a tile stands behind what all lanes have of its address.
template <int D> struct Offsets {
  uint32_t k, ks, v, vs;  // bytes
  __device__ __forceinline__ explicit Offsets(uint32_t lane) {
    const uint32_t kb = lane >> 4, slot = lane & 15;
    k = slot * (D / 2) + kb * (D / 8), ks = slot * (D / 32) + kb * (D / 4) / 32;
    v = lane * (D / 8), vs = kb * (D / 8) + slot * (D / 16) / 32 * 4;
  }
  // (once a turn of a loop: known to stay the same they would be kept in 64 bits and added to
  // the address, where a load takes 32 bits beside a scalar one)
  __device__ __forceinline__ void hold() { asm volatile("" : "+v"(k), "+v"(ks), "+v"(v), "+v"(vs)); }
};

// A lane's share of tile i, tokens tok .. tok + 15 of a page, of which kp is a head's block of
// keys and `values` bytes on that of its values (codes: bytes of a block's codes).
template <int D, bool VALUES>
__device__ __forceinline__ void load_tile(const uint8_t *kp, int64_t values, int tok, int codes, const Offsets<D> &at,
                                          int i, Stage4<D, VALUES> &x) {
  constexpr int N = D / 32;
  const uint8_t *k = kp + tok * (D / 2), *s = kp + codes + tok * (D / 32);
  load_words<N>(k + at.k, x.k[i]);
  x.ks[i] = s[at.ks];
  if constexpr (VALUES) {
    load_words<N>(k + values + at.v, x.v[i]);
    x.vs[i] = *reinterpret_cast<const uint32_t *>(s + values + at.vs);
  }
}

// Whether a lane's share has a group that holds an infinity or NaN.
template <int D, bool VALUES> __device__ __forceinline__ bool holds_nan(const Stage4<D, VALUES> &x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    bad |= x.ks[i] == 255;
    if constexpr (VALUES) {
      const uint32_t y = ~x.vs[i];
      bad |= ((y - 0x01010101u) & ~y & 0x80808080u) != 0;
    }
  }
  return bad;
}

// Operands of the values of 32 keys (tiles 2 u and 2 u + 1, f: their scales) in two of the
// lane's channels.
template <int D>
__device__ __forceinline__ void value_ops(const Stage4<D, true> &x, const float (&f)[8], int u, int y, u32x4 &even,
                                          u32x4 &odd) {
  uint32_t z[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = 2 * u + e / 4, k = e % 4;
    z[e] = pair_at(D == 128 ? y : D == 64 ? 2 * (k % 2) + y : k, x.v[i][D == 128 ? k : D == 64 ? k / 2 : 0], f[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    even[e] = __builtin_amdgcn_perm(z[2 * e + 1], z[2 * e], 0x05040100u);
    odd[e] = __builtin_amdgcn_perm(z[2 * e + 1], z[2 * e], 0x07060302u);
  }
}

// The weights w of scores S on the row's grid.
template <int CALIB, int RECON, int NE>
__device__ __forceinline__ void grid_weights(const float (&S)[TILES][NE], float (&w)[TILES][NE],
                                             const RowConst &rc, float Mx, float Mn, const CachedArgs &a) {
  const float Kf = (float)a.K, edge = 2.f * Kf - 1.f, span = 1.f - rc.emh;
  bool any = false;
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      w[i][e] = fmaf(S[i][e], rc.alpha, rc.beta);
      any |= is_ambiguous<CALIB>(w[i][e], rc.margin2, edge);
    }
  if (__any(any)) {
    // keys within rounding of a boundary: decided in 64 bits
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const bool amb = is_ambiguous<CALIB>(w[i][e], rc.margin2, edge);
        if (!__any(amb)) continue;
        const float x = 0.5f * exact_v2<CALIB>(S[i][e] * a.scale, 2.f * w[i][e], Mx, Mn, a.K, a.tau);
        w[i][e] = amb ? x : w[i][e];
      }
  }
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const KeyDec k = key_of<CALIB>(w[i][e], Kf);
      const float up = grid_upper(k.rf, rc);
      float x;
      if constexpr (RECON == REC_NEAREST) x = k.up ? up : up * rc.emh;
      else x = up * fmaf(k.t, span, rc.emh);
      x = k.tail ? 0.f : x;
      // an infinite or NaN score makes its row NaN
      x = fabsf(S[i][e]) < INFINITY ? x : NAN;
      w[i][e] = x;
    }
}

}  // namespace kia
