// kia_cache.hpp -- the layout of the 4-bit key/value cache (documented in kia.h), and
// eight channels of a token on their way into it and back.
#pragma once

#include "kia_around.hpp"

namespace kia {

// Byte offset of one head's block of a page: which = 0 its keys, 1 its values.
// A block is codes (D / 2 bytes a token), then scale bytes (D / 32 a token).
template <int D>
__device__ __forceinline__ int64_t cache_block(int page, int which, int h, int Hkv, int lpage) {
  return (((int64_t)page * 2 + which) * Hkv + h) * (int64_t)((D / 2 + D / 32) << lpage);
}

template <typename TI> __device__ __forceinline__ void load8(const TI *p, float (&x)[8]) {
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const f32x4 v = load4(p + 4 * g);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * g + e] = v[e];
  }
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
#pragma unroll
  for (int g = 0; g < 2; ++g)
    *reinterpret_cast<f32x4 *>(p + 4 * g) =
        f32x4{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = cvt_bf16x2(x[2 * e], x[2 * e + 1]);
  *reinterpret_cast<u32x4 *>(p) = w;
}

// Codes of eight values in units of their group's scale (to the nearest level, an even
// one between two, at most 6), and the values of eight codes: an instruction a pair.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8]) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], 1.f, 3);
}
template <int S> __device__ __forceinline__ void pair_of(uint32_t w, float f, float (&x)[8]) {
  const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, S);
  x[2 * S] = v[0] * f;
  x[2 * S + 1] = v[1] * f;
}
__device__ __forceinline__ void values_of(uint32_t w, float f, float (&x)[8]) {
  pair_of<0>(w, f, x);
  pair_of<1>(w, f, x);
  pair_of<2>(w, f, x);
  pair_of<3>(w, f, x);
}

// byte `s` of a word of codes as two bf16
template <int S> __device__ __forceinline__ uint32_t pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, S));
}
__device__ __forceinline__ uint32_t pair_at(int s, uint32_t w, float scale) {
  return s == 0 ? pair<0>(w, scale) : s == 1 ? pair<1>(w, scale) : s == 2 ? pair<2>(w, scale)
                                                                     : pair<3>(w, scale);
}

// The exponent of a group's scale from its largest magnitude (as bits: NaN above infinity
// above every finite value): top = 1.m 2^k is at most 6 2^(k - 2) if 1.m <= 1.5, and
// 6 2^(k - 1) otherwise.
__device__ __forceinline__ int scale_exp(uint32_t top) {
  const int e = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x400000u ? 2 : 1);
  return min(max(e, -126), 125);
}

// The largest of a group's four lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));    // quad_perm 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));  // quad_perm 2 3 0 1
}

// The codes w and the scale byte s of eight channels of a token: the other 24 of the group
// are the next lanes' of four.
__device__ __forceinline__ void quantise(const float (&x)[8], uint32_t &w, uint32_t &s) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = quad_max(top);
  const int e = scale_exp(top);
  const bool bad = top >= 0x7f800000u;
  const float f = __uint_as_float((uint32_t)(127 - e) << 23);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * f;
  w = bad ? 0u : codes_of(y);
  s = bad ? 255 : e + 127;
}

// Eight channels of one token into its page's block c.
template <int D>
__device__ __forceinline__ void put(uint32_t w, uint32_t s, uint8_t *c, int tok, int which, int oct,
                                    int lpage) {
  const int codes = D / 2 << lpage, g = oct / 4;
  if (which == 0) {
    *reinterpret_cast<uint32_t *>(c + tok * (D / 2) + 4 * oct) = w;
    if (oct % 4 == 0) c[codes + tok * (D / 32) + g] = (uint8_t)s;
  } else {
    // four tokens side by side: column r holds D / 16 channels, D / 32 bytes a token
    uint8_t *d = c + tok / 4 * (2 * D) + tok % 4 * (D / 32);
    if constexpr (D == 128) {
      *reinterpret_cast<uint32_t *>(d + oct * 16) = w;
    } else if constexpr (D == 64) {
      *reinterpret_cast<uint16_t *>(d + 2 * oct * 8) = (uint16_t)w;
      *reinterpret_cast<uint16_t *>(d + (2 * oct + 1) * 8) = (uint16_t)(w >> 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) d[(4 * oct + i) * 4] = (uint8_t)(w >> (8 * i));
    }
    if (oct % 4 == 0) c[codes + tok / 4 * (D / 8) + 4 * g + tok % 4] = (uint8_t)s;
  }
}

// The codes of eight channels of a token in block c, and their group's scale byte.
template <int D>
__device__ __forceinline__ void held_of(const uint8_t *c, int tok, int which, int oct, int lpage,
                                         uint32_t &w, uint32_t &s) {
  const int codes = D / 2 << lpage, g = oct / 4;
  if (which == 0) {
    w = *reinterpret_cast<const uint32_t *>(c + tok * (D / 2) + 4 * oct);
    s = c[codes + tok * (D / 32) + g];
    return;
  }
  const uint8_t *d = c + tok / 4 * (2 * D) + tok % 4 * (D / 32);
  if constexpr (D == 128) {
    w = *reinterpret_cast<const uint32_t *>(d + oct * 16);
  } else if constexpr (D == 64) {
    w = *reinterpret_cast<const uint16_t *>(d + 2 * oct * 8) |
        (uint32_t)*reinterpret_cast<const uint16_t *>(d + (2 * oct + 1) * 8) << 16;
  } else {
    w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= (uint32_t)d[(4 * oct + i) * 4] << (8 * i);
  }
  s = c[codes + tok / 4 * (D / 8) + 4 * g + tok % 4];
}

}  // namespace kia
