// kia_cache.hip -- the paged key/value cache in 4 bits: tokens written to it and read
// back. (kia_cached.hip is the attention over it.)
//
// 32 neighbouring channels of a token share a scale 2^e, e the least power of two
// under which none of them passes 6, the largest of the 15 values that a code stands
// for (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives: E2M1). A value is held as the
// nearest of them, an even code between two: an error of at most 1/4 to 1 units of
// the scale. 4.25 bits a value. The values are exact in bf16, and gfx950 turns a
// pair of codes with its scale into a pair of bf16 in one instruction.
//
// Both kernels are bound by memory: a thread takes eight channels, so that four
// neighbouring lanes hold a group and find its largest value by two lane exchanges.
// Keys and values of 4 x 16 heads of 128 at T = 2048 in bf16, 85 MB: written in 22 us (3.9
// TB/s; the vector unit, busy half of the time, shares the bound), read back in 16 (5.2).
#include "kia_cache.hpp"

namespace kia {
namespace {

constexpr int CACHE_NT = 256;

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

// The place of a thread: eight channels of REP tokens, TOKENS apart, of one head's keys or
// values. What is the same for all of a workgroup is in scalar registers.
template <int D, int REP> struct Place {
  static constexpr int TOKENS = CACHE_NT * 8 / D;
  int which, b, h, t0, oct;
  __device__ __forceinline__ Place(const CacheArgs &a) {
    const int nb = (a.T + REP * TOKENS - 1) / (REP * TOKENS), s = blockIdx.x / nb;
    which = s % 2;
    h = s / 2 % a.Hkv;
    b = s / 2 / a.Hkv;
    t0 = (int)(blockIdx.x % nb) * REP * TOKENS + threadIdx.x / (D / 8);
    oct = threadIdx.x % (D / 8);
  }
  __device__ __forceinline__ int token(int i) const { return t0 + i * TOKENS; }
  // the head's block of the token's page, or nullptr; tok: the token in the page
  __device__ __forceinline__ uint8_t *held(const CacheArgs &a, int t, int &tok) const {
    if (t >= a.T || (a.counts && t >= a.counts[b])) return nullptr;
    const int64_t pos = (int64_t)a.starts[b] + t;
    if (pos < 0 || pos >= (int64_t)a.width << a.lpage) return nullptr;
    const int page = a.table[(int64_t)b * a.width + (pos >> a.lpage)];
    if (page < 0 || page >= a.pages) return nullptr;
    tok = (int)(pos & ((1 << a.lpage) - 1));
    return a.cache + cache_block<D>(page, which, h, a.Hkv, a.lpage);
  }
};

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

// Eight channels of one token into its page's block c.
template <int D>
__device__ __forceinline__ void hold(const float (&x)[8], uint8_t *c, int tok, int which, int oct,
                                     int lpage) {
  // (as bits: NaN above infinity above every finite value)
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  if (!c) return;
  // top = 1.m 2^k: at most 6 2^(k - 2) if 1.m <= 1.5, and 6 2^(k - 1) otherwise
  int e = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x400000u ? 2 : 1);
  e = min(max(e, -126), 125);
  const bool bad = top >= 0x7f800000u;
  const float f = __uint_as_float((uint32_t)(127 - e) << 23);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * f;
  const uint32_t w = bad ? 0u : codes_of(y);
  const uint8_t s = bad ? 255 : (uint8_t)(e + 127);
  const int codes = D / 2 << lpage, g = oct / 4;
  if (which == 0) {
    *reinterpret_cast<uint32_t *>(c + tok * (D / 2) + 4 * oct) = w;
    if (oct % 4 == 0) c[codes + tok * (D / 32) + g] = s;
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
    if (oct % 4 == 0) c[codes + tok / 4 * (D / 8) + 4 * g + tok % 4] = s;
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

template <typename TI, int D, int REP>
__global__ __launch_bounds__(CACHE_NT) void write_kernel(CacheArgs a) {
  const Place<D, REP> p(a);
  const View &v = p.which ? a.v : a.k;
  const TI *src = slice_of<TI>(v, p.b, p.h) + 8 * p.oct;
  // (rows are read whether they are held or not: their way does not wait for the table's)
  float x[REP][8] = {};
#pragma unroll
  for (int i = 0; i < REP; ++i)
    if (p.token(i) < a.T) load8(src + p.token(i) * v.st, x[i]);
#pragma unroll
  for (int i = 0; i < REP; ++i) {
    int tok = 0;
    uint8_t *c = p.held(a, p.token(i), tok);
    hold<D>(x[i], c, tok, p.which, p.oct, a.lpage);
  }
}

template <typename TI, int D, int REP>
__global__ __launch_bounds__(CACHE_NT) void read_kernel(CacheArgs a) {
  const Place<D, REP> p(a);
  const View &v = p.which ? a.v : a.k;
  TI *dst = slice_of<TI>(v, p.b, p.h) + 8 * p.oct;
  uint32_t w[REP] = {}, s[REP] = {};
#pragma unroll
  for (int i = 0; i < REP; ++i) {
    int tok = 0;
    if (const uint8_t *c = p.held(a, p.token(i), tok))
      held_of<D>(c, tok, p.which, p.oct, a.lpage, w[i], s[i]);
  }
#pragma unroll
  for (int i = 0; i < REP; ++i) {
    if (p.token(i) >= a.T) return;
    const float f = s[i] == 255 ? NAN : __uint_as_float(s[i] << 23);
    float x[8];
    values_of(w[i], f, x);
    store8(dst + p.token(i) * v.st, x);
  }
}

template <typename TI, int D, int REP> void launch_as(const CacheArgs &a, bool write, hipStream_t s) {
  constexpr int per = REP * Place<D, REP>::TOKENS;
  const dim3 grid(2u * a.B * a.Hkv * ((a.T + per - 1) / per)), block(CACHE_NT);
  if (write) hipLaunchKernelGGL((write_kernel<TI, D, REP>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((read_kernel<TI, D, REP>), grid, block, 0, s, a);
}

template <typename TI, int D> void launch_t(const CacheArgs &a, bool write, int cus, hipStream_t s) {
  if (cache_tokens(a.B, a.Hkv, a.T, D, cus) > Place<D, 1>::TOKENS) launch_as<TI, D, 4>(a, write, s);
  else launch_as<TI, D, 1>(a, write, s);
}
template <int D> void launch(const CacheArgs &a, bool write, int dtype, int cus, hipStream_t s) {
  if (dtype == KIA_F32) launch_t<float, D>(a, write, cus, s);
  else launch_t<uint16_t, D>(a, write, cus, s);
}
void launch_any(const CacheArgs &a, bool write, int d, int dtype, int cus, hipStream_t s) {
  if (d == 32) launch<32>(a, write, dtype, cus, s);
  else if (d == 64) launch<64>(a, write, dtype, cus, s);
  else launch<128>(a, write, dtype, cus, s);
}

}  // namespace

void launch_cache_write(const CacheArgs &a, int d, int dtype, int cus, hipStream_t s) {
  launch_any(a, true, d, dtype, cus, s);
}
void launch_cache_read(const CacheArgs &a, int d, int dtype, int cus, hipStream_t s) {
  launch_any(a, false, d, dtype, cus, s);
}

}  // namespace kia
