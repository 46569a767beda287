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

// The place of eight channels of one token: thread index -> (which, head, token,
// channels), and whether the table has a page for it.
template <int D> struct Place {
  int which, b, h, t, oct;
  bool in, held;
  int64_t base;  // of the head's block of the page
  int tok;
  __device__ __forceinline__ Place(const CacheArgs &a, int64_t i) {
    oct = (int)(i % (D / 8));
    i /= D / 8;
    t = (int)(i % a.T);
    i /= a.T;
    h = (int)(i % a.Hkv);
    i /= a.Hkv;
    b = (int)(i % a.B);
    which = (int)(i / a.B);
    in = which < 2;
    held = false;
    base = 0, tok = 0;
    if (!in || (a.counts && t >= a.counts[b])) return;
    const int64_t pos = (int64_t)a.starts[b] + t;
    if (pos < 0 || pos >= (int64_t)a.width << a.lpage) return;
    const int page = a.table[(int64_t)b * a.width + (pos >> a.lpage)];
    if (page < 0 || page >= a.pages) return;
    held = true;
    tok = (int)(pos & ((1 << a.lpage) - 1));
    base = cache_block<D>(page, which, h, a.Hkv, a.lpage);
  }
};

// The code of a value in units of its group's scale: bit 3 the sign, bits 0-2 the level.
__device__ __forceinline__ uint32_t code_of(float x) {
  const float a = fabsf(x);
  const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) +
                     (a >= 3.5f) + (a > 5.f);
  return c | (__float_as_uint(x) >> 31 << 3);
}
__device__ __forceinline__ float value_of(uint32_t code) {
  // 0, .5, 1, 1.5, 2, 3, 4, 6: levels 2 and up are 1.m 2^(e - 1)
  const uint32_t l = code & 7;
  const float v = l < 2 ? 0.5f * l : __uint_as_float((127u - 1u + (l >> 1)) << 23 | (l & 1) << 22);
  return code & 8 ? -v : v;
}

template <typename TI, int D> __global__ __launch_bounds__(CACHE_NT) void write_kernel(CacheArgs a) {
  const Place<D> p(a, (int64_t)blockIdx.x * CACHE_NT + threadIdx.x);
  float x[8] = {};
  if (p.held) {
    const View &v = p.which ? a.v : a.k;
    load8(slice_of<TI>(v, p.b, p.h) + p.t * v.st + 8 * p.oct, x);
  }
  // (as bits: NaN above infinity above every finite value)
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  if (!p.held) return;
  // top = 1.m 2^k: at most 6 2^(k - 2) if 1.m <= 1.5, and 6 2^(k - 1) otherwise
  int e = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x400000u ? 2 : 1);
  e = min(max(e, -126), 125);
  const bool bad = top >= 0x7f800000u;
  // (2^-e in two factors: 2^126 is the largest, and tiny values are not lost)
  const float f = __uint_as_float((uint32_t)(127 - e) << 23);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) w |= bad ? 0u : code_of(x[i] * f) << (4 * i);
  const uint8_t s = bad ? 255 : (uint8_t)(e + 127);
  uint8_t *c = a.cache + p.base;
  const int codes = D / 2 << a.lpage, g = p.oct / 4;
  if (p.which == 0) {
    *reinterpret_cast<uint32_t *>(c + p.tok * (D / 2) + 4 * p.oct) = w;
    if (p.oct % 4 == 0) c[codes + p.tok * (D / 32) + g] = s;
  } else {
    // four tokens side by side: column r holds D / 16 channels, D / 32 bytes a token
    uint8_t *d = c + p.tok / 4 * (2 * D) + p.tok % 4 * (D / 32);
    if constexpr (D == 128) {
      *reinterpret_cast<uint32_t *>(d + p.oct * 16) = w;
    } else if constexpr (D == 64) {
      *reinterpret_cast<uint16_t *>(d + 2 * p.oct * 8) = (uint16_t)w;
      *reinterpret_cast<uint16_t *>(d + (2 * p.oct + 1) * 8) = (uint16_t)(w >> 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) d[(4 * p.oct + i) * 4] = (uint8_t)(w >> (8 * i));
    }
    if (p.oct % 4 == 0) c[codes + p.tok / 4 * (D / 8) + 4 * g + p.tok % 4] = s;
  }
}

template <typename TI, int D> __global__ __launch_bounds__(CACHE_NT) void read_kernel(CacheArgs a) {
  const Place<D> p(a, (int64_t)blockIdx.x * CACHE_NT + threadIdx.x);
  if (!p.in) return;
  float x[8] = {};
  if (p.held) {
    const uint8_t *c = a.cache + p.base;
    const int codes = D / 2 << a.lpage, g = p.oct / 4;
    uint32_t w = 0;
    uint8_t s;
    if (p.which == 0) {
      w = *reinterpret_cast<const uint32_t *>(c + p.tok * (D / 2) + 4 * p.oct);
      s = c[codes + p.tok * (D / 32) + g];
    } else {
      const uint8_t *d = c + p.tok / 4 * (2 * D) + p.tok % 4 * (D / 32);
      if constexpr (D == 128) {
        w = *reinterpret_cast<const uint32_t *>(d + p.oct * 16);
      } else if constexpr (D == 64) {
        w = *reinterpret_cast<const uint16_t *>(d + 2 * p.oct * 8) |
            (uint32_t)*reinterpret_cast<const uint16_t *>(d + (2 * p.oct + 1) * 8) << 16;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= (uint32_t)d[(4 * p.oct + i) * 4] << (8 * i);
      }
      s = c[codes + p.tok / 4 * (D / 8) + 4 * g + p.tok % 4];
    }
    const float f = s == 255 ? NAN : __uint_as_float((uint32_t)s << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = value_of(w >> (4 * i)) * f;
  }
  const View &v = p.which ? a.v : a.k;
  store8(slice_of<TI>(v, p.b, p.h) + p.t * v.st + 8 * p.oct, x);
}

template <int D> void launch(const CacheArgs &a, bool write, int dtype, hipStream_t s) {
  const int64_t n = (int64_t)2 * a.B * a.Hkv * a.T * (D / 8);
  const dim3 grid((unsigned)((n + CACHE_NT - 1) / CACHE_NT)), block(CACHE_NT);
  if (write) {
    if (dtype == KIA_F32) hipLaunchKernelGGL((write_kernel<float, D>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((write_kernel<uint16_t, D>), grid, block, 0, s, a);
  } else {
    if (dtype == KIA_F32) hipLaunchKernelGGL((read_kernel<float, D>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_kernel<uint16_t, D>), grid, block, 0, s, a);
  }
}
void launch_any(const CacheArgs &a, bool write, int d, int dtype, hipStream_t s) {
  if (d == 32) launch<32>(a, write, dtype, s);
  else if (d == 64) launch<64>(a, write, dtype, s);
  else launch<128>(a, write, dtype, s);
}

}  // namespace

void launch_cache_write(const CacheArgs &a, int d, int dtype, hipStream_t s) {
  launch_any(a, true, d, dtype, s);
}
void launch_cache_read(const CacheArgs &a, int d, int dtype, hipStream_t s) {
  launch_any(a, false, d, dtype, s);
}

}  // namespace kia
