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
    uint32_t w, sc;
    quantise(x[i], w, sc);
    if (c) put<D>(w, sc, c, tok, p.which, p.oct, a.lpage);
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
