// kia_append.hip -- new tokens into the 4-bit cache: queries and keys rotated by their
// positions on the way, keys and values held, and the bounds of each page's keys (their
// least and largest value in every channel), which page selection reads.
//
// Bound by memory: q, k and v are read once, q is written, k and v leave 17/32 byte a value.
// A workgroup takes 64 positions of a sequence (a page, if pages are larger) and a share of
// its heads; sine and cosine of its tokens go to LDS once for all of them. Spans start at
// multiples of their size, so that the tokens of a page are one workgroup's, and the bounds
// need no atomics and no second pass: the held values of the page's tokens go to LDS, the
// earlier ones read back from the page.
//
// A rotated key is rounded once, to its 4 bits. The rotation in 32 bits is off by up to
// 2^-21 of the pair's magnitudes, which decides another code for about one value in 10^7: where
// any of a group's codes or its scale could differ within 2^-20, the group is taken again in
// 64 bits.
#include "kia_cache.hpp"

namespace kia {
namespace {

constexpr int SUB = 64;  // positions of one table of angles
// Threads of a workgroup: eight channels of a token each.
template <int D> struct Threads { static constexpr int N = SUB * D / 8 < 512 ? SUB * D / 8 : 512; };
enum { HALF8, HALF, NEIGHBOURS };  // which channels make a pair; HALF8: in chunks of eight

// The series of sin x / x and cos x in x^2, from the last terms (-1/18! and 1/17!) on. (From
// memory: as literals they would take the kernel's registers for a path that is rare.)
__constant__ double SERIES[9][2] = {{1.0 / 355687428096000.0, -1.0 / 6402373705728000.0},
                                    {-1.0 / 1307674368000.0, 1.0 / 20922789888000.0},
                                    {1.0 / 6227020800.0, -1.0 / 87178291200.0},
                                    {-1.0 / 39916800.0, 1.0 / 479001600.0},
                                    {1.0 / 362880.0, -1.0 / 3628800.0},
                                    {-1.0 / 5040.0, 1.0 / 40320.0},
                                    {1.0 / 120.0, -1.0 / 720.0},
                                    {-1.0 / 6.0, 1.0 / 24.0},
                                    {1.0, -0.5}};

// sin and cos of x in 64 bits: quarter turns off (exact to 2^-53 for |x| < 2^31 pi / 2), then
// their series on +- pi / 4 (the first terms left out are below 10^-19).
__device__ __forceinline__ void turn64(double x, double &s, double &c) {
  const double q = rint(x * 0.63661977236758134308);
  double r = fma(-q, 1.57079632679489655800, x);
  r = fma(-q, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double u = 0.0, w = 0.0;
#pragma unroll 1
  for (int i = 0; i < 9; ++i) {
    u = fma(u, z, SERIES[i][0]);
    w = fma(w, z, SERIES[i][1]);
  }
  u *= r;
  w = fma(w, z, 1.0);
  const int k = (int)(q - 4.0 * floor(q * 0.25));
  s = k & 1 ? w : u;
  c = k & 1 ? -u : w;
  if (k & 2) s = -s, c = -c;
}

// Codes and scale byte of eight channels y of a token from 64 bits (the group's other
// channels are the next lanes').
__device__ __forceinline__ void quantise64(const double (&y)[8], uint32_t &w, uint32_t &s) {
  double top = 0;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bad |= !(fabs(y[e]) < INFINITY);
    top = fmax(top, fabs(y[e]));
  }
#pragma unroll
  for (int i = 1; i < 4; i *= 2) {
    top = fmax(top, __shfl_xor(top, i));
    bad |= (bool)__shfl_xor((int)bad, i);
  }
  // top = 1.m 2^k, as scale_exp
  const uint64_t bits = (uint64_t)__double_as_longlong(top);
  int e = (int)(bits >> 52) - 1023 - ((bits & 0xfffffffffffffull) <= 0x8000000000000ull ? 2 : 1);
  e = min(max(e, -126), 125);
  const double f = __longlong_as_double((long long)(1023 - e) << 52);
  w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double a = fabs(y[i]) * f;
    const uint32_t level = (a > 0.25) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) +
                           (a >= 3.5) + (a > 5.0);
    w |= (level | (signbit(y[i]) ? 8u : 0u)) << (4 * i);
  }
  w = bad ? 0u : w;
  s = bad ? 255u : (uint32_t)(e + 127);
}

// The eight channels of a token that a thread has, and their partners in the rotation.
template <int MODE> struct Chunk {
  float x[8], y[8];  // y: the partners
};

// Channel c = 8 oct + e of a rotated part of 2 n: its pair, its partner's channel, and
// whether it is the first of the two.
template <int MODE> struct Pair {
  bool turns, first;
  int pair, partner;
  __device__ __forceinline__ Pair(int c, int n) {
    turns = c < 2 * n;
    if constexpr (MODE == NEIGHBOURS) {
      first = c % 2 == 0;
      pair = c / 2;
      partner = c ^ 1;
    } else {
      first = c < n;
      pair = first ? c : c - n;
      partner = first ? c + n : c - n;
    }
  }
};

template <typename TI, int MODE>
__device__ __forceinline__ void load_pairs(const TI *row, int oct, int n, Chunk<MODE> &k) {
  load8(row + 8 * oct, k.x);
  if constexpr (MODE == NEIGHBOURS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) k.y[e] = k.x[e ^ 1];
  } else if constexpr (MODE == HALF8) {
    const Pair<MODE> p(8 * oct, n);
    load8(row + (p.turns ? p.partner : 8 * oct), k.y);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const Pair<MODE> p(8 * oct + e, n);
      k.y[e] = load1(row + (p.turns ? p.partner : 8 * oct + e));
    }
  }
}

// The rotated chunk; tol: what its values may be off by, at most.
template <int MODE, bool TOL>
__device__ __forceinline__ void turned(const Chunk<MODE> &k, const float2 *turn, int oct, int n,
                                       float factor, float (&z)[8], float (&tol)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const Pair<MODE> p(8 * oct + e, n);
    const float2 w = p.turns ? turn[p.pair] : make_float2(1.f, 0.f);
    const float r = p.first ? fmaf(k.x[e], w.x, -(k.y[e] * w.y)) : fmaf(k.x[e], w.x, k.y[e] * w.y);
    z[e] = p.turns ? r : k.x[e];
    if constexpr (TOL) tol[e] = p.turns ? (fabsf(k.x[e]) + fabsf(k.y[e])) * factor : 0.f;
  }
}

// Codes and scale of a rotated key's chunk from 32 bits; whether the exact rotation's
// could be others.
template <int MODE>
__device__ __forceinline__ bool quantise_turned(const Chunk<MODE> &k, const float2 *turn, int oct, int n,
                                                float factor, uint32_t &w, uint32_t &s) {
  float z[8], tol[8], hi = 0.f, lo = 0.f;
  turned<MODE, true>(k, turn, oct, n, fabsf(factor) * 0x1p-20f, z, tol);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // (NaN: as large as it gets)
    const float up = fabsf(z[e]) + tol[e];
    hi = up > hi || up != up ? up : hi;
    lo = fmaxf(lo, fabsf(z[e]) - tol[e]);
  }
  uint32_t h = __float_as_uint(hi) & 0x7fffffffu;
#pragma unroll
  for (int i = 1; i < 4; i *= 2) {
    h = max(h, (uint32_t)__shfl_xor((int)h, i));
    lo = fmaxf(lo, __shfl_xor(lo, i));
  }
  const int e = scale_exp(h);
  const float f = __uint_as_float((uint32_t)(127 - e) << 23);
  float up[8], down[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    up[i] = (z[i] + tol[i]) * f;
    down[i] = (z[i] - tol[i]) * f;
  }
  w = codes_of(up);
  s = (uint32_t)(e + 127);
  return h >= 0x7f800000u || e != scale_exp(__float_as_uint(lo)) || w != codes_of(down);
}
// The exact rotation's.
template <int MODE>
__device__ __forceinline__ void quantise_turned64(const Chunk<MODE> &k, double pos, int oct, int n,
                                                  const AppendArgs &a, uint32_t &w, uint32_t &s) {
  double y[8] = {};
  const double factor = (double)a.factor;
  // (channel by channel: rare, and unrolled it would take twice the kernel's registers)
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    float x = k.x[0], o = k.y[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) x = i == j ? k.x[j] : x, o = i == j ? k.y[j] : o;
    const Pair<MODE> p(8 * oct + i, n);
    double sn, cs;
    turn64(pos * a.freq[p.turns ? p.pair : 0], sn, cs);
    const double b = (double)o * (sn * factor);
    const double r = fma((double)x, cs * factor, p.first ? -b : b);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = i == j ? (p.turns ? r : (double)x) : y[j];
  }
  quantise64(y, w, s);
}

__device__ __forceinline__ float least(float a, float b) { return b < a || b != b ? b : a; }
__device__ __forceinline__ float most(float a, float b) { return b > a || b != b ? b : a; }

// The bounds of the pages of 64 positions from their tokens' values in LDS, of tokens
// from .. to - 1; page_at(t): where those of token t's page go, or nullptr. `go_on`: the
// page's earlier positions are in its bounds already. All threads call it after a barrier; the
// next write to l.val needs none, the next call does.
template <int D> struct BoundsLds {
  uint32_t val[SUB][D / 2];
  float4 part[Threads<D>::N];
};
template <int D, class F>
__device__ __forceinline__ void bounds_of(BoundsLds<D> &l, int lpage, int from, int to, bool go_on, F page_at) {
  constexpr int C = D / 2, GROUPS = Threads<D>::N / C;
  const int tid = threadIdx.x, c = tid % C, g = tid / C;
  const int ltok = min(lpage, 6), pages = SUB >> ltok, parts = GROUPS / pages;  // (GROUPS >= 8, pages 1, 2 or 4)
  // thread: two channels of a page, and a part of its tokens
  const int p = g % pages, part = g / pages, size = (1 << ltok) / parts;
  const int t0 = max(from, (p << ltok) + part * size), t1 = min(to, (p << ltok) + (part + 1) * size);
  float4 r = make_float4(INFINITY, INFINITY, -INFINITY, -INFINITY);
  for (int t = t0; t < t1; ++t) {
    const uint32_t v = l.val[t][c];
    const float x = __uint_as_float(v << 16), y = __uint_as_float(v & 0xffff0000u);
    r = make_float4(least(r.x, x), least(r.y, y), most(r.z, x), most(r.w, y));
  }
  l.part[tid] = r;
  __syncthreads();
  if (part) return;
  for (int i = 1; i < parts; ++i) {
    const float4 o = l.part[tid + i * pages * C];
    r = make_float4(least(r.x, o.x), least(r.y, o.y), most(r.z, o.z), most(r.w, o.w));
  }
  uint32_t *b = max(from, p << ltok) < min(to, (p + 1) << ltok) ? page_at(p << ltok) : nullptr;
  if (!b) return;
  if (go_on) {
    const uint32_t x = b[c], y = b[C + c];
    r = make_float4(least(r.x, __uint_as_float(x << 16)), least(r.y, __uint_as_float(x & 0xffff0000u)),
                    most(r.z, __uint_as_float(y << 16)), most(r.w, __uint_as_float(y & 0xffff0000u)));
  }
  b[c] = cvt_bf16x2(r.x, r.y);
  b[C + c] = cvt_bf16x2(r.z, r.w);
}

template <int D> __device__ __forceinline__ void keep(BoundsLds<D> &l, int t, int oct, uint32_t w, uint32_t s) {
  float x[8];
  values_of(w, s == 255 ? NAN : __uint_as_float(s << 23), x);
#pragma unroll
  for (int e = 0; e < 4; ++e) l.val[t][4 * oct + e] = cvt_bf16x2(x[2 * e], x[2 * e + 1]);
}

// The page of position `pos` of sequence b, or -1.
__device__ __forceinline__ int page_of(const CacheArgs &c, int b, int64_t pos) {
  if (pos < 0 || pos >= (int64_t)c.width << c.lpage) return -1;
  const int page = c.table[(int64_t)b * c.width + (pos >> c.lpage)];
  return page < 0 || page >= c.pages ? -1 : page;
}

template <typename TI, int D, int MODE>
__global__ __launch_bounds__(Threads<D>::N) void append_kernel(AppendArgs a) {
  constexpr int NT = Threads<D>::N, OCTS = D / 8, TOKENS = NT / OCTS;
  __shared__ __attribute__((aligned(16))) BoundsLds<D> lds;
  extern __shared__ float2 turn[];  // [64][n]
  const CacheArgs &c = a.c;
  const int tid = threadIdx.x, oct = tid % OCTS, n = a.rot / 2;
  const int b = blockIdx.x / a.spans, lspan = max(c.lpage, 6);
  const int64_t start = c.starts[b], end = start + c.T;
  const int64_t p0 = ((start >> lspan) + (int)(blockIdx.x % a.spans)) << lspan;
  if (p0 >= end) return;
  const int64_t held = start + (c.counts ? min(max(c.counts[b], 0), c.T) : c.T);  // end of what is held
  const int heads = c.Hkv, streams = 2 * c.Hkv + a.H;
  for (int sub = 0; sub < 1 << (lspan - 6); ++sub) {
    const int64_t base = p0 + sub * SUB;
    if (base >= end) break;
    const int lo = (int)max((int64_t)0, start - base), hi = (int)min((int64_t)SUB, end - base);  // (lo > hi: none)
    if (lo >= hi && !a.bounds) continue;
    // angles of the new tokens
    __syncthreads();
    for (int e = tid; e < (hi - lo) * n; e += NT) {
      float s, w;
      turn_of((double)(base + lo + e / n), a.freq[e % n], s, w);
      turn[lo * n + e] = make_float2(w * a.factor, s * a.factor);
    }
    __syncthreads();
    // tokens whose keys are on a page that gets tokens: in bounds from `old` on
    const int64_t page0 = max(start >> c.lpage << c.lpage, (int64_t)0);
    const int old = (int)min((int64_t)SUB, max((int64_t)0, page0 - base));
    const int to = (int)max((int64_t)0, min((int64_t)SUB, held - base));
    for (int st = blockIdx.y; st < streams; st += gridDim.y) {
      const int kind = st < heads ? 0 : st < 2 * heads ? 1 : 2;  // keys, values, queries
      const int h = kind == 0 ? st : kind == 1 ? st - heads : st - 2 * heads;
      const View &v = kind == 0 ? c.k : kind == 1 ? c.v : a.q;
      const TI *src = slice_of<TI>(v, b, h);
      const bool bounds = kind == 0 && a.bounds && held > start;
#pragma unroll 1
      for (int t = tid / OCTS; t < SUB; t += TOKENS) {
        const bool in = t >= lo && t < hi;
        const TI *row = src + (base + t - start) * v.st;
        Chunk<MODE> x = {};
        if (in) {
          if (kind == 1) load8(row + 8 * oct, x.x);
          else load_pairs<TI, MODE>(row, oct, n, x);
        }
        if (kind == 2) {
          if (!in) continue;
          float z[8], tol[8];
          turned<MODE, false>(x, turn + t * n, oct, n, 0.f, z, tol);
          store8(slice_of<TI>(a.qo, b, h) + (base + t - start) * a.qo.st + 8 * oct, z);
          continue;
        }
        const bool live = in && base + t < held, before = bounds && t >= old && base + t < start;
        const int page = live || before ? page_of(c, b, base + t) : -1;
        uint32_t w, s;
        if (kind == 0) {
          const bool open = quantise_turned<MODE>(x, turn + (live ? t : 0) * n, oct, n, a.factor, w, s);
          // a group goes again if one of its four lanes asks for it
          const uint64_t again = __ballot(open && live && page >= 0) >> (tid & 60) & 15;
          if (__builtin_expect(__any(again != 0), 0)) {
            if (again) quantise_turned64<MODE>(x, (double)(base + t), oct, n, a, w, s);
          }
        } else {
          quantise(x.x, w, s);
        }
        if (page < 0) continue;
        const int tok = (int)((base + t) & ((1 << c.lpage) - 1));
        uint8_t *at = c.cache + cache_block<D>(page, kind, h, c.Hkv, c.lpage);
        if (live) put<D>(w, s, at, tok, kind, oct, c.lpage);
        else held_of<D>(at, tok, kind, oct, c.lpage, w, s);
        if (bounds) keep<D>(lds, t, oct, w, s);
      }
      if (!bounds) continue;
      __syncthreads();
      bounds_of<D>(lds, c.lpage, old, to, sub > 0, [&](int t) -> uint32_t * {
        const int page = page_of(c, b, base + t);
        return page < 0 ? nullptr : a.bounds + ((int64_t)page * c.Hkv + h) * D;
      });
    }
  }
}

// The bounds of the pages that hold positions starts[b] .. ends[b] - 1 (c.counts: the
// ends), over their tokens before ends[b]: a workgroup a page and head.
template <int D> __global__ __launch_bounds__(Threads<D>::N) void bounds_kernel(AppendArgs a) {
  constexpr int OCTS = D / 8, TOKENS = Threads<D>::N / OCTS;
  __shared__ __attribute__((aligned(16))) BoundsLds<D> lds;
  const CacheArgs &c = a.c;
  const int tid = threadIdx.x, oct = tid % OCTS;
  const int h = blockIdx.x % c.Hkv, lspan = max(c.lpage, 6);
  const int b = blockIdx.x / c.Hkv / a.spans;
  const int64_t p0 = (int64_t)(blockIdx.x / c.Hkv % a.spans) << lspan;
  const int64_t start = max(c.starts[b], 0), end = min((int64_t)c.counts[b], (int64_t)c.width << c.lpage);
  const int64_t page0 = start >> c.lpage << c.lpage;  // the first page's first position
  if (start >= end || p0 >= end || p0 + (1 << lspan) <= page0) return;
  for (int sub = 0; sub < 1 << (lspan - 6); ++sub) {
    const int64_t base = p0 + sub * SUB;
    if (base >= end) break;
    const int from = (int)min((int64_t)SUB, max((int64_t)0, page0 - base)), to = (int)min((int64_t)SUB, end - base);
    for (int t = tid / OCTS; t < to; t += TOKENS) {
      const int page = t >= from ? page_of(c, b, base + t) : -1;
      if (page < 0) continue;
      uint32_t w, s;
      held_of<D>(c.cache + cache_block<D>(page, 0, h, c.Hkv, c.lpage), (int)((base + t) & ((1 << c.lpage) - 1)),
                 0, oct, c.lpage, w, s);
      keep<D>(lds, t, oct, w, s);
    }
    __syncthreads();
    bounds_of<D>(lds, c.lpage, from, to, sub > 0, [&](int t) -> uint32_t * {
      const int page = page_of(c, b, base + t);
      return page < 0 ? nullptr : a.bounds + ((int64_t)page * c.Hkv + h) * D;
    });
  }
}

template <typename TI, int D> void append_as(const AppendArgs &a, dim3 grid, hipStream_t s) {
  const size_t lds = (size_t)SUB * (a.rot / 2) * sizeof(float2);
  if (a.layout == KIA_ROTARY_NEIGHBOURS)
    hipLaunchKernelGGL((append_kernel<TI, D, NEIGHBOURS>), grid, dim3(Threads<D>::N), lds, s, a);
  else if (a.rot / 2 % 8 == 0)
    hipLaunchKernelGGL((append_kernel<TI, D, HALF8>), grid, dim3(Threads<D>::N), lds, s, a);
  else
    hipLaunchKernelGGL((append_kernel<TI, D, HALF>), grid, dim3(Threads<D>::N), lds, s, a);
}
template <int D> void append_d(const AppendArgs &a, dim3 grid, int dtype, hipStream_t s) {
  if (dtype == KIA_F32) append_as<float, D>(a, grid, s);
  else append_as<uint16_t, D>(a, grid, s);
}

}  // namespace

void launch_append(const AppendArgs &a, int d, int dtype, int cus, hipStream_t s) {
  const unsigned spans = (unsigned)a.c.B * a.spans, streams = 2u * a.c.Hkv + a.H;
  const unsigned shares = std::min(streams, std::max(1u, (4u * cus + spans - 1) / spans));
  const dim3 grid(spans, shares);
  if (d == 32) append_d<32>(a, grid, dtype, s);
  else if (d == 64) append_d<64>(a, grid, dtype, s);
  else append_d<128>(a, grid, dtype, s);
}

void launch_bounds(const AppendArgs &a, int d, hipStream_t s) {
  const dim3 grid((unsigned)a.c.B * a.spans * a.c.Hkv);
  if (d == 32) hipLaunchKernelGGL((bounds_kernel<32>), grid, dim3(Threads<32>::N), 0, s, a);
  else if (d == 64) hipLaunchKernelGGL((bounds_kernel<64>), grid, dim3(Threads<64>::N), 0, s, a);
  else hipLaunchKernelGGL((bounds_kernel<128>), grid, dim3(Threads<128>::N), 0, s, a);
}

}  // namespace kia
