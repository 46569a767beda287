// kia_append.hip -- new tokens into the 4-bit cache: queries and keys rotated by their
// positions on the way, keys and values held, and the bounds of each page's keys (their
// least and largest value in every channel), which page selection reads.
//
// Bound by memory: q, k and v are read once, q is written, k and v leave 17/32 byte a value.
// A workgroup takes 64 positions of a sequence (a page, if pages are larger) and a share of
// its heads; sine and cosine of its tokens go to LDS once for all of them. Spans start at
// multiples of their size, so that the tokens of a page are one workgroup's, and the bounds
// need no atomics and no second pass: the held values of the page's tokens go to LDS, the
// earlier ones read back from the page. 4 prompts of 2048 tokens, 16
// heads of 128 for queries and keys, bf16, with bounds: 47 us for 153 MB, 3.3 TB/s of the 5.1
// that a copy reaches; rotating, finding codes and bounds keeps the vector units active for 56% of the
// cycles. Neither is full: 128 registers leave two workgroups of eight waves a CU. A token each of 32
// sequences, 16 heads of 128 over 4: 10 us, loads of the length, page, keys and earlier tokens one
// after another, by 16 of a workgroup's 512 lanes.
//
// A rotated key is rounded once, to its 4 bits. The rotation in 32 bits is off by up to 7.4 roundings
// (2^-24) of the pair's magnitudes: 4 of sine and cosine, 0.4 of the angle's rest in 32 bits, one each
// of the factor, the product and the fma. That decides another code for about one value in
// 10^7: where any of a group's codes or its scale could differ within 10 roundings, the group
// is taken again in 64 bits.
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

// sin and cos of the same angle in 32 bits for that check: the rest behind the quarter turns is that
// of the angle itself however far it is (2 / pi in two parts; rounded to 53 bits, their product is
// off by more than the check allows for from 2^30 radians on, as rotated queries are there).
__device__ __forceinline__ void turn_key(double x, float &s, float &c) {
  constexpr double HI = 0.63661977236758134308, LO = -3.9357353350364972e-17;
  const double q = rint(x * HI);
  sincospif(0.5f * (float)fma(x, LO, fma(x, HI, -q)), &s, &c);
  const int k = (int)(q - 4.0 * floor(q * 0.25));
  if (k & 1) { const float y = s; s = c; c = -y; }
  if (k & 2) { s = -s; c = -c; }
}

// The code and scale byte of a channel y from 64 bits: the other 31 of its group are the next
// lanes' of 32.
__device__ __forceinline__ void quantise64(double y, uint32_t &w, uint32_t &s) {
  double top = fabs(y);
  bool bad = !(top < INFINITY);
#pragma unroll
  for (int i = 1; i < 32; i *= 2) {
    top = fmax(top, __shfl_xor(top, i));
    bad |= (bool)__shfl_xor((int)bad, i);
  }
  // top = 1.m 2^k, as scale_exp
  const uint64_t bits = (uint64_t)__double_as_longlong(top);
  int e = (int)(bits >> 52) - 1023 - ((bits & 0xfffffffffffffull) <= 0x8000000000000ull ? 2 : 1);
  e = min(max(e, -126), 125);
  const double a = fabs(y) * __longlong_as_double((long long)(1023 - e) << 52);
  w = (a > 0.25) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0);
  w = bad ? 0u : w | (signbit(y) ? 8u : 0u);
  s = bad ? 255u : (uint32_t)(e + 127);
}

// The eight channels of a token that a thread has, and their partners in the rotation.
struct Chunk {
  float x[8], y[8];
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

// Eight channels as they are loaded.
template <typename TI> struct Raw;
template <> struct Raw<uint16_t> {
  u32x4 w = {};
  __device__ __forceinline__ void load(const uint16_t *p) { w = *reinterpret_cast<const u32x4 *>(p); }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  // the lane's at `from`
  __device__ __forceinline__ Raw of(int from) const {
    Raw r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.w[e] = (uint32_t)__shfl((int)w[e], from);
    return r;
  }
};
template <> struct Raw<float> {
  f32x4 w[2] = {};
  __device__ __forceinline__ void load(const float *p) { w[0] = load4(p), w[1] = load4(p + 4); }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = w[e / 4][e % 4];
  }
  __device__ __forceinline__ Raw of(int from) const {
    Raw r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.w[e / 4][e % 4] = __shfl(w[e / 4][e % 4], from);
    return r;
  }
};

// The partners' values: neighbours are the thread's own, a chunk of eight another lane's of
// the token, all else (row: the token, or nullptr) is read again.
template <typename TI, int MODE>
__device__ __forceinline__ void pairs_of(const Raw<TI> &own, const TI *row, int oct, int n, Chunk &k) {
  own.values(k.x);
  if constexpr (MODE == NEIGHBOURS) {
#pragma unroll
    for (int e = 0; e < 8; ++e) k.y[e] = k.x[e ^ 1];
  } else if constexpr (MODE == HALF8) {
    const Pair<MODE> p(8 * oct, n);
    own.of((threadIdx.x & 63) + (p.turns ? (p.partner - 8 * oct) / 8 : 0)).values(k.y);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const Pair<MODE> p(8 * oct + e, n);
      k.y[e] = p.turns && row ? load1(row + p.partner) : 0.f;
    }
  }
}

// Where a token's table holds a pair's cosine and sine: those of a chunk in pairs of pairs,
// the chunks' first ones side by side, so that neighbouring lanes read neighbouring 16 bytes
// (in order, they met in a quarter of the banks: 67 us for the prompts above).
template <int MODE> struct Table {
  static constexpr int OF = MODE == HALF8 ? 8 : 4;  // pairs of a chunk
  int chunks;
  __host__ __device__ __forceinline__ explicit Table(int n) : chunks((n + OF - 1) / OF) {}
  __host__ __device__ __forceinline__ int size() const { return chunks * OF; }
  __device__ __forceinline__ int at(int pair) const { return pair % OF / 2 * 2 * chunks + pair / OF * 2 + pair % 2; }
};

// The rotated chunk, and the largest magnitude of its pairs: |x| + |y|.
template <int MODE>
__device__ __forceinline__ float turned(const Chunk &k, const float2 *turn, int oct, int n, float (&z)[8]) {
  const Pair<MODE> chunk(8 * oct, n);
  const Table<MODE> table(n);
  const float2 *at = turn + 2 * (MODE == HALF8 ? chunk.pair / 8 : oct);
  float size = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    Pair<MODE> p = MODE == HALF8 ? chunk : Pair<MODE>(8 * oct + e, n);
    if (MODE == NEIGHBOURS) p.first = e % 2 == 0;
    const int j = MODE == HALF8 ? e : e / 2;  // of the chunk's pairs
    const float2 w = !p.turns ? make_float2(1.f, 0.f)
                     : MODE == HALF ? turn[table.at(p.pair)] : at[j / 2 * 2 * table.chunks + j % 2];
    const float r = fmaf(k.x[e], w.x, p.first ? -(k.y[e] * w.y) : k.y[e] * w.y);
    z[e] = p.turns ? r : k.x[e];
    size = fmaxf(size, p.turns ? fabsf(k.x[e]) + fabsf(k.y[e]) : 0.f);
  }
  return size;
}

// Codes of eight values over 2^e (the conversion divides by a scale by itself).
__device__ __forceinline__ uint32_t codes_over(const float (&x)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// Codes and scale of a rotated key's chunk from 32 bits; whether the exact rotation's
// could be others.
template <int MODE>
__device__ __forceinline__ bool quantise_turned(const Chunk &k, const float2 *turn, int oct, int n, float factor,
                                                uint32_t &w, uint32_t &s) {
  float z[8];
  // what a turned channel may be off by: 10 roundings
  const float off = turned<MODE>(k, turn, oct, n, z) * fabsf(factor) * 0x1.4p-21f;
  uint32_t top = 0;  // (as bits: NaN above infinity above every finite value)
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(z[e]) & 0x7fffffffu);
  const float far = __uint_as_float(quad_max(__float_as_uint(off)));
  const float t = __uint_as_float(quad_max(top));
  const int e = scale_exp(__float_as_uint(t + far));
  s = (uint32_t)(e + 127);
  float up[8], down[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float o = MODE == HALF8 || Pair<MODE>(8 * oct + i, n).turns ? off : 0.f;
    up[i] = z[i] + o;
    down[i] = z[i] - o;
  }
  const float scale = __uint_as_float(s << 23);
  w = codes_over(up, scale);
  // (far NaN, or top: not below infinity)
  return !(t + far < INFINITY) || e != scale_exp(__float_as_uint(fmaxf(t - far, 0.f))) || w != codes_over(down, scale);
}
// The exact rotation's, of the row's channel c; the codes of eight channels in the first of
// their lanes.
template <typename TI, int MODE>
__device__ __forceinline__ void quantise_turned64(const TI *row, double pos, int c, int n, const AppendArgs &a,
                                                  uint32_t &w, uint32_t &s) {
  const Pair<MODE> p(c, n);
  const double x = (double)load1(row + c), o = (double)load1(row + (p.turns ? p.partner : c));
  double sn, cs;
  turn64(pos * a.freq[p.turns ? p.pair : 0], sn, cs);
  const double b = o * (sn * (double)a.factor), r = fma(x, cs * (double)a.factor, p.first ? -b : b);
  quantise64(p.turns ? r : x, w, s);
#pragma unroll
  for (int i = 1; i < 8; i *= 2) w |= (uint32_t)__shfl_down((int)w, i) << (4 * i);
}

// Two bf16 as integers of their order, and back; NaN is the largest.
typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t ordered(uint32_t x) { return x ^ ((x >> 15 & 0x00010001u) * 0x7fffu); }
__device__ __forceinline__ i16x2 pack2(uint32_t x) { return __builtin_bit_cast(i16x2, x); }
struct Ends {
  i16x2 lo = {0x7fff, 0x7fff}, hi = {-0x8000, -0x8000};
  __device__ __forceinline__ void take(uint32_t l, uint32_t h) {
    lo = __builtin_elementwise_min(lo, pack2(l));
    hi = __builtin_elementwise_max(hi, pack2(h));
  }
};

// The bounds of the pages of 64 positions from their tokens' values in LDS, of tokens
// from .. to - 1; page_at(t): where those of token t's page go, or nullptr. `go_on`: the
// page's earlier positions are in its bounds already. All threads call it after a barrier; the
// next write to l.val needs none, the next call does.
template <int D> struct BoundsLds {
  uint32_t val[SUB][D / 2];
  uint2 part[Threads<D>::N];
};
// Of a key stream: the groups of four lanes (token and group of a span) to take in 64 bits, as
// a list and how many. Stream i of a workgroup counts in i % 3, so that a barrier a stream
// is enough: the next but one's is cleared behind it.
template <int D> struct Again {
  uint16_t list[SUB * D / 32];
  int count[3];
};
template <int D, class F>
__device__ __forceinline__ void bounds_of(BoundsLds<D> &l, int lpage, int from, int to, bool go_on, F page_at) {
  constexpr int C = D / 2, GROUPS = Threads<D>::N / C;
  const int tid = threadIdx.x, c = tid % C, g = tid / C;
  const int ltok = min(lpage, 6), pages = SUB >> ltok, parts = GROUPS / pages;  // (GROUPS >= 8, pages 1, 2 or 4)
  // thread: two channels of a page, and a part of its tokens
  const int p = g % pages, part = g / pages, size = (1 << ltok) / parts;
  const int t0 = max(from, (p << ltok) + part * size), t1 = min(to, (p << ltok) + (part + 1) * size);
  Ends r;
  for (int t = t0; t < t1; ++t) r.take(l.val[t][c], l.val[t][c]);
  l.part[tid] = make_uint2(__builtin_bit_cast(uint32_t, r.lo), __builtin_bit_cast(uint32_t, r.hi));
  __syncthreads();
  if (part) return;
  for (int i = 1; i < parts; ++i) {
    const uint2 o = l.part[tid + i * pages * C];
    r.take(o.x, o.y);
  }
  uint32_t *b = max(from, p << ltok) < min(to, (p + 1) << ltok) ? page_at(p << ltok) : nullptr;
  if (!b) return;
  if (go_on) {
    const uint32_t x = ordered(b[c]), y = ordered(b[C + c]);
    r.take(x, y);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) r.lo[i] = r.hi[i] > 0x7f80 ? r.hi[i] : r.lo[i];  // (NaN)
  b[c] = ordered(__builtin_bit_cast(uint32_t, r.lo));
  b[C + c] = ordered(__builtin_bit_cast(uint32_t, r.hi));
}

// Eight channels of token t for its page's bounds.
template <int D> __device__ __forceinline__ void keep(BoundsLds<D> &l, int t, int oct, uint32_t w, uint32_t s) {
  const float f = __uint_as_float(s << 23);
  u32x4 x = {pair<0>(w, f), pair<1>(w, f), pair<2>(w, f), pair<3>(w, f)};
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = s == 255 ? 0x7fc07fc0u : ordered(x[e]);
  *reinterpret_cast<u32x4 *>(&l.val[t][4 * oct]) = x;
}

// The page of position `pos` of sequence b, or -1.
__device__ __forceinline__ int page_of(const CacheArgs &c, int b, int64_t pos) {
  if (pos < 0 || pos >= (int64_t)c.width << c.lpage) return -1;
  const int page = c.table[(int64_t)b * c.width + (pos >> c.lpage)];
  return page < 0 || page >= c.pages ? -1 : page;
}

// A workgroup's 64 positions, in the 64-bit and the thread's own terms: `base` the first one;
// tokens lo .. hi - 1 of them are new, those before `to` held, those from `old` on for the
// bounds of pages that get tokens. Thread: token t0 + r TOKENS, channels 8 oct on.
struct Span {
  int64_t base, first;  // first: of token 0 of the 64, in the call's tokens
  int lo, hi, to, old;
};

// One head after the other of a workgroup's share, from h on in steps; each thread's rows of
// the next head are on their way while one is worked on.
template <typename TI, int REP> struct Rows {
  const TI *p[REP];
  Raw<TI> next[REP];
  bool in[REP];
  int64_t step;
  __device__ __forceinline__ Rows(const View &v, int b, int h, int by, const Span &s, int t0, int tokens, int oct) {
    step = by * v.sh;
#pragma unroll
    for (int r = 0; r < REP; ++r) {
      const int t = t0 + r * tokens;
      in[r] = t >= s.lo && t < s.hi;
      p[r] = slice_of<TI>(v, b, h) + (s.first + (in[r] ? t : s.lo)) * v.st + 8 * oct;
      if (in[r]) next[r].load(p[r]);
    }
  }
  // row r of this head; with `more` the next head's is asked for
  __device__ __forceinline__ Raw<TI> take(int r, bool more) {
    const Raw<TI> x = next[r];
    p[r] += step;
    if (in[r] && more) next[r].load(p[r]);
    return x;
  }
};

template <typename TI, int D, int MODE>
__global__ __launch_bounds__(Threads<D>::N, 4) void append_kernel(AppendArgs a) {
  constexpr int NT = Threads<D>::N, OCTS = D / 8, TOKENS = NT / OCTS, REP = SUB / TOKENS;
  __shared__ __attribute__((aligned(16))) BoundsLds<D> lds;
  __shared__ Again<D> again;
  __shared__ int held_on[4];  // pages of the 64 positions (or -1)
  extern __shared__ __attribute__((aligned(16))) float2 turns_of[];  // [min(T, 64)][table.size()]
  const CacheArgs &c = a.c;
  const int tid = threadIdx.x, oct = tid % OCTS, t0 = tid / OCTS, n = a.rot / 2;
  const Table<MODE> table(n);
  const int b = blockIdx.x / a.spans, lspan = max(c.lpage, 6), ltok = min(c.lpage, 6);
  const int64_t start = c.starts[b], end = start + c.T;
  const int64_t p0 = ((start >> lspan) + (int)(blockIdx.x % a.spans)) << lspan;
  if (p0 >= end) return;
  const int64_t held = start + (c.counts ? min(max(c.counts[b], 0), c.T) : c.T);  // end of what is held
  // the share's kind (keys, values, queries), first head, heads and step
  const int share = blockIdx.y, kind = share < a.kshares ? 0 : share < a.kshares + a.vshares ? 1 : 2;
  const int h0 = share - (kind == 0 ? 0 : kind == 1 ? a.kshares : a.kshares + a.vshares);
  const int by = kind == 0 ? a.kshares : kind == 1 ? a.vshares : (int)gridDim.y - a.kshares - a.vshares;
  const int heads = kind == 2 ? a.H : c.Hkv;
  const bool bounds = kind == 0 && a.bounds && held > start;
  if (tid < 3) again.count[tid] = 0;
  int turns = 0;  // heads of keys so far
  for (int sub = 0; sub < 1 << (lspan - 6); ++sub) {
    Span s;
    s.base = p0 + sub * SUB;
    if (s.base >= end) break;
    s.first = s.base - start;
    s.lo = (int)min((int64_t)SUB, max((int64_t)0, -s.first)), s.hi = (int)min((int64_t)SUB, end - s.base);
    if (s.lo >= s.hi && !bounds) continue;
    const int64_t page0 = max(start >> c.lpage << c.lpage, (int64_t)0);
    s.old = (int)min((int64_t)SUB, max((int64_t)0, page0 - s.base));
    s.to = (int)max((int64_t)0, min((int64_t)SUB, held - s.base));
    Rows<TI, REP> rows(kind == 0 ? c.k : kind == 1 ? c.v : a.q, b, h0, by, s, t0, TOKENS, oct);
    __syncthreads();
    if (tid < 4) held_on[tid] = tid < SUB >> ltok ? page_of(c, b, s.base + (tid << ltok)) : -1;
    if (kind != 1) {
      // angles of the new tokens
      for (int e = tid; e < (s.hi - s.lo) * n; e += NT) {
        const int t = s.lo + e / n, m = e % n;
        float sn, cs;
        const double p = (double)(s.base + t);
        if (kind == 0) turn_key(p * a.freq[m], sn, cs);
        else turn_of(p, a.freq[m], sn, cs);
        turns_of[(t - s.lo) * table.size() + table.at(m)] = make_float2(cs * a.factor, sn * a.factor);
      }
    }
    __syncthreads();
    auto turn_at = [&](int t, bool in) { return turns_of + (in ? t - s.lo : 0) * table.size(); };
    if (kind == 2) {
      TI *out[REP];
#pragma unroll
      for (int r = 0; r < REP; ++r)
        out[r] = slice_of<TI>(a.qo, b, h0) + (s.first + t0 + r * TOKENS) * a.qo.st + 8 * oct;
#pragma unroll 1
      for (int h = h0; h < heads; h += by) {
#pragma unroll
        for (int r = 0; r < REP; ++r) {
          const TI *row = rows.p[r] - 8 * oct;
          const Raw<TI> raw = rows.take(r, h + by < heads);
          Chunk x;
          pairs_of<TI, MODE>(raw, rows.in[r] ? row : nullptr, oct, n, x);
          float z[8];
          turned<MODE>(x, turn_at(t0 + r * TOKENS, rows.in[r]), oct, n, z);
          if (rows.in[r]) store8(out[r], z);
          out[r] += by * a.qo.sh;
        }
      }
      continue;
    }
    // where the thread's tokens are held: the codes of its channels, and their group's scale
    // byte behind them; steps of a head
    const int codes = D / 2 << c.lpage;
    const int64_t block = codes + (D / 32 << c.lpage);
    uint8_t *at[REP];
#pragma unroll
    for (int r = 0; r < REP; ++r) {
      const int t = t0 + r * TOKENS, page = t < s.to ? held_on[t >> ltok] : -1;
      at[r] = page < 0 ? nullptr : c.cache + (((int64_t)page * 2 + kind) * c.Hkv + h0) * block;
    }
    auto token_of = [&](int t) { return (int)((s.base + t) & ((1 << c.lpage) - 1)); };
    if (kind == 1) {
#pragma unroll 1
      for (int h = h0; h < heads; h += by) {
#pragma unroll
        for (int r = 0; r < REP; ++r) {
          const Raw<TI> raw = rows.take(r, h + by < heads);
          float x[8];
          raw.values(x);
          uint32_t w, sc;
          quantise(x, w, sc);
          if (at[r]) {
            if (rows.in[r]) put<D>(w, sc, at[r], token_of(t0 + r * TOKENS), 1, oct, c.lpage);
            at[r] += by * block;
          }
        }
      }
      continue;
    }
#pragma unroll 1
    for (int h = h0; h < heads; h += by, ++turns) {
      if (bounds && s.old < s.lo) {
        // the page's earlier tokens
        uint32_t w[REP], sc[REP];
#pragma unroll
        for (int r = 0; r < REP; ++r) {
          const int t = t0 + r * TOKENS;
          sc[r] = 256;
          if (at[r] && t >= s.old && t < s.lo) held_of<D>(at[r], token_of(t), 0, oct, c.lpage, w[r], sc[r]);
        }
#pragma unroll
        for (int r = 0; r < REP; ++r)
          if (sc[r] < 256) keep<D>(lds, t0 + r * TOKENS, oct, w[r], sc[r]);
      }
#pragma unroll
      for (int r = 0; r < REP; ++r) {
        const int t = t0 + r * TOKENS;
        const TI *row = rows.p[r] - 8 * oct;
        const Raw<TI> raw = rows.take(r, h + by < heads);
        if (!__any(rows.in[r])) continue;
        Chunk x;
        pairs_of<TI, MODE>(raw, rows.in[r] ? row : nullptr, oct, n, x);
        uint32_t w, sc;
        const bool open = quantise_turned<MODE>(x, turn_at(t, rows.in[r]), oct, n, a.factor, w, sc);
        const bool live = rows.in[r] && at[r];
        // a group goes again if one of its four lanes asks for it
        if (__ballot(open && live) >> (tid & 60) & 15) {
          if (tid % 4 == 0) again.list[atomicAdd(&again.count[turns % 3], 1)] = (uint16_t)(t * (D / 32) + oct / 4);
        } else if (live) {
          put<D>(w, sc, at[r], token_of(t), 0, oct, c.lpage);
          if (bounds) keep<D>(lds, t, oct, w, sc);
        }
      }
      __syncthreads();
      const int count = again.count[turns % 3];
      if (tid == 0) again.count[(turns + 2) % 3] = 0;
      if (count) {
        // (a lane a channel)
        const TI *src = slice_of<TI>(c.k, b, h) + s.first * c.k.st;
        for (int e = tid / 32; e < count; e += NT / 32) {
          const int t = again.list[e] / (D / 32), ch = again.list[e] % (D / 32) * 32 + tid % 32;
          uint32_t w, sc;
          quantise_turned64<TI, MODE>(src + t * c.k.st, (double)(s.base + t), ch, n, a, w, sc);
          if (ch % 8) continue;
          put<D>(w, sc, c.cache + cache_block<D>(held_on[t >> ltok], 0, h, c.Hkv, c.lpage), token_of(t), 0, ch / 8, c.lpage);
          if (bounds) keep<D>(lds, t, ch / 8, w, sc);
        }
        __syncthreads();
      }
      if (bounds)
        bounds_of<D>(lds, c.lpage, s.old, s.to, sub > 0, [&](int t) -> uint32_t * {
          const int page = held_on[t >> ltok];
          return page < 0 ? nullptr : a.bounds + ((int64_t)page * c.Hkv + h) * D;
        });
#pragma unroll
      for (int r = 0; r < REP; ++r)
        if (at[r]) at[r] += by * block;
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

template <typename TI, int D, int MODE> void append_mode(const AppendArgs &a, dim3 grid, hipStream_t s) {
  const size_t lds = (size_t)std::min(a.c.T, SUB) * Table<MODE>(a.rot / 2).size() * sizeof(float2);
  hipLaunchKernelGGL((append_kernel<TI, D, MODE>), grid, dim3(Threads<D>::N), lds, s, a);
}
template <typename TI, int D> void append_as(const AppendArgs &a, dim3 grid, hipStream_t s) {
  if (a.layout == KIA_ROTARY_NEIGHBOURS) append_mode<TI, D, NEIGHBOURS>(a, grid, s);
  else if (a.rot / 2 % 8 == 0) append_mode<TI, D, HALF8>(a, grid, s);
  else append_mode<TI, D, HALF>(a, grid, s);
}
template <int D> void append_d(const AppendArgs &a, dim3 grid, int dtype, hipStream_t s) {
  if (dtype == KIA_F32) append_as<float, D>(a, grid, s);
  else append_as<uint16_t, D>(a, grid, s);
}

}  // namespace

// Workgroups: the spans of 64 positions (or a page), and of each span's heads as many shares
// as make four workgroups a CU, twice what the registers let run at once (the prompts above with three
// / four / six / eight / twelve: 49 / 47 / 51 / 58 / 66 us: fewer leave the last round emptier, more
// compute the same angles again); keys, values and queries have shares of their own, by their
// heads and not by their work, of which keys have the most.
void launch_append(AppendArgs a, int d, int dtype, int cus, hipStream_t s) {
  const unsigned spans = (unsigned)a.c.B * a.spans;
  const int want = (int)std::max(1u, (4u * cus + spans - 1) / spans), all = 2 * a.c.Hkv + a.H;
  auto part = [&](int heads) { return std::min(heads, std::max(1, (heads * want + all - 1) / all)); };
  a.kshares = a.vshares = part(a.c.Hkv);
  const dim3 grid(spans, 2 * a.kshares + part(a.H));
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
