// kia_select.hip -- the pages that attention over a long cache reads: for every new token
// and key head those whose keys could score highest.
//
// A page's keys lie between its bounds lo and hi in every channel c, so no score q.k of the
// page is above sum_c max(q_c lo_c, q_c hi_c) = q+ . hi + q- . lo, with the positive and the
// negative parts of q. The largest of that over the key head's query heads ranks the page, and
// pages are ranked in 64 bits: of bf16 queries the terms and nearly every sum are exact there,
// so that the order depends on no order of summation.
//
// Sums in 64 bits for all pages would take longer than reading the bounds. The matrix unit
// finds them within an error E first (16 pages by 16 heads, bf16 operands, fp32 queries as
// three pieces), and the count-th largest, c, digit by digit of its bits. An approximate rank
// above c + 2 E is one of the count largest for certain, one below c - 2 E is none; only what
// lies between is summed in 64 bits and chosen from. E is 2^-13 of the largest page's sum of
// magnitudes: 2 D <= 256 products of bf16 queries, each rounded to 24 bits in the sum, add up
// to an eighth of that (three pieces: 768, to three eighths); magnitudes below 2^-96 count as
// that, for factors that the matrix unit may flush, and E has 2^-116 beside, for the products and
// sums that it may (768 times less than 2^-126): without it E itself is 0 for sums below 2^-136,
// whose ranks are rounded to multiples of 2^-149.
// Up to 500 pages of 32 sequences, 16 heads of 128 over 4 (17 MB of bounds), bf16: ranks 9.3 us,
// the cut and the list 7.1, both mostly loads that wait for each other; with 64-bit sums for all
// the two took 1.5 us longer together. One token of 12 heads of 64 over 63 pages, one launch: 8.4.
//
// A workgroup selects for a token and key head. Where it can rank all of its pages soon
// enough, it does that itself; else a launch before ranks them in batches.
#include "kia_around.hpp"
#include "kia_host.hpp"

namespace kia {
namespace {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
constexpr uint64_t ALWAYS = ~0ull;  // the rank of pages that are taken; 0: no candidate
constexpr uint32_t ALWAYS32 = ~0u;

// A double's place in their order as an integer (not 0 and not ALWAYS); NaN ranks as infinity.
__device__ __forceinline__ uint64_t rank_of(double x) {
  if (x != x) x = INFINITY;
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | 1ull << 63;
}
// A float's, and back.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b >> 31 ? ~b : b | 1u << 31;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

template <int CTRL> __device__ __forceinline__ double moved(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = __builtin_amdgcn_mov_dpp((int)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(b >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// The sum over the D / 8 lanes of a page.
template <int D> __device__ __forceinline__ double page_sum(double x) {
  x += moved<0xb1>(x);                           // quad_perm 1 0 3 2
  x += moved<0x4e>(x);                           // quad_perm 2 3 0 1
  if constexpr (D >= 64) x += moved<0x141>(x);   // row_half_mirror
  if constexpr (D >= 128) x += moved<0x140>(x);  // row_mirror
  return x;
}
struct Most { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); } };
struct Least { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return min(a, b); } };
// The larger magnitude, or NaN.
__device__ __forceinline__ float larger(float a, float b) {
  return __uint_as_float(max(__float_as_uint(a) & 0x7fffffffu, __float_as_uint(b) & 0x7fffffffu));
}
// (of magnitudes and NaNs as integers: NaN is the largest)
__device__ __forceinline__ float largest64(float x) {
  return __uint_as_float(over64(__float_as_uint(x) & 0x7fffffffu, Most()));
}

// What a token's selection goes by: its sequence, key head, place in the call and the page
// of its position (below 0: it sees nothing).
struct Token {
  int b, hk, t, at;
  __device__ __forceinline__ Token(const SelectArgs &a, int id) {
    t = id % a.T, hk = id / a.T % a.Hkv, b = id / a.T / a.Hkv;
    const int64_t length = min((int64_t)a.lengths[b], (int64_t)a.width << a.lpage);
    const int64_t pos = length - a.T + t;
    at = pos < 0 ? -1 : (int)(pos >> a.lpage);
  }
  __device__ __forceinline__ int page(const SelectArgs &a, int w) const {  // of the cache, or -1
    const int p = w <= at ? a.table[(int64_t)b * a.width + w] : -1;
    return p < 0 || p >= a.pages ? -1 : p;
  }
  __device__ __forceinline__ bool always(const SelectArgs &a, int w) const { return w < a.first || w > at - a.last; }
};

// Approximate ranks of the pages first .. end - 1 of a token by NW waves, into key[] (by
// number), and the largest error of one (the lanes' own parts of it; NaN: anything).
template <typename TI, int D, int NW>
__device__ __forceinline__ float approximate(const SelectArgs &a, const Token &k, int first, int end, uint32_t *key) {
  constexpr int NP = Pieces<TI>::N, N = D / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slot = lane & 15, kb = lane >> 4, G = a.H / a.Hkv;
  uint32_t error = 0;
  if (first >= end) return 0.f;
  for (int g0 = 0; g0 < G; g0 += 16) {
    // column `slot`: a head's queries, their two parts and their magnitudes
    bf16x8 plus[NP][N], minus[NP][N], size[N];
    const TI *q = slice_of<TI>(a.q, k.b, k.hk * G + min(g0 + slot, G - 1)) + k.t * a.q.st + 8 * kb;
#pragma unroll
    for (int c = 0; c < N; ++c) {
      float p[8], m[8], f[8];
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const f32x4 x = load4(q + 32 * c + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (a NaN stays in both)
          p[e + i] = x[i] < 0.f ? 0.f : x[i];
          m[e + i] = x[i] > 0.f ? 0.f : x[i];
          f[e + i] = fabsf(x[i]) < 0x1p-96f ? 0x1p-96f : fabsf(x[i]);
        }
      }
      bf16x8 y[NP], z[NP], x[1];
      to_pieces<NP>(p, y);
      to_pieces<NP>(m, z);
      to_pieces<1>(f, x);
      size[c] = x[0];
#pragma unroll
      for (int i = 0; i < NP; ++i) plus[i][c] = y[i], minus[i][c] = z[i];
    }
    // (a tile's bounds are on their way while the one before is worked on, and the table's
    // entry of the one after)
    // (without branches: a branch waits for what was loaded before it. Of no page the first one's
    // bounds are read, and nothing is taken from them)
    u32x4 lo[N], hi[N];
    const int *table = a.table + (int64_t)k.b * a.width;
    auto load = [&](int page) {
      const u32x4 *p = reinterpret_cast<const u32x4 *>(
          a.bounds + ((int64_t)(page < 0 || page >= a.pages ? 0 : page) * a.Hkv + k.hk) * D) + kb;
#pragma unroll
      for (int c = 0; c < N; ++c) lo[c] = p[4 * c], hi[c] = p[D / 8 + 4 * c];
    };
    int page = table[min(first + 16 * wave + slot, end - 1)];
    int next = table[min(first + 16 * (wave + NW) + slot, end - 1)];
    load(page);
    for (int w0 = first + 16 * wave; w0 < end; w0 += 16 * NW) {
      f32x4 sum = {}, far = {};
#pragma unroll
      for (int c = 0; c < N; ++c) {
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) {
          sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_op(hi[c]), plus[i][c], sum, 0, 0, 0);
          sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_op(lo[c]), minus[i][c], sum, 0, 0, 0);
        }
        u32x4 most;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // (as integers: NaN is above all)
          const u16x2 x = __builtin_bit_cast(u16x2, lo[c][e] & 0x7fff7fffu), y = __builtin_bit_cast(u16x2, hi[c][e] & 0x7fff7fffu);
          const u16x2 least = {0x0f80, 0x0f80};  // 2^-96
          most[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_max(x, y), least));
        }
        far = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_op(most), size[c], far, 0, 0, 0);
      }
      const uint32_t have = (uint32_t)__ballot(page >= 0 && page < a.pages && w0 + slot < end) & 0xffff;
      page = next;
      next = table[min(w0 + 32 * NW + slot, end - 1)];
      load(page);
      // page 4 kb + i of the tile, column `slot`
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (as keys, NaN as infinity; magnitudes as integers, NaN the largest)
        const uint32_t x = over16(key_of(sum[i] == sum[i] ? sum[i] : INFINITY), Most());
        const uint32_t f = max(__float_as_uint(far[i]) & 0x7fffffffu, sum[i] == sum[i] ? 0 : 0x7fc00000u);
        const int w = w0 + 4 * kb + i;
        const bool is = have >> (4 * kb + i) & 1;
        error = is ? max(error, f) : error;
        if (slot == 0 && w < end) key[w] = !is ? 0 : k.always(a, w) ? ALWAYS32 : g0 ? max(x, key[w]) : x;
      }
    }
  }
  return fmaf(__uint_as_float(error), 0x1p-13f, 0x1p-116f);
}

// The search for the place of a cut among the ranks K (32 or 64 bits) of a token's pages
// 0 .. n - 1, by NT threads, each with its first ones in registers.
constexpr int OPEN = 512;  // pages of a refinement that have a place in a list
template <int NT> struct SelectLds {
  uint32_t bins[256], sums[2][2 * NT / 64];
  uint64_t ends[2 * NT / 64];
  int pick[3];
  float errors[NT / 64];
  int open[OPEN], opened, above;  // of a refinement: its pages, how many, and how many are above
};
// What the `count` largest are: all candidates (every), else those that are taken in any case,
// ranks with (rank & mask) > cut, and of those equal to it the first `equal`.
template <typename K> struct Cut {
  K cut = (K)~(K)0, mask = (K)~(K)0;
  uint32_t equal, must;
  bool every;
};
template <int NT, typename K>
__device__ __forceinline__ Cut<K> cut_of(SelectLds<NT> &l, const K *rank, int n, int count) {
  constexpr int KEEP = 4, NW = NT / 64, BITS = 8 * sizeof(K);
  constexpr K ALWAYS = (K)~(K)0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  K mine[KEEP];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) mine[i] = tid + i * NT < n ? rank[tid + i * NT] : 0;
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < KEEP; ++i) f(mine[i]);
    for (int i = tid + KEEP * NT; i < n; i += NT) f(rank[i]);
  };
  // candidates, pages taken in any case, least and largest rank of the others
  uint32_t all = 0, must = 0;
  K least = ALWAYS, most = 0;
  each([&](K x) {
    all += x != 0;
    must += x == ALWAYS;
    if (x && x != ALWAYS) least = min(least, x), most = max(most, x);
  });
  all = over64(all, Sum()), must = over64(must, Sum());
  if constexpr (sizeof(K) == 4) {
    least = over64(least, Least()), most = over64(most, Most());
  } else {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      least = min(least, (K)__shfl_xor((unsigned long long)least, i));
      most = max(most, (K)__shfl_xor((unsigned long long)most, i));
    }
  }
  if (lane == 0) l.sums[0][wave] = all, l.sums[0][NW + wave] = must, l.ends[wave] = least, l.ends[NW + wave] = most;
  if (tid < 256) l.bins[tid] = 0;
  __syncthreads();
  all = must = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    all += l.sums[0][i], must += l.sums[0][NW + i];
    least = min(least, (K)l.ends[i]), most = max(most, (K)l.ends[NW + i]);
  }
  Cut<K> r;
  r.every = (int)all <= count;
  r.equal = r.every ? 0 : count - must;  // (must <= first + last <= count)
  r.must = must;
  if (!r.equal) return r;
  // (the undecided low bits)
  int bits = least == most ? 0 : sizeof(K) == 8 ? 64 - __builtin_clzll(least ^ most) : 32 - __builtin_clz((uint32_t)(least ^ most));
  r.mask = bits == BITS ? 0 : ALWAYS << bits;
  r.cut = most & r.mask;
  // (of an approximate rank 16 of the undecided bits. Where the ranks have their sign and five bits of
  // the exponent in common, what is left is below 2^-13 of a rank and so within E; else it is up to
  // 2^-7, and more pages are left open to the sums in 64 bits than need be: the selection is the same)
  for (int i = 0; bits > 0 && (sizeof(K) == 8 || i < 2); ++i) {
    const int shift = max(bits - 8, 0);
    const uint32_t digit = (1u << (bits - shift)) - 1;
    each([&](K x) {
      if (x && x != ALWAYS && (x & r.mask) == r.cut) atomicAdd(&l.bins[(uint32_t)(x >> shift) & digit], 1u);
    });
    __syncthreads();
    if (wave == 0) {
      // from the top: bins 255 - 4 lane and three below it, and how many lie above each
      uint32_t v[4], to = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = l.bins[255 - 4 * lane - i];
        l.bins[255 - 4 * lane - i] = 0;
        to += v[i];
      }
      uint32_t above = sum_to(to);
      above -= to;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < r.equal && above + v[i] >= r.equal)
          l.pick[0] = 255 - 4 * lane - i, l.pick[1] = (int)(r.equal - above), l.pick[2] = (int)v[i];
        above += v[i];
      }
    }
    __syncthreads();
    r.cut |= (K)l.pick[0] << shift;
    r.equal = (uint32_t)l.pick[1];
    bits = shift;
    r.mask = ALWAYS << bits;
    if (sizeof(K) == 8 && (int)r.equal == l.pick[2]) break;  // every rank with these digits is taken
  }
  return r;
}

// The list of what a cut among ranks takes, in order, NT pages at a time.
template <int NT>
__device__ __forceinline__ void write_list(SelectLds<NT> &l, const uint64_t *rank, int n, int count,
                                           const Cut<uint64_t> &c, int *list) {
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t done = 0, same = 0;
  int turn = 0;
  // a lane's place among the lanes of the workgroup that have one (a barrier a turn: turns
  // alternate between two rows of sums)
  auto place = [&](bool has, uint32_t &total) {
    const uint64_t ones = __ballot(has);
    uint32_t at = total + __popcll(ones & ((1ull << lane) - 1));
    if (lane == 0) l.sums[turn][wave] = __popcll(ones);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const uint32_t x = l.sums[turn][i];
      at += i < wave ? x : 0;
      total += x;
    }
    turn ^= 1;
    return at;
  };
  for (int i0 = 0; i0 < n; i0 += NT) {
    const uint64_t x = i0 + tid < n ? rank[i0 + tid] : 0;
    bool take = x && (c.every || x == ALWAYS || (x & c.mask) > c.cut);
    if (c.equal) {
      const bool eq = x && x != ALWAYS && (x & c.mask) == c.cut;
      const uint32_t before = place(eq, same);
      take = eq ? before < c.equal : take;
    }
    const uint32_t at = place(take, done);
    if (take && at < (uint32_t)count) list[at] = i0 + tid;
  }
  for (int i = done + tid; i < count; i += NT) list[i] = -1;
}

// The exact rank of a page by D / 8 lanes.
template <int D>
__device__ __forceinline__ uint64_t exact(const SelectArgs &a, const Token &k, int w, const float *rows, int oct) {
  const u32x4 *p = reinterpret_cast<const u32x4 *>(a.bounds + ((int64_t)k.page(a, w) * a.Hkv + k.hk) * D) + oct;
  const u32x4 lo = p[0], hi = p[D / 8];
  const int G = a.H / a.Hkv;
  uint64_t top = 0;
  for (int g = 0; g < G; ++g) {
    const float *q = rows + g * D + 8 * oct;
    double s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = q[i] > 0.f ? hi[i / 2] : lo[i / 2];
      s = fma((double)q[i], (double)__uint_as_float(i % 2 ? b & 0xffff0000u : b << 16), s);
    }
    top = max(top, rank_of(page_sum<D>(s)));
  }
  return top;
}

// A token's queries to LDS, [heads][D].
template <typename TI, int D, int NT> __device__ __forceinline__ void load_rows(const SelectArgs &a, const Token &k, float *rows) {
  for (int e = threadIdx.x; e < a.H / a.Hkv * (D / 4); e += NT) {
    const int g = e / (D / 4), c = e % (D / 4) * 4;
    *reinterpret_cast<f32x4 *>(rows + g * D + c) =
        load4(slice_of<TI>(a.q, k.b, k.hk * (a.H / a.Hkv) + g) + k.t * a.q.st + c);
  }
}

// The ranks in 64 bits of what the approximate ones leave open between c - 2 E and c + 2 E
// (c: the last that they would take, or its bounds): ALWAYS above, 0 below, the exact ones of
// the pages between. Where these are few they are chosen from at once, ALWAYS or 0. Whether
// a choice is left.
template <int D, int NT>
__device__ __forceinline__ bool refine(SelectLds<NT> &l, const SelectArgs &a, const Token &k, const uint32_t *key, int n,
                                       const Cut<uint32_t> &cut, float error, const float *rows, uint64_t *rank) {
  constexpr int OCTS = D / 8;
  constexpr uint64_t PENDING = 1;  // (no rank: -infinity has a larger one)
  const int tid = threadIdx.x, lane = tid & 63, oct = tid % OCTS;
  const float up = of_key(cut.cut | ~cut.mask) + 2.125f * error, down = of_key(cut.cut) - 2.125f * error;  // (and their roundings)
  for (int w = tid; w < n; w += NT) {
    const uint32_t x = key[w];
    const float v = of_key(x);
    uint64_t r = 0;
    if (x && (cut.every || x == ALWAYS32)) {
      r = ALWAYS;
    } else if (x && cut.equal && v > up) {
      r = ALWAYS;
      atomicAdd(&l.above, 1);
    } else if (x && cut.equal && !(v < down)) {
      r = PENDING;
      const int i = atomicAdd(&l.opened, 1);
      if (i < OPEN) l.open[i] = w;
    }
    rank[w] = r;
  }
  __syncthreads();
  const int open = l.opened, need = a.count - (int)cut.must - l.above;
  if (!open) return false;
  if (open > OPEN) {
    for (int w = tid / OCTS; w < n; w += NT / OCTS) {
      if (rank[w] != PENDING) continue;
      const uint64_t r = exact<D>(a, k, w, rows, oct);
      if (oct == 0) rank[w] = r;
    }
    __syncthreads();
    return true;
  }
  if (open > need) {
    for (int e = tid / OCTS; e < open; e += NT / OCTS) {
      const uint64_t r = exact<D>(a, k, l.open[e], rows, oct);
      if (oct == 0) rank[l.open[e]] = r;
    }
    __syncthreads();
    if (open > 64) return true;
  }
  if (tid < 64) {
    const int w = lane < open ? l.open[lane] : -1;
    const uint64_t r = w < 0 ? 0 : rank[w];
    int before = 0;  // those that come before this page
    if (open > need)
      for (int i = 0; i < open; ++i) {
        const int v = __builtin_amdgcn_readlane(w, i);
        const uint64_t o = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(r >> 32), i) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)r, i);
        before += o > r || (o == r && v < w);
      }
    if (open <= 64 && w >= 0) rank[w] = before < need ? ALWAYS : 0;
  }
  if (open > 64)  // (all of them)
    for (int e = tid; e < open; e += NT) rank[l.open[e]] = ALWAYS;
  __syncthreads();
  return false;
}

// A token's selection from its approximate ranks (`error`: the thread's part of E).
template <typename TI, int D, int NT>
__device__ __forceinline__ void select(SelectLds<NT> &l, const SelectArgs &a, const Token &k, int id, const uint32_t *key,
                                       float error, float *rows, uint64_t *rank) {
  const int n = k.at + 1;
  load_rows<TI, D, NT>(a, k, rows);
  error = largest64(error);
  if ((threadIdx.x & 63) == 0) l.errors[threadIdx.x >> 6] = error;
  if (threadIdx.x == 0) l.opened = l.above = 0;
  const Cut<uint32_t> cut = cut_of<NT>(l, key, n, a.count);
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) error = larger(error, l.errors[i]);
  Cut<uint64_t> last;
  last.every = true, last.equal = 0;
  if (refine<D, NT>(l, a, k, key, n, cut, error, rows, rank)) last = cut_of<NT>(l, rank, n, a.count);
  __syncthreads();
  write_list<NT>(l, rank, n, a.count, last, a.list + (int64_t)id * a.count);
}

// A token's workspace: ranks, approximate ranks, and the batches' errors.
constexpr int SCORE_NT = 256;
// (fp32 queries take three pieces' registers)
template <typename TI> constexpr int OWN_NT = sizeof(TI) == 4 ? 512 : 1024;
struct Space {
  uint64_t *rank;
  uint32_t *key;
  float *error;
  __device__ __forceinline__ Space(const SelectArgs &a, int id) {
    rank = reinterpret_cast<uint64_t *>(static_cast<char *>(a.ws) + id * select_space(a.width));
    key = reinterpret_cast<uint32_t *>(rank + a.width);
    error = reinterpret_cast<float *>(key + a.width);
  }
};

// Approximate ranks of a batch of pages of one token.
template <typename TI, int D> __global__ __launch_bounds__(SCORE_NT) void score_kernel(SelectArgs a) {
  constexpr int NW = SCORE_NT / 64;
  const int batches = (a.width + a.batch - 1) / a.batch;
  const int id = blockIdx.x / batches, batch = blockIdx.x % batches, first = batch * a.batch;
  const Token k(a, id);
  if (first > k.at) return;
  const Space to(a, id);
  const float e = largest64(approximate<TI, D, NW>(a, k, first, min(first + a.batch, k.at + 1), to.key));
  if (threadIdx.x % 64 == 0) to.error[batch * NW + threadIdx.x / 64] = e;
}

// A selection from the ranks of a launch before; its own ones in LDS for up to RANKS pages (0: in the
// workspace). 128 selections of up to 500 pages: 7.1 us, from the workspace one more; four of 3125: 10.8
// and 0.7 more. (With 1024 threads the first took one more too, with 256 the other five.)
template <typename TI, int D, int NT, int RANKS> __global__ __launch_bounds__(NT) void select_kernel(SelectArgs a) {
  extern __shared__ __attribute__((aligned(16))) float rows[];
  __shared__ SelectLds<NT> l;
  __shared__ uint64_t rank[RANKS ? RANKS : 1];
  const Token k(a, blockIdx.x);
  const Space from(a, blockIdx.x);
  float e = 0.f;
  for (int i = threadIdx.x; i / (SCORE_NT / 64) * a.batch <= k.at; i += NT) e = larger(e, from.error[i]);
  if constexpr (RANKS > 0) select<TI, D, NT>(l, a, k, blockIdx.x, from.key, e, rows, rank);
  else select<TI, D, NT>(l, a, k, blockIdx.x, from.key, e, rows, from.rank);
}

// Both for pages that one workgroup ranks.
template <typename TI, int D> __global__ __launch_bounds__(OWN_NT<TI>) void own_select_kernel(SelectArgs a) {
  extern __shared__ __attribute__((aligned(16))) float rows[];
  __shared__ SelectLds<OWN_NT<TI>> l;
  __shared__ uint64_t rank[SELECT_OWN];
  __shared__ uint32_t key[SELECT_OWN];
  const Token k(a, blockIdx.x);
  const float e = approximate<TI, D, OWN_NT<TI> / 64>(a, k, 0, k.at + 1, key);
  __syncthreads();
  select<TI, D, OWN_NT<TI>>(l, a, k, blockIdx.x, key, e, rows, rank);
}

template <typename TI, int D> void run(const SelectArgs &a, hipStream_t s) {
  const unsigned tokens = (unsigned)a.B * a.Hkv * a.T, batches = (a.width + a.batch - 1) / a.batch;
  const size_t lds = (size_t)(a.H / a.Hkv) * D * sizeof(float);
  if (a.own) {
    timed_call("kia_cache4_select", s, [&] {
      hipLaunchKernelGGL((own_select_kernel<TI, D>), dim3(tokens), dim3(OWN_NT<TI>), lds, s, a);
    });
    return;
  }
  timed_call("kia_cache4_score", s, [&] {
    hipLaunchKernelGGL((score_kernel<TI, D>), dim3(batches * tokens), dim3(SCORE_NT), 0, s, a);
  });
  timed_call("kia_cache4_select", s, [&] {
    const dim3 g(tokens);
    if (a.width <= 1024) hipLaunchKernelGGL((select_kernel<TI, D, 256, 1024>), g, dim3(256), lds, s, a);
    else if (a.width <= 4096) hipLaunchKernelGGL((select_kernel<TI, D, 1024, 4096>), g, dim3(1024), lds, s, a);
    else hipLaunchKernelGGL((select_kernel<TI, D, 1024, 0>), g, dim3(1024), lds, s, a);
  });
}

}  // namespace

void launch_select(const SelectArgs &a, int d, int dtype, hipStream_t s) {
  if (dtype == KIA_F32) {
    if (d == 32) run<float, 32>(a, s);
    else if (d == 64) run<float, 64>(a, s);
    else run<float, 128>(a, s);
  } else {
    if (d == 32) run<uint16_t, 32>(a, s);
    else if (d == 64) run<uint16_t, 64>(a, s);
    else run<uint16_t, 128>(a, s);
  }
}

}  // namespace kia
