// kia_cached.hip -- attention of a few new tokens over the 4-bit cache on gfx950, for
// one head dimension (KIA_HEAD): softmax, or the interval weights (LERP, Nearest; MinMax,
// FWM, resolved) of a model that was trained with them.
//
// Bound by memory: every visible key and value is read once, 17/32 byte a channel,
// and everything else hides under that. Rows (token, head of the key head's group)
// fill the 16 columns of v_mfma_f32_16x16x32_bf16, the keys its 16 rows: scores come
// as S^T, lane l holding of row l % 16 the keys 4 (l / 16) + i of each 16-key tile, and
// so its weights are the B operand of O^T = V^T P^T as they stand, with the key order
// 16 (e / 4) + 4 (l / 16) + e % 4 in the slots of 32 keys. The cache is laid out for
// that: a lane's share of a tile, of the keys by token and of the values by column
// with four tokens side by side, is one access of D / 8 bytes, and a wave's is
// contiguous. No LDS in the loop; codes become bf16 operands by one instruction a pair
// (values by another, which puts neighbouring tokens together).
//
// A wave takes 32 keys at a time, the four waves of a workgroup and the workgroups
// that share a row tile each take a part of the keys; parts are joined in order.
// Softmax runs in one pass with a running maximum. The interval weights' grid
// depends on the row's extrema, so a first pass over the keys alone (a third of the
// bytes) finds them; the weights are absolute then and the parts' sums just add.
// 32 sequences of up to 32 000 keys, 16 heads of 128 over 4, LERP: extrema 32 us (144 MB,
// 4.5 TB/s), weights 63 us (289 MB, 4.6 TB/s), join 6; Nearest takes as long, softmax 60 and 6.
// (While a tile's loads stood behind branches and the page's number came by vector loads, each
// wait was for all of them: 35 and 74 us.)
//
// bf16 queries: scores are sums of exact products, weights are rounded to bf16 (2^-8
// of each) for the product with V: an output's error is up to 1.4 times that of its own
// rounding (2-norm; with weights in two pieces 1.0 times, and their pass took 6 to 8%
// longer). fp32
// queries and weights go as three bf16 pieces (exact for 2^-100 to 2^126; smaller ones lose
// less than 2^-133), which the idle matrix unit takes for free. Sums, extrema and
// statistics are fp32.
#include "kia_host.hpp"
#include "kia_prefix.hpp"

#ifndef KIA_MODE
#define KIA_MODE 0
#endif

namespace kia {
namespace {

// Which keys a row sees: all of its sequence's up to its own (within a window, and the
// first ones); those of the pages that a list names for its token and key head; or those
// behind the tokens that the batch shares (kia_prefix.hpp takes these, in the launch's first
// workgroups).
enum { SEQUENCE, LISTED, BEHIND };
constexpr int MODE = KIA_MODE;

// A row's value over the lanes that share it, in a fixed order (with FEW the columns 8 and 4
// on, by rotations of the 16; then 16 and 32 lanes on).
template <bool FEW, class F> __device__ __forceinline__ float across(float x, F f) {
  if constexpr (FEW) {
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xf, 0xf, true)));
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x124, 0xf, 0xf, true)));
  }
  x = f(x, __shfl_xor(x, 16));
  return f(x, __shfl_xor(x, 32));
}
// The value of the lane 4 e on (in columns 0 .. 3; the others' results are not used).
__device__ __forceinline__ float from_column(float x, int e) {
  const int v = __float_as_int(x);
  const int y = e == 0   ? v
                : e == 1 ? __builtin_amdgcn_mov_dpp(v, 0x104, 0xf, 0xf, true)   // row_shl:4
                : e == 2 ? __builtin_amdgcn_mov_dpp(v, 0x108, 0xf, 0xf, true)   // row_shl:8
                         : __builtin_amdgcn_mov_dpp(v, 0x10c, 0xf, 0xf, true);  // row_shl:12
  return __int_as_float(y);
}

// The chunks of keys that rows at positions lo .. hi see: the first tokens', then the
// window's.
struct Chunks {
  int sink = 0, low = 0, count = 0;
  Chunks() = default;
  __device__ __forceinline__ Chunks(const CachedArgs &a, int lo, int hi) {
    const int from = max(0, lo - a.window + 1);  // (window INT_MAX: 0)
    low = from / CHUNK;
    const int first = min(a.sinks, from);
    sink = min(first / CHUNK + (first % CHUNK != 0), low);  // (up to 2^31 - 2 keys)
    count = hi < 0 ? 0 : sink + hi / CHUNK + 1 - low;
  }
  __device__ __forceinline__ int at(int n) const { return (n < sink ? n : low + n - sink) * CHUNK; }
};

// A sequence's keys.
struct Length { int n; };
__device__ __forceinline__ Length length_of(const CachedArgs &a, int b) {
  return {(int)min((int64_t)max(a.lengths[b], 0), (int64_t)a.width << a.lpage)};
}
// The positions of the first and the last row of a row tile.
struct Rows16 {
  int n, lo, hi;  // n: the sequence's keys
  __device__ __forceinline__ Rows16(const CachedArgs &a, int b, int tile) : Rows16(a, tile, length_of(a, b)) {}
  __device__ __forceinline__ Rows16(const CachedArgs &a, int tile, Length x) : n(x.n) {
    const unsigned G = (unsigned)a.H / (unsigned)a.Hkv, total = a.T * G;
    lo = n - a.T + (int)(tile * 16u / G);
    hi = n - a.T + (int)(min(tile * 16u + 15, total - 1) / G);
  }
  __device__ __forceinline__ Chunks chunks(const CachedArgs &a) const {
    return Chunks(a, max(lo, 0), hi);
  }
};

// The parts that the sequences' keys are cut into for one key head's row tile: about
// a.shares in all, of one size for every sequence, so that a batch of unequal lengths
// keeps all workgroups busy for the same time (32 000 keys to 1 000, 32 sequences:
// 18% longer with eight parts for each). Every sequence has one at least. Part w of
// all of them is part w - first of sequence b. (64 sequences at a time; at most
// a.shares + B parts in all.)
struct Share {
  int b = -1, first = 0, parts = 0;
  // which sequence part w belongs to (by_b: the parts of sequence w)
  __device__ __forceinline__ Share(const CachedArgs &a, int tile, int w, bool by_b) {
    const int lane = threadIdx.x & 63;
    auto count = [&](int i) { return i < a.B ? Rows16(a, i, tile).chunks(a).count : 0; };
    double all = 0;
    for (int i = 0; i < a.B; i += 64) {
      double c = count(i + lane);
#pragma unroll
      for (int k = 1; k < 64; k *= 2) c += __shfl_xor(c, k);
      all += c;
    }
    const int per = max(NWAVE, (int)ceil(all / a.shares));
    int base = 0;
    for (int i = 0; i < a.B; i += 64) {
      const int p = i + lane < a.B ? max(1, (count(i + lane) + per - 1) / per) : 0;
      int to = p;
#pragma unroll
      for (int k = 1; k < 64; k *= 2) {
        const int y = __shfl_up(to, k);
        if (lane >= k) to += y;
      }
      const uint64_t hit = __ballot(by_b ? i + lane == w : base + to > w);
      if (hit) {
        const int at = __builtin_ctzll(hit);
        b = __builtin_amdgcn_readfirstlane(i + at);
        parts = __builtin_amdgcn_readfirstlane(__shfl(p, at));
        first = __builtin_amdgcn_readfirstlane(base + __shfl(to, at)) - parts;
        return;
      }
      base += __shfl(to, 63);
    }
  }
};

// The same of what lies behind shared tokens: about a.spread parts in all, one at least and a.most at
// most for a sequence. (256 sequences at a time, whose lengths are asked for together, and sums
// without LDS.)
struct Spread {
  int b = -1, first = 0, parts = 0;
  Length length = {0};
  __device__ __forceinline__ Spread(const CachedArgs &a, int tile, int w) {
    constexpr int U = 4;
    const int lane = threadIdx.x & 63, before = a.shared / CHUNK;
    Length n[U];  // of sequences i + 64 u + lane
    auto load = [&](int i) {
#pragma unroll
      for (int u = 0; u < U; ++u) n[u] = length_of(a, min(i + 64 * u + lane, a.B - 1));
    };
    auto chunks = [&](int u) { return max(0, Rows16(a, tile, n[u]).chunks(a).count - before); };
    double all = 0;
    for (int i = 0; i < a.B; i += 64 * U) {
      load(i);
      uint32_t x = 0;  // (up to 2^28)
#pragma unroll
      for (int u = 0; u < U; ++u) x += i + 64 * u + lane < a.B ? chunks(u) : 0;
      all += over64(x & 0xffff, Sum()) + 65536.0 * over64(x >> 16, Sum());
    }
    const int per = max(NWAVE, (int)ceil(all / a.spread));
    int base = 0;
    for (int i = 0; i < a.B; i += 64 * U) {
      if (a.B > 64 * U) load(i);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = i + 64 * u + lane < a.B ? min(max(1, (chunks(u) + per - 1) / per), a.most) : 0;
        const int to = (int)sum_to((uint32_t)p);
        const uint64_t hit = __ballot(base + to > w);
        if (hit) {
          const int at = __builtin_ctzll(hit);
          b = __builtin_amdgcn_readfirstlane(i + 64 * u + at);
          length = {__builtin_amdgcn_readlane(n[u].n, at)};
          parts = __builtin_amdgcn_readlane(p, at);
          first = base + __builtin_amdgcn_readlane(to, at) - parts;
          return;
        }
        base += __builtin_amdgcn_readlane(to, 63);
      }
    }
  }
};
// Of part w of a key head's row tile: its place in the workspace, in rows.
__device__ __forceinline__ int64_t slot_of(const CachedArgs &a, int hk, int tile, int w) {
  const int slots = MODE == SEQUENCE ? a.shares + a.B : a.shares;
  return (((int64_t)hk * a.tiles + tile) * slots + w) * 16;
}

// What a workgroup takes: rows of tokens t0 on of sequence b, at positions lo .. hi, and
// chunks c0 .. c1 of their keys, as part w - first of `parts`.
struct Work {
  int b, t0, rows, n, lo, hi, first, parts, c0, c1;
  Chunks chunks;
  __device__ __forceinline__ Work(const CachedArgs &a, int tile, int w) {
    const int G = (unsigned)a.H / (unsigned)a.Hkv;
    Length length;
    if constexpr (MODE == SEQUENCE) {
      const Share share(a, tile, w, false);
      b = share.b, first = share.first, parts = share.parts;
      if (b < 0) return;
      length = length_of(a, b);
    } else if (MODE == BEHIND && a.plan) {
      const int4 x = a.plan[(int64_t)tile * a.shares + w];
      b = __builtin_amdgcn_readfirstlane(x.x), first = __builtin_amdgcn_readfirstlane(x.y);
      parts = __builtin_amdgcn_readfirstlane(x.z), length = {__builtin_amdgcn_readfirstlane(x.w)};
      if (b < 0) return;
    } else if (MODE == BEHIND && a.spread) {
      const Spread x(a, tile, w);
      b = x.b, first = x.first, parts = x.parts, length = x.length;
      if (b < 0) return;
    } else {
      // (as many parts for every sequence, or for every token of one)
      const unsigned id = (unsigned)w / (unsigned)a.parts;
      parts = a.parts, first = id * parts;
      b = MODE == LISTED ? id / (unsigned)a.T : id;
      length = length_of(a, b);
    }
    const Rows16 rows16(a, tile, length);
    n = rows16.n;
    if constexpr (MODE == LISTED) {
      t0 = first / parts - b * a.T, rows = G;
      lo = hi = n - a.T + t0;
      // (before the text too, so that the list need not wait for the length)
      chunks.count = (int)((((int64_t)a.count << a.lpage) + CHUNK - 1) / CHUNK);
    } else {
      t0 = 0, rows = a.T * G;
      lo = rows16.lo, hi = rows16.hi;
      chunks = rows16.chunks(a);
      if constexpr (MODE == BEHIND) {
        chunks.low = a.shared / CHUNK;
        chunks.count = max(0, chunks.count - chunks.low);
      }
    }
    c0 = share_of(chunks.count, w - first, parts);
    c1 = share_of(chunks.count, w - first + 1, parts);
  }
};

// FEW: a key head has at most four rows. The 16 columns then hold them four times over, and
// of the four keys that a lane has scores of it takes one's weight, the (l / 4)-th: a
// quarter of the work on weights. The interval weights are bound by that work: LERP over
// the 32 sequences above 76 -> 63 us; 32 sequences of 16 000 keys, 32 heads of 128 over 8,
// Nearest 117 -> 101. The softmax, whose maximum then crosses more lanes, gains nothing to
// speak of (103 and 101 us there), and extrema without the minimum lose by it (16 of those
// sequences in fp32: 40 -> 45 us).
// RT: row tiles of a wave over shared tokens (0: there are none).
template <typename TI, int D, int PASS, int CALIB, int RECON, bool FEW, int RT>
__global__ __launch_bounds__(64 * NWAVE, 2) void cached_kernel(CachedArgs a) {
  constexpr int NP = Pieces<TI>::N, N = D / 32, NT = D / 16, NE = FEW ? 1 : 4;
  constexpr bool VALUES = PASS != PASS_EXTREMA;
  __shared__ WaveStats stats[RT ? RT : 1];
  WaveStats &red = stats[0];
  __shared__ int2 listed[MODE == LISTED ? LISTED_MOST : 1];
  __shared__ __attribute__((aligned(16))) float rows[VALUES ? NWAVE * 16 * (D + 4) : 4];
  const int tid = threadIdx.x, lane = tid & 63, kb = lane >> 4;
  const int slot = lane & 15;               // its key of a tile, its channels of the values
  const int col = FEW ? slot & 3 : slot;    // its row
  const int own = FEW ? slot >> 2 : 0;      // of its four scores a tile, the one it weighs
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  unsigned block_id = blockIdx.x;
  if constexpr (RT > 0) {
    if (block_id < a.pre.blocks) {
      prefix_part<TI, D, PASS, CALIB, RECON, RT>(a, stats, rows);
      return;
    }
    block_id -= a.pre.blocks;
  }
  const unsigned pair = block_id / (unsigned)a.Hkv;
  const int hk = block_id % (unsigned)a.Hkv, tile = pair % (unsigned)a.tiles, w = pair / (unsigned)a.tiles;
  const Work work(a, tile, w);
  if (work.b < 0) return;
  const int b = work.b, G = (unsigned)a.H / (unsigned)a.Hkv, total = work.rows, lo = work.lo, hi = work.hi;
  // this lane's row, and its position (-1 or less: before the text, sees nothing)
  const unsigned r = min(tile * 16 + col, total - 1);
  const int t = work.t0 + r / (unsigned)G, h = hk * G + r % (unsigned)G;
  const int pos = work.n - a.T + t;
  const int c0 = work.c0, c1 = work.c1;

  bf16x8 q[NP][N];
  {
    const TI *p = slice_of<TI>(a.q, b, h) + t * a.q.st + kb * (D / 4);
#pragma unroll
    for (int c = 0; c < N; ++c) load_query<TI>(p + 8 * c, q, c);
  }

  // the list's pages of this part, and where they stand in the text (-1: none)
  const int per = a.lpage - 4;  // (a page is 2^per tiles)
  const int e0 = (2 * c0) >> per;
  if constexpr (MODE == LISTED) {
    const int *list = a.list + (((int64_t)b * a.Hkv + hk) * a.T + work.t0) * a.count;
    const int e1 = min(min(a.count, e0 + LISTED_MOST), ((2 * c1 - 1) >> per) + 1);
    for (int e = e0 + tid; e < e1; e += 64 * NWAVE) {
      const int at = list[e];
      const int page = at >= 0 && at < a.width ? a.table[(int64_t)b * a.width + at] : -1;
      listed[e - e0] = make_int2(page >= 0 && page < a.pages ? page : -1, at);
    }
    __syncthreads();
  }

  const int codes = D / 2 << a.lpage;
  const int64_t block = (int64_t)codes + (D / 32 << a.lpage);  // bytes of a head's block
  // (the table's entries of a chunk are asked for a turn before its keys)
  int entry[TILES];
  auto ask = [&](int c) {
    if constexpr (MODE != LISTED) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int at = (work.chunks.at(min(c, c1 - 1)) + 16 * i) >> a.lpage;
        entry[i] = entry_of(a.table, (int64_t)b * a.width + min(at, a.width - 1));
        if (at >= a.width) entry[i] = -1;
      }
    }
  };
  Offsets<D> where(lane);
  auto load = [&](int c, Stage4<D, VALUES> &x) {
    where.hold();
    x.ok = 0;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      int key, page;
      if constexpr (MODE == LISTED) {
        const int e = (2 * c + i) >> per;
        const int2 y = e < a.count ? listed[e - e0] : make_int2(-1, -1);
        page = __builtin_amdgcn_readfirstlane(y.x);
        // (a page past the table has no number, so no product overflows)
        key = page < 0 ? 0
                       : (__builtin_amdgcn_readfirstlane(y.y) << a.lpage) + ((2 * c + i) & ((1 << per) - 1)) * 16;
        if (key > pos) page = -1;
      } else {
        key = work.chunks.at(c) + 16 * i;
        page = entry[i];
      }
      const bool ok = page >= 0 && page < a.pages;
      x.at[i] = key;
      x.ok |= ok << i;
      load_tile<D, VALUES>(a.cache + cache_block<D>(ok ? page : 0, 0, hk, a.Hkv, a.lpage), a.Hkv * block,
                           key & ((1 << a.lpage) - 1), codes, where, i, x);
    }
  };

  // the row's grid, from the extrema that the first pass left
  RowConst rc{};
  float Mx = -INFINITY, Mn = INFINITY;
  if constexpr (PASS == PASS_GRID) {
    const float2 *e = reinterpret_cast<const float2 *>(a.ext) +
                      slot_of(a, hk, tile, work.first) + col;
#pragma unroll 4
    for (int i = kb; i < work.parts; i += 4) {
      const float2 x = e[16 * i];
      Mx = fmaxf(Mx, x.x);
      Mn = fminf(Mn, x.y);
    }
    if constexpr (MODE == BEHIND) {
      // and over the shared tokens
      e = reinterpret_cast<const float2 *>(a.pre.ext) + a.pre.slot(hk, b * total + r);
      for (int i = kb; i < a.pre.parts; i += 4) {
        const float2 x = e[16 * i];
        Mx = fmaxf(Mx, x.x);
        Mn = fminf(Mn, x.y);
      }
    }
    Mx = fmaxf(Mx, __shfl_xor(Mx, 16));
    Mx = fmaxf(Mx, __shfl_xor(Mx, 32));
    Mn = fminf(Mn, __shfl_xor(Mn, 16));
    Mn = fminf(Mn, __shfl_xor(Mn, 32));
    Mx *= a.scale, Mn *= a.scale;
    rc = row_const(Mx, Mn, a.K, CALIB, a.tau, a.scale);
  }
  const float c2 = a.scale * 1.44269504f;

  f32x4 o[VALUES ? NT : 1] = {};
  float m = -INFINITY, l = 0.f, low = INFINITY;  // (extrema: m and low)
  Stage4<D, VALUES> cur, nxt;
  int c = c0 + wave;
  if (c < c1) {
    ask(c);
    load(c, cur);
    ask(c + NWAVE);
  }
  for (; c < c1; c += NWAVE) {
    // (the last chunk again at the end: behind a branch, the wait for this chunk would be one for
    // what the branch may have asked for too)
    load(min(c + NWAVE, c1 - 1), nxt);
    ask(c + 2 * NWAVE);
    if (MODE == LISTED && !cur.ok) {
      cur = nxt;
      continue;
    }
    // every row of the tile sees every key of the chunk
    const int j = cur.at[0], end = (MODE == LISTED ? max(cur.at[0], cur.at[1]) + 16 : j + CHUNK) - 1;
    const bool all = end <= lo && cur.ok == (1 << TILES) - 1 &&
                     (MODE == LISTED || (int64_t)hi - j < a.window || end < a.sinks);
    // tile i's key 4 kb + e
    auto key_at = [&](int i, int e) { return (MODE == LISTED ? cur.at[i] : j + 16 * i) + 4 * kb + e; };
    auto sees = [&](int key, int i) {
      return key <= pos && ((int64_t)pos - key < a.window || key < a.sinks) && (cur.ok >> i & 1);
    };
    // groups that hold an infinity or NaN
    const bool bad = __any(holds_nan<D, VALUES>(cur));
    float Q[TILES][4];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const float f = scale_of(cur.ks[i]);
      f32x4 acc = {};
      u32x4 w[N];
#pragma unroll
      for (int x = 0; x < N; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[x][e] = pair_at(e, cur.k[i][x], f);
#pragma unroll
      for (int p = NP - 1; p >= 0; --p)
#pragma unroll
        for (int x = 0; x < N; ++x) acc = mma16(as_op(w[x]), q[p][x], acc);
#pragma unroll
      for (int e = 0; e < 4; ++e) Q[i][e] = acc[e];
    }
    if (__builtin_expect(bad, 0)) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        uint64_t y = __ballot(cur.ks[i] == 255);
        y |= y >> 32;
        y |= y >> 16;
#pragma unroll
        for (int e = 0; e < 4; ++e) Q[i][e] = y >> (4 * kb + e) & 1 ? NAN : Q[i][e];
      }
    }
    // the scores of the keys that the lane weighs: tile i's 4 kb + own + e
    float S[TILES][NE];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      if constexpr (FEW)
        S[i][0] = own < 2 ? (own ? Q[i][1] : Q[i][0]) : own == 2 ? Q[i][2] : Q[i][3];
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i][e] = Q[i][e];
    }
    auto counts = [&](int i, int e) { return sees(key_at(i, own + e), i); };
    if (!all) {
#pragma unroll
      for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int e = 0; e < NE; ++e) S[i][e] = counts(i, e) ? S[i][e] : -INFINITY;
    }
    if constexpr (PASS == PASS_EXTREMA) {
#pragma unroll
      for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          m = fmaxf(m, S[i][e]);
          const bool in = all || counts(i, e);
          if constexpr (CALIB != CAL_FWM) low = in ? fminf(low, S[i][e]) : low;
        }
    } else {
      float w[TILES][NE];
      if constexpr (PASS == PASS_SOFTMAX) {
        float top = S[0][0];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < NE; ++e) top = fmaxf(top, S[i][e]);
        // (moved, and the sums scaled, only when passed by 2^8, row by row: no row's bits
        // depend on another's. Where no lane sees that, no row does)
        if (__any((top - m) * c2 > 8.f)) {
          top = across<FEW>(top, [](float x, float y) { return fmaxf(x, y); });
          const bool up = (top - m) * c2 > 8.f;
          const float f = up ? __builtin_amdgcn_exp2f((m - top) * c2) : 1.f;
          m = up ? top : m;
          l *= f;
#pragma unroll
          for (int x = 0; x < NT; ++x) o[x] *= f;
        }
        const float mm = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < NE; ++e) w[i][e] = __builtin_amdgcn_exp2f((S[i][e] - mm) * c2);
      } else {
        grid_weights<CALIB, RECON, NE>(S, w, rc, Mx, Mn, a);
        if (!all) {
#pragma unroll
          for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int e = 0; e < NE; ++e)
              w[i][e] = counts(i, e) ? w[i][e] : 0.f;
        }
      }
      if (!all) {
        // values of tokens that no row sees (past the end, on no page) as zeros
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key_at(i, e) > hi || !(cur.ok >> i & 1)) cur.clear(i, e);
      }
      if (__builtin_expect(bad, 0)) {
        // groups of NaN: their values as zeros here, and NaN for the rows that see them
        bf16x8 is[TILES / 2], one[TILES / 2];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool nan = (cur.vs[i] >> (8 * e) & 255) == 255;
            if (nan) cur.clear(i, e);
            is[i / 2][i % 2 * 4 + e] = (__bf16)(nan ? 1.f : 0.f);
            one[i / 2][i % 2 * 4 + e] = (__bf16)(sees(key_at(i, e), i) ? 1.f : 0.f);
          }
        // (column `slot` of the values here is row 4 kb + e of the sums)
        f32x4 k = {};
#pragma unroll
        for (int u = 0; u < TILES / 2; ++u) k = mma16(is[u], one[u], k);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int x = 0; x < NT; ++x) o[x][e] = k[e] > 0.f ? NAN : o[x][e];
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        if constexpr (FEW) l += w[i][0];
        else l += (w[i][0] + w[i][1]) + (w[i][2] + w[i][3]);
      }
#pragma unroll
      for (int u = 0; u < TILES / 2; ++u) {
        // the weights of the lane's eight keys of 32, and those keys' values
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (FEW) x[e] = from_column(w[2 * u + e / 4][0], e % 4);
          else x[e] = w[2 * u + e / 4][e % 4];
        }
        bf16x8 p[NP];
        to_pieces<NP>(x, p);
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = scale_of(cur.vs[2 * u + e / 4] >> (8 * (e % 4)) & 255);
#pragma unroll
        for (int y = 0; y < NT / 2; ++y) {
          u32x4 even, odd;
          value_ops<D>(cur, f, u, y, even, odd);
#pragma unroll
          for (int i = NP - 1; i >= 0; --i) {
            o[2 * y] = mma16(as_op(even), p[i], o[2 * y]);
            o[2 * y + 1] = mma16(as_op(odd), p[i], o[2 * y + 1]);
          }
        }
      }
    }
    cur = nxt;
  }

  const int64_t out = slot_of(a, hk, tile, w);
  if constexpr (MODE == BEHIND && PASS != PASS_GRID) {
    // (the first pass, for later launches)
    if (a.spread && !a.plan && hk == 0 && w == work.first && tid == 0)
      a.own[(int64_t)tile * a.B + b] = make_int2(work.first, work.parts);
  }
  if constexpr (PASS == PASS_EXTREMA) {
    m = across<FEW>(m, [](float x, float y) { return fmaxf(x, y); });
    low = across<FEW>(low, [](float x, float y) { return fminf(x, y); });
    if (kb == 0) red[wave][col][0] = m, red[wave][col][1] = low;
    __syncthreads();
    if (tid < (FEW ? 4 : 16)) {
#pragma unroll
      for (int i = 1; i < NWAVE; ++i) {
        m = fmaxf(m, red[i][col][0]);
        low = fminf(low, red[i][col][1]);
      }
      a.ext[(out + col) * 2] = m;
      a.ext[(out + col) * 2 + 1] = low;
    }
  } else {
    l = across<FEW>(l, [](float x, float y) { return x + y; });
    if (kb == 0) red[wave][col][0] = m, red[wave][col][1] = l;
    // channel (4 kb + e) NT + x of row `col`
    if (!FEW || own == 0) {
      float *mine = rows + (wave * 16 + col) * (D + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int x = 0; x < NT; ++x) mine[(4 * kb + e) * NT + x] = o[x][e];
    }
    __syncthreads();
    // joined in wave order: 256 threads, 16 rows, D / 16 channels each
    const int row = tid / 16, part = tid % 16;
    float top = 0.f;
    if constexpr (PASS == PASS_SOFTMAX) {
      top = red[0][row][0];
#pragma unroll
      for (int i = 1; i < NWAVE; ++i) top = fmaxf(top, red[i][row][0]);
      if (top == -INFINITY) top = 0.f;
    }
    float sum = 0.f, x[NT] = {};
#pragma unroll
    for (int i = 0; i < NWAVE; ++i) {
      const float f = PASS == PASS_SOFTMAX ? __builtin_amdgcn_exp2f((red[i][row][0] - top) * c2) : 1.f;
      sum = fmaf(red[i][row][1], f, sum);
#pragma unroll
      for (int e = 0; e < NT; ++e)
        x[e] = fmaf(rows[(i * 16 + row) * (D + 4) + part * NT + e], f, x[e]);
    }
    if (MODE != BEHIND && work.parts == 1) {
      const int rr = tile * 16 + row;
      if (rr < total) {
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        TI *y = slice_of<TI>(a.o, b, hk * G + rr % G) + (work.t0 + rr / G) * a.o.st + part * NT;
#pragma unroll
        for (int e = 0; e < NT; ++e) {
          if constexpr (sizeof(TI) == 4) y[e] = x[e] * f;
          else y[e] = (uint16_t)cvt_bf16x2(x[e] * f, 0.f);
        }
      }
    } else if (tile * 16 + row < total) {
      float *y = a.part + (out + row) * D + part * NT;
#pragma unroll
      for (int e = 0; e < NT; ++e) y[e] = x[e];
      if (part == 0) {
        a.stat[(out + row) * 2] = PASS == PASS_SOFTMAX ? top : 0.f;
        a.stat[(out + row) * 2 + 1] = sum;
      }
    }
  }
}

// The power of two that a part's maximum m stands for, behind `top`: of a sequence's own keys m is a
// score, of shared ones in log2 units already (`shared`), and so is `top` where there are shared ones.
__device__ __forceinline__ float power_of(float m, float top, bool shared, float c2) {
  if constexpr (MODE == BEHIND) return shared ? m - top : fmaf(m, c2, -top);
  else return (m - top) * c2;
}
__device__ __forceinline__ float top_of(float m, bool shared, float c2) {
  return MODE == BEHIND && !shared ? m * c2 : m;
}

// The parts of one row, joined in order: D / 4 threads a part, the parts in 1024 / D
// groups whose sums are added in order of the groups.
template <typename TI, int D> __global__ __launch_bounds__(256) void join_kernel(CachedArgs a) {
  constexpr int W = D / 4, NG = 256 / W;
  __shared__ float f[256], red[8];  // (at most 256 parts)
  __shared__ f32x4 sums[NG][W];
  const unsigned kvs = a.B * a.Hkv, s = blockIdx.x % kvs, b = s / (unsigned)a.Hkv, hk = s % (unsigned)a.Hkv;
  const unsigned G = (unsigned)a.H / (unsigned)a.Hkv, r = blockIdx.x / kvs;  // r: token and head
  const int tid = threadIdx.x, wave = tid >> 6;
  int64_t first, before = 0;
  int parts, shared = 0;  // parts over the shared tokens, then the row's own
  if constexpr (MODE == SEQUENCE) {
    const Share share(a, r / 16, b, true);
    if (share.parts == 1) return;  // (written by its only part)
    first = slot_of(a, hk, r / 16, share.first) + r % 16;
    parts = share.parts;
  } else if constexpr (MODE == LISTED) {
    first = slot_of(a, hk, r % G / 16, (b * a.T + r / G) * a.parts) + r % G % 16;
    parts = a.parts;
  } else {
    const int2 own = own_parts(a, r / 16, b);
    first = slot_of(a, hk, r / 16, own.x) + r % 16;
    before = a.pre.slot(hk, b * a.T * G + r);
    shared = a.pre.parts;
    parts = own.y + shared;
  }
  const float c2 = a.scale * 1.44269504f;
  float m = -INFINITY, l = 0.f;
  if (tid < parts) {
    const float2 st = tid < shared ? reinterpret_cast<const float2 *>(a.pre.stat)[before + 16 * tid]
                                   : reinterpret_cast<const float2 *>(a.stat)[first + 16 * (tid - shared)];
    l = st.y;
    if (l != 0.f) m = st.x;  // (a part that saw a key)
  }
  float top = top_of(m, tid < shared, c2);
#pragma unroll
  for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
  if ((tid & 63) == 0) red[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float g = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(power_of(m, top, tid < shared, c2));
  float sum = l * g;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
  f[tid] = g;
  if ((tid & 63) == 0) red[4 + wave] = sum;
  __syncthreads();
  const int at = tid % W, grp = tid / W;
  const f32x4 *p = reinterpret_cast<const f32x4 *>(a.part + first * D) + at;
  f32x4 x = {};
  if constexpr (MODE == BEHIND) {
    const f32x4 *y = reinterpret_cast<const f32x4 *>(a.pre.part + before * D) + at;
#pragma unroll 4
    for (int i = grp; i < parts; i += NG)
      x += (i < shared ? y[(int64_t)i * 16 * W] : p[(int64_t)(i - shared) * 16 * W]) * f[i];
  } else {
#pragma unroll 4
    for (int i = grp; i < parts; i += NG)
      x += p[(int64_t)i * 16 * W] * f[i];  // (a NaN stays one, however small its part's weight)
  }
  sums[grp][at] = x;
  __syncthreads();
  if (grp) return;
#pragma unroll
  for (int i = 1; i < NG; ++i) x += sums[i][at];
  sum = (red[4] + red[5]) + (red[6] + red[7]);
  x *= sum == 0.f ? 0.f : 1.f / sum;
  TI *y = slice_of<TI>(a.o, b, hk * G + r % G) + r / G * a.o.st + 4 * at;
  if constexpr (sizeof(TI) == 4) *reinterpret_cast<f32x4 *>(y) = x;
  else *reinterpret_cast<u32x2 *>(y) = u32x2{cvt_bf16x2(x[0], x[1]), cvt_bf16x2(x[2], x[3])};
}

// The same for many rows of few parts: D / 4 lanes a row, which walk its parts in order, and
// 1024 / D rows a workgroup. (4096 rows of five parts: 5.0 us, a workgroup each 8.3; 1024 rows of 13
// parts 5.6 and 4.4.)
template <typename TI, int D> __global__ __launch_bounds__(256) void join_few_kernel(CachedArgs a) {
  constexpr int W = D / 4, ROWS = 256 / W;
  const unsigned G = (unsigned)a.H / (unsigned)a.Hkv, per = a.T * G, id = blockIdx.x * ROWS + threadIdx.x / W;
  const int at = threadIdx.x % W;
  if (id >= (unsigned)a.B * a.H * a.T) return;
  // rows of a key head and sequence side by side
  const unsigned r = id % per, hk = id / per % (unsigned)a.Hkv, b = id / per / (unsigned)a.Hkv;
  int64_t first, before = 0;
  int shared = 0, parts;
  if constexpr (MODE == LISTED) {
    first = slot_of(a, hk, r % G / 16, (b * a.T + r / G) * a.parts) + r % G % 16;
    parts = a.parts;
  } else {
    const int2 own = own_parts(a, r / 16, b);
    first = slot_of(a, hk, r / 16, own.x) + r % 16;
    before = a.pre.slot(hk, b * per + r);
    shared = a.pre.parts;
    parts = own.y + shared;
  }
  auto stat = [&](int i) {
    return i < shared ? reinterpret_cast<const float2 *>(a.pre.stat)[before + 16 * i]
                      : reinterpret_cast<const float2 *>(a.stat)[first + 16 * (i - shared)];
  };
  const float c2 = a.scale * 1.44269504f;
  float top = -INFINITY;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    const float2 s = stat(i);
    if (s.y != 0.f) top = fmaxf(top, top_of(s.x, i < shared, c2));  // (a part that saw a key)
  }
  const f32x4 *p = reinterpret_cast<const f32x4 *>(a.part + first * D) + at;
  const f32x4 *y = reinterpret_cast<const f32x4 *>(a.pre.part + before * D) + at;
  f32x4 x = {};
  float sum = 0.f;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    const float2 s = stat(i);
    const float g = s.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(power_of(s.x, top, i < shared, c2));
    sum = fmaf(s.y, g, sum);
    // (a NaN stays one, however small its part's weight)
    x += (i < shared ? y[(int64_t)i * 16 * W] : p[(int64_t)(i - shared) * 16 * W]) * g;
  }
  x *= sum == 0.f ? 0.f : 1.f / sum;
  TI *out = slice_of<TI>(a.o, b, hk * G + r % G) + r / G * a.o.st + 4 * at;
  if constexpr (sizeof(TI) == 4) *reinterpret_cast<f32x4 *>(out) = x;
  else *reinterpret_cast<u32x2 *>(out) = u32x2{cvt_bf16x2(x[0], x[1]), cvt_bf16x2(x[2], x[3])};
}

// The parts by lengths of what lies behind shared tokens, a wave each.
__global__ __launch_bounds__(64 * NWAVE) void plan_kernel(CachedArgs a) {
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * NWAVE + (threadIdx.x >> 6));
  if (id >= a.shares * a.tiles) return;
  const int tile = (unsigned)id / (unsigned)a.shares, w = (unsigned)id % (unsigned)a.shares;
  const Spread x(a, tile, w);
  if ((threadIdx.x & 63) != 0) return;
  a.plan[id] = make_int4(x.b, x.first, x.parts, x.length.n);
  if (x.b >= 0 && w == x.first) a.own[(int64_t)tile * a.B + x.b] = make_int2(x.first, x.parts);
}

// The passes' launches (g: workgroups, join: whether a row has several parts).
template <typename TI, int D, bool FEW, int CALIB, int RT>
void grid_passes(const CachedArgs &a, dim3 g, hipStream_t s) {
  const dim3 t(64 * NWAVE);
  timed_call("kia_cache4_extrema", s, [&] {
    hipLaunchKernelGGL((cached_kernel<TI, D, PASS_EXTREMA, CALIB, REC_LERP, FEW && CALIB != CAL_FWM, RT>),
                       g, t, 0, s, a);
  });
  timed_call("kia_cache4_attn", s, [&] {
    if (a.recon == REC_LERP)
      hipLaunchKernelGGL((cached_kernel<TI, D, PASS_GRID, CALIB, REC_LERP, FEW, RT>), g, t, 0, s, a);
    else
      hipLaunchKernelGGL((cached_kernel<TI, D, PASS_GRID, CALIB, REC_NEAREST, FEW, RT>), g, t, 0, s, a);
  });
}

template <typename TI, int D, int CALIB, int RT> void grid_rows(const CachedArgs &a, dim3 g, hipStream_t s) {
  if ((MODE == LISTED ? 1 : a.T) * (a.H / a.Hkv) <= 4) grid_passes<TI, D, true, CALIB, RT>(a, g, s);
  else grid_passes<TI, D, false, CALIB, RT>(a, g, s);
}

template <typename TI, int D, int RT> void run(const CachedArgs &a, bool join, hipStream_t s) {
  const int parts = MODE == SEQUENCE ? a.shares + a.B : a.shares;
  const dim3 g((RT ? a.pre.blocks : 0) + (unsigned)parts * a.Hkv * a.tiles);
  if constexpr (RT > 0) {
    if (a.plan)
      timed_call("kia_cache4_plan", s, [&] {
        hipLaunchKernelGGL(plan_kernel, dim3(((unsigned)a.shares * a.tiles + NWAVE - 1) / NWAVE), dim3(64 * NWAVE), 0, s, a);
      });
  }
  if (a.recon == REC_SOFTMAX) {
    timed_call("kia_cache4_attn", s, [&] {
      hipLaunchKernelGGL((cached_kernel<TI, D, PASS_SOFTMAX, CAL_FWM, REC_SOFTMAX, false, RT>), g,
                         dim3(64 * NWAVE), 0, s, a);
    });
  } else if (a.calib == CAL_MINMAX) {
    grid_rows<TI, D, CAL_MINMAX, RT>(a, g, s);
  } else if (a.calib == CAL_FWM) {
    grid_rows<TI, D, CAL_FWM, RT>(a, g, s);
  } else {
    grid_rows<TI, D, CAL_RESOLVED, RT>(a, g, s);
  }
  if (join) {
    timed_call("kia_cache4_join", s, [&] {
      if constexpr (MODE != SEQUENCE) {
        const unsigned rows = (unsigned)a.B * a.H * a.T, of = 1024 / D;
        if (a.parts + (RT ? a.pre.parts : 0) <= FEW_PARTS && rows >= MANY_ROWS) {
          hipLaunchKernelGGL((join_few_kernel<TI, D>), dim3((rows + of - 1) / of), dim3(256), 0, s, a);
          return;
        }
      }
      hipLaunchKernelGGL((join_kernel<TI, D>), dim3((unsigned)(a.B * a.Hkv) * (a.T * (a.H / a.Hkv))), dim3(256), 0,
                         s, a);
    });
  }
}
}  // namespace

template <int RT> static void run_typed(const CachedArgs &a, int dtype, bool join, hipStream_t s) {
  if (dtype == KIA_F32) run<float, KIA_HEAD, RT>(a, join, s);
  else run<uint16_t, KIA_HEAD, RT>(a, join, s);
}

#if KIA_MODE == 0
template <> void launch_cached<KIA_HEAD>(const CachedArgs &a, int dtype, hipStream_t s) {
  run_typed<0>(a, dtype, a.shares > 1, s);
}
#elif KIA_MODE == 1
template <> void launch_listed<KIA_HEAD>(const CachedArgs &a, int dtype, hipStream_t s) {
  run_typed<0>(a, dtype, a.parts > 1, s);
}
#else
template <> void launch_shared<KIA_HEAD>(const CachedArgs &a, int dtype, hipStream_t s) {
  const int rt = prefix_tiles(a.pre.tiles, KIA_HEAD, dtype);
  if (rt == 1) run_typed<1>(a, dtype, true, s);
  else if (dtype == KIA_BF16) run<uint16_t, KIA_HEAD, 2>(a, true, s);
  // (fp32 heads of 128: two tiles do not fit the registers)
  else run<float, KIA_HEAD, KIA_HEAD == 128 ? 1 : 2>(a, true, s);
}
#endif

}  // namespace kia
