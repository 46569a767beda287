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
// 32 sequences of up to 32 000 keys, 16 heads of 128 over 4, LERP: extrema 35 us (144 MB,
// 4.2 TB/s), weights 74 us (289 MB, 3.9 TB/s), join 6; Nearest takes as long.
//
// bf16 queries: scores are sums of exact products, weights are rounded to bf16 (2^-8
// of each) for the product with V: an output's error is up to 1.4 times that of its own
// rounding (2-norm; with weights in two pieces 1.0 times, and their pass takes 6 to 8%
// longer: 76 -> 81 us above, the softmax of kia_around_abi.hip's figures 59 -> 63). fp32
// queries and weights go as three bf16 pieces (exact for 2^-100 to 2^126; smaller ones lose
// less than 2^-133), which the idle matrix unit takes for free. Sums, extrema and
// statistics are fp32.
#include <limits.h>

#include "kia_cache.hpp"
#include "kia_host.hpp"

namespace kia {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 32 keys at a time: two tiles of 16 and the next two on their way leave room for three
// workgroups a CU in bf16 (162 registers; with 64 keys 217, two workgroups, and the
// interval weights of 32 x 16 500 keys took 101 us against 88).
constexpr int TILES = 2, CHUNK = 16 * TILES, NWAVE = 4;
enum { PASS_SOFTMAX, PASS_EXTREMA, PASS_GRID };

__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// byte `s` of a word of codes as two bf16
template <int S> __device__ __forceinline__ uint32_t pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, S));
}
__device__ __forceinline__ uint32_t pair_at(int s, uint32_t w, float scale) {
  return s == 0 ? pair<0>(w, scale) : s == 1 ? pair<1>(w, scale) : s == 2 ? pair<2>(w, scale)
                                                                     : pair<3>(w, scale);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// One lane's share of a chunk: codes and scales of its keys and values.
template <int D, bool VALUES> struct Stage4 {
  static constexpr int N = D / 32;  // words of codes of a 16-key tile
  uint32_t k[TILES][N], v[VALUES ? TILES : 1][N], vs[VALUES ? TILES : 1];
  uint8_t ks[TILES];
  int ok;  // bit t: the tile's page is one of the cache's
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
  int sink, low, count;
  __device__ __forceinline__ Chunks(const CachedArgs &a, int lo, int hi) {
    const int from = max(0, lo - a.window + 1);  // (window INT_MAX: 0)
    low = from / CHUNK;
    const int first = min(a.sinks, from);
    sink = min(first / CHUNK + (first % CHUNK != 0), low);  // (up to 2^31 - 2 keys)
    count = hi < 0 ? 0 : sink + hi / CHUNK + 1 - low;
  }
  __device__ __forceinline__ int at(int n) const { return (n < sink ? n : low + n - sink) * CHUNK; }
};

// The positions of the first and the last row of a row tile.
struct Rows16 {
  int n, lo, hi;  // n: the sequence's keys
  __device__ __forceinline__ Rows16(const CachedArgs &a, int b, int tile) {
    const int G = a.H / a.Hkv, total = a.T * G;
    n = (int)min((int64_t)max(a.lengths[b], 0), (int64_t)a.width << a.lpage);
    lo = n - a.T + tile * 16 / G;
    hi = n - a.T + min(tile * 16 + 15, total - 1) / G;
  }
  __device__ __forceinline__ Chunks chunks(const CachedArgs &a) const {
    return Chunks(a, max(lo, 0), hi);
  }
};

// The parts that the sequences' keys are cut into for one key head's row tile: about
// a.shares in all, of one size for every sequence, so that a batch of unequal lengths
// keeps all workgroups busy for the same time (32 000 keys to 1 000, 32 sequences:
// 158 us with eight parts for each, 134 us so). Every sequence has one at least. Part w of
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
// Of part w of a key head's row tile: its place in the workspace, in rows.
__device__ __forceinline__ int64_t slot_of(const CachedArgs &a, int hk, int tile, int w) {
  return (((int64_t)hk * a.tiles + tile) * (a.shares + a.B) + w) * 16;
}

// FEW: a key head has at most four rows. The 16 columns then hold them four times over, and
// of the four keys that a lane has scores of it takes one's weight, the (l / 4)-th: a
// quarter of the work on weights. The interval weights are bound by that work: LERP over
// the 32 sequences above 86 -> 76 us; 32 sequences of 16 000 keys, 32 heads of 128 over 8,
// Nearest with MinMax 124 -> 107 and its extrema 73 -> 65. The softmax, whose maximum then
// crosses more lanes, is not (118 and 119 us there), nor are extrema without the minimum
// (16 of those sequences in fp32: 40 -> 45 us).
template <typename TI, int D, int PASS, int CALIB, int RECON, bool FEW>
__global__ __launch_bounds__(64 * NWAVE, 2) void cached_kernel(CachedArgs a) {
  constexpr int NP = Pieces<TI>::N, N = D / 32, NT = D / 16, NE = FEW ? 1 : 4;
  constexpr bool VALUES = PASS != PASS_EXTREMA;
  __shared__ float red[NWAVE][16][2];
  __shared__ __attribute__((aligned(16))) float rows[VALUES ? NWAVE * 16 * (D + 4) : 4];
  const int tid = threadIdx.x, lane = tid & 63, kb = lane >> 4;
  const int slot = lane & 15;               // its key of a tile, its channels of the values
  const int col = FEW ? slot & 3 : slot;    // its row
  const int own = FEW ? slot >> 2 : 0;      // of its four scores a tile, the one it weighs
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hk = blockIdx.x % a.Hkv, tile = (int)(blockIdx.x / a.Hkv) % a.tiles;
  const int w = blockIdx.x / (a.Hkv * a.tiles);
  const Share share(a, tile, w, false);
  if (share.b < 0) return;
  const int b = share.b, G = a.H / a.Hkv, total = a.T * G;
  const Rows16 rows16(a, b, tile);
  const int lo = rows16.lo, hi = rows16.hi;
  // this lane's row, and its position (-1 or less: before the text, sees nothing)
  const int r = min(tile * 16 + col, total - 1), t = r / G, h = hk * G + r % G;
  const int pos = rows16.n - a.T + t;
  const Chunks chunks = rows16.chunks(a);
  const int c0 = (int)((int64_t)chunks.count * (w - share.first) / share.parts);
  const int c1 = (int)((int64_t)chunks.count * (w - share.first + 1) / share.parts);

  bf16x8 q[NP][N];
  {
    const TI *p = slice_of<TI>(a.q, b, h) + t * a.q.st + kb * (D / 4);
#pragma unroll
    for (int c = 0; c < N; ++c) {
      if constexpr (NP == 1) {
        q[0][c] = as_op(*reinterpret_cast<const u32x4 *>(p + 8 * c));
      } else {
        float x[8];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const f32x4 v = load4(p + 8 * c + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[4 * g + e] = v[e];
        }
        bf16x8 y[3];
        to_pieces<3>(x, y);
#pragma unroll
        for (int i = 0; i < 3; ++i) q[i][c] = y[i];
      }
    }
  }

  const int codes = D / 2 << a.lpage;
  const int64_t block = (int64_t)codes + (D / 32 << a.lpage);  // bytes of a head's block
  auto load = [&](int j, Stage4<D, VALUES> &x) {
    x.ok = 0;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int key = j + 16 * i, at = key >> a.lpage;
      int page = at < a.width ? a.table[(int64_t)b * a.width + at] : -1;
      page = __builtin_amdgcn_readfirstlane(page);
      const bool ok = page >= 0 && page < a.pages;
      x.ok |= ok << i;
      const uint8_t *kp = a.cache + cache_block<D>(ok ? page : 0, 0, hk, a.Hkv, a.lpage);
      const int tok = key & ((1 << a.lpage) - 1);
      load_words<N>(kp + (tok + slot) * (D / 2) + kb * (D / 8), x.k[i]);
      x.ks[i] = kp[codes + (tok + slot) * (D / 32) + kb * (D / 4) / 32];
      if constexpr (VALUES) {
        const uint8_t *vp = kp + a.Hkv * block;
        load_words<N>(vp + tok * (D / 2) + lane * (D / 8), x.v[i]);
        x.vs[i] = *reinterpret_cast<const uint32_t *>(vp + codes + tok * (D / 32) + kb * (D / 8) +
                                                      slot * (D / 16) / 32 * 4);
      }
    }
  };

  // the row's grid, from the extrema that the first pass left
  RowConst rc{};
  float Mx = -INFINITY, Mn = INFINITY;
  if constexpr (PASS == PASS_GRID) {
    const float2 *e = reinterpret_cast<const float2 *>(a.ext) +
                      slot_of(a, hk, tile, share.first) + col;
#pragma unroll 4
    for (int i = kb; i < share.parts; i += 4) {
      const float2 x = e[16 * i];
      Mx = fmaxf(Mx, x.x);
      Mn = fminf(Mn, x.y);
    }
    Mx = fmaxf(Mx, __shfl_xor(Mx, 16));
    Mx = fmaxf(Mx, __shfl_xor(Mx, 32));
    Mn = fminf(Mn, __shfl_xor(Mn, 16));
    Mn = fminf(Mn, __shfl_xor(Mn, 32));
    Mx *= a.scale, Mn *= a.scale;
    rc = row_const(Mx, Mn, a.K, CALIB, a.tau, a.scale);
  }
  const float Kf = (float)a.K, edge = 2.f * Kf - 1.f, span = 1.f - rc.emh;
  const float c2 = a.scale * 1.44269504f;

  f32x4 o[VALUES ? NT : 1] = {};
  float m = -INFINITY, l = 0.f, low = INFINITY;  // (extrema: m and low)
  Stage4<D, VALUES> cur, nxt;
  int c = c0 + wave;
  if (c < c1) load(chunks.at(c), cur);
  for (; c < c1; c += NWAVE) {
    const int j = chunks.at(c);
    if (c + NWAVE < c1) load(chunks.at(c + NWAVE), nxt);
    // every row of the tile sees every key of the chunk
    const bool all = j + CHUNK - 1 <= lo && cur.ok == (1 << TILES) - 1 &&
                     ((int64_t)hi - j < a.window || j + CHUNK - 1 < a.sinks);
    auto sees = [&](int key, int i) {
      return key <= pos && ((int64_t)pos - key < a.window || key < a.sinks) && (cur.ok >> i & 1);
    };
    // groups that hold an infinity or NaN
    bool bad = false;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      bad |= cur.ks[i] == 255;
      if constexpr (VALUES) {
        const uint32_t y = ~cur.vs[i];
        bad |= ((y - 0x01010101u) & ~y & 0x80808080u) != 0;
      }
    }
    bad = __any(bad);
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
    // the scores of the keys that the lane weighs: key j + 16 i + 4 kb + own + e
    float S[TILES][NE];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      if constexpr (FEW)
        S[i][0] = own < 2 ? (own ? Q[i][1] : Q[i][0]) : own == 2 ? Q[i][2] : Q[i][3];
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i][e] = Q[i][e];
    }
    auto counts = [&](int i, int e) { return sees(j + 16 * i + 4 * kb + own + e, i); };
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
        top = across<FEW>(top, [](float x, float y) { return fmaxf(x, y); });
        // (moved, and the sums scaled, only when passed by 2^8, row by row: no row's bits
        // depend on another's)
        const bool up = (top - m) * c2 > 8.f;
        if (__any(up)) {
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
            if (j + 16 * i + 4 * kb + e > hi || !(cur.ok >> i & 1)) cur.clear(i, e);
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
            one[i / 2][i % 2 * 4 + e] = (__bf16)(sees(j + 16 * i + 4 * kb + e, i) ? 1.f : 0.f);
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
          uint32_t z[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int i = 2 * u + e / 4, k = e % 4;
            z[e] = pair_at(D == 128 ? y : D == 64 ? 2 * (k % 2) + y : k,
                           cur.v[i][D == 128 ? k : D == 64 ? k / 2 : 0], f[e]);
          }
          u32x4 even, odd;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            even[e] = __builtin_amdgcn_perm(z[2 * e + 1], z[2 * e], 0x05040100u);
            odd[e] = __builtin_amdgcn_perm(z[2 * e + 1], z[2 * e], 0x07060302u);
          }
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
    if (share.parts == 1) {
      const int rr = tile * 16 + row;
      if (rr < total) {
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        TI *y = slice_of<TI>(a.o, b, hk * G + rr % G) + rr / G * a.o.st + part * NT;
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

// The parts of one row, joined in order: D / 4 threads a part, the parts in 1024 / D
// groups whose sums are added in order of the groups.
template <typename TI, int D> __global__ __launch_bounds__(256) void join_kernel(CachedArgs a) {
  constexpr int W = D / 4, NG = 256 / W;
  __shared__ float f[256], red[8];  // (a.shares < 256)
  __shared__ f32x4 sums[NG][W];
  const int kvs = a.B * a.Hkv, s = blockIdx.x % kvs, b = s / a.Hkv, hk = s % a.Hkv;
  const int G = a.H / a.Hkv, r = blockIdx.x / kvs, tid = threadIdx.x, wave = tid >> 6;
  const Share share(a, r / 16, b, true);
  if (share.parts == 1) return;  // (written by its only part)
  const int64_t first = slot_of(a, hk, r / 16, share.first) + r % 16;
  float m = -INFINITY, l = 0.f;
  if (tid < share.parts) {
    const float2 st = reinterpret_cast<const float2 *>(a.stat)[first + 16 * tid];
    l = st.y;
    if (l != 0.f) m = st.x;  // (a part that saw a key)
  }
  float top = m;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
  if ((tid & 63) == 0) red[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float g = l == 0.f ? 0.f : __builtin_amdgcn_exp2f((m - top) * (a.scale * 1.44269504f));
  float sum = l * g;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
  f[tid] = g;
  if ((tid & 63) == 0) red[4 + wave] = sum;
  __syncthreads();
  const int at = tid % W, grp = tid / W;
  const f32x4 *p = reinterpret_cast<const f32x4 *>(a.part + first * D) + at;
  f32x4 x = {};
#pragma unroll 4
  for (int i = grp; i < share.parts; i += NG)
    x += p[(int64_t)i * 16 * W] * f[i];  // (a NaN stays one, however small its part's weight)
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

template <typename TI, int D, bool FEW, int CALIB>
void grid_passes(const CachedArgs &a, dim3 g, hipStream_t s) {
  const dim3 t(64 * NWAVE);
  timed_call("kia_cache4_extrema", s, [&] {
    hipLaunchKernelGGL((cached_kernel<TI, D, PASS_EXTREMA, CALIB, REC_LERP, FEW && CALIB != CAL_FWM>),
                       g, t, 0, s, a);
  });
  timed_call("kia_cache4_attn", s, [&] {
    if (a.recon == REC_LERP)
      hipLaunchKernelGGL((cached_kernel<TI, D, PASS_GRID, CALIB, REC_LERP, FEW>), g, t, 0, s, a);
    else
      hipLaunchKernelGGL((cached_kernel<TI, D, PASS_GRID, CALIB, REC_NEAREST, FEW>), g, t, 0, s, a);
  });
}

template <typename TI, int D, int CALIB> void grid_rows(const CachedArgs &a, dim3 g, hipStream_t s) {
  if (a.T * (a.H / a.Hkv) <= 4) grid_passes<TI, D, true, CALIB>(a, g, s);
  else grid_passes<TI, D, false, CALIB>(a, g, s);
}

template <typename TI, int D> void run(const CachedArgs &a, hipStream_t s) {
  const dim3 g((unsigned)(a.shares + a.B) * a.Hkv * a.tiles);
  if (a.recon == REC_SOFTMAX) {
    timed_call("kia_cache4_attn", s, [&] {
      hipLaunchKernelGGL((cached_kernel<TI, D, PASS_SOFTMAX, CAL_FWM, REC_SOFTMAX, false>), g,
                         dim3(64 * NWAVE), 0, s, a);
    });
  } else if (a.calib == CAL_MINMAX) {
    grid_rows<TI, D, CAL_MINMAX>(a, g, s);
  } else if (a.calib == CAL_FWM) {
    grid_rows<TI, D, CAL_FWM>(a, g, s);
  } else {
    grid_rows<TI, D, CAL_RESOLVED>(a, g, s);
  }
  if (a.shares > 1) {
    timed_call("kia_cache4_join", s, [&] {
      hipLaunchKernelGGL((join_kernel<TI, D>), dim3((unsigned)(a.B * a.Hkv) * (a.T * (a.H / a.Hkv))), dim3(256), 0,
                         s, a);
    });
  }
}

}  // namespace

template <> void launch_cached<KIA_HEAD>(const CachedArgs &a, int dtype, hipStream_t s) {
  if (dtype == KIA_F32) run<float, KIA_HEAD>(a, s);
  else run<uint16_t, KIA_HEAD>(a, s);
}

}  // namespace kia
