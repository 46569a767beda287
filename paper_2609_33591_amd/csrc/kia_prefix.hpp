// kia_prefix.hpp -- attention over the tokens that all sequences of a batch share: the part
// of each row's sums that those over what lies behind them (kia_cached.hip) complete, in
// workgroups of the same launch.
//
// The rows (sequence, token, head of the group) of a key head meet the same keys, so they
// are one product: 16 rows a tile as in kia_cached.hip, with its operands and orders, and RT
// tiles a wave, which takes the codes of 32 keys apart once for all of them. That work, some
// 100 vector operations, and a tile's weights, some 45, bound the kernel before the matrix unit
// does; the keys come out of the L2 after the first tile. Key heads go round the workgroups, so
// that an XCD's share of them are few and fit.
// 1024 rows a key head over 16 384 tokens, four heads of 128, softmax, bf16: 58 us, 600 TFLOP/s (one
// tile a wave: 80 us); 256 rows over 8192, LERP: 9 to 10 and 25 us (10 and 27). For a few row tiles it
// does not matter (six of fp32 heads of 64, two key heads: 4.7 and 8.7 us, 4.8 and 8.1).
#pragma once

#include "kia_cached.hpp"

namespace kia {

// The last key of the shared tokens that a row at `pos` sees.
__device__ __forceinline__ int last_of(const CachedArgs &a, int pos) { return min(pos, a.shared - 1); }

// LDS of a workgroup: its waves' statistics and, tile by tile, their rows.
typedef float WaveStats[NWAVE][16][2];

// The parts of what lies behind the shared tokens, of row tile `tile` of sequence b: the first
// one's number, and how many.
__device__ __forceinline__ int2 own_parts(const CachedArgs &a, unsigned tile, unsigned b) {
  return a.spread ? a.own[(int64_t)tile * a.B + b] : make_int2(b * a.parts, a.parts);
}

// A row's extrema (scaled) over the shared tokens and what lies behind them, from the first pass.
__device__ __forceinline__ void row_extrema(const CachedArgs &a, int hk, unsigned row, int kb, float &Mx, float &Mn) {
  const unsigned per = a.T * ((unsigned)a.H / (unsigned)a.Hkv), b = row / per, r = row % per;
  Mx = -INFINITY, Mn = INFINITY;
  auto among = [&](const float *ext, int64_t first, int parts) {
    const float2 *e = reinterpret_cast<const float2 *>(ext) + first;
    for (int i = kb; i < parts; i += 4) {
      const float2 y = e[16 * i];
      Mx = fmaxf(Mx, y.x);
      Mn = fminf(Mn, y.y);
    }
  };
  among(a.pre.ext, a.pre.slot(hk, row), a.pre.parts);
  const int2 own = own_parts(a, r / 16, b);
  among(a.ext, (((int64_t)hk * a.tiles + r / 16) * a.shares + own.x) * 16 + r % 16, own.y);
  Mx = fmaxf(Mx, __shfl_xor(Mx, 16)), Mx = fmaxf(Mx, __shfl_xor(Mx, 32));
  Mn = fminf(Mn, __shfl_xor(Mn, 16)), Mn = fminf(Mn, __shfl_xor(Mn, 32));
  Mx *= a.scale, Mn *= a.scale;
}

// Weights of a row's scores of 32 keys against its running maximum m. That is moved, and the
// sums scaled, only when passed by 2^8: where no lane sees that, no row does. m is in log2 units,
// rounded once where it is set: weights, rescaling and the joins all take that value, so that
// its rounding (2^-16 of a weight at a score of 350 nats) is the same everywhere and divides out.
// (Against m c2 rounded anew beside joins by the maximum itself, waves and parts were weighted
// apart by that much.)
template <int NT>
__device__ __forceinline__ void softmax_weights(const float (&S)[TILES][4], float (&w)[TILES][4], float &m, float &sum,
                                                f32x4 (&o)[NT], float c2) {
  float top = S[0][0];
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = fmaxf(top, S[i][e]);
  if (__any(fmaf(top, c2, -m) > 8.f)) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const bool up = fmaf(top, c2, -m) > 8.f;
    const float to = top * c2, f = up ? __builtin_amdgcn_exp2f(m - to) : 1.f;
    m = up ? to : m;
    sum *= f;
#pragma unroll
    for (int y = 0; y < NT; ++y) o[y] *= f;
  }
  const float mm = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) w[i][e] = __builtin_amdgcn_exp2f(fmaf(S[i][e], c2, -mm));
}

template <typename TI, int D, int PASS, int CALIB, int RECON, int RT>
__device__ __forceinline__ void prefix_part(const CachedArgs &a, WaveStats *red, float *rows) {
  constexpr int NP = Pieces<TI>::N, N = D / 32, NT = D / 16;
  constexpr bool VALUES = PASS != PASS_EXTREMA;
  const int tid = threadIdx.x, lane = tid & 63, kb = lane >> 4, slot = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned G = (unsigned)a.H / (unsigned)a.Hkv, per = a.T * G, total = a.B * per;  // rows of a sequence, of all
  const unsigned Hkv = a.Hkv, groups = ((unsigned)a.pre.tiles + RT - 1) / RT, id = blockIdx.x / Hkv;
  const int hk = blockIdx.x % Hkv, tile0 = id % groups * RT, part = id / groups;

  // this lane's row of each tile, and the last key that it sees (below 0: none)
  int last[RT], lo = INT_MAX, hi = -1;
  bf16x8 q[RT][NP][N];
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    const unsigned row = min((unsigned)(tile0 + x) * 16 + slot, total - 1), b = row / per, r = row % per;
    const int t = r / G;
    const int n = (int)min((int64_t)max(a.lengths[b], 0), (int64_t)a.width << a.lpage);
    last[x] = last_of(a, n - a.T + t);
    lo = min(lo, last[x]), hi = max(hi, last[x]);
    const TI *p = slice_of<TI>(a.q, b, hk * G + r % G) + t * a.q.st + kb * (D / 4);
#pragma unroll
    for (int c = 0; c < N; ++c) load_query<TI>(p + 8 * c, q[x], c);
  }
#pragma unroll
  for (int i = 1; i < 16; i *= 2) {
    lo = min(lo, __shfl_xor(lo, i));
    hi = max(hi, __shfl_xor(hi, i));
  }
  lo = __builtin_amdgcn_readfirstlane(lo), hi = __builtin_amdgcn_readfirstlane(hi);
  const int chunks = a.shared / CHUNK, seen = hi < 0 ? 0 : hi / CHUNK + 1;
  const int c0 = share_of(chunks, part, a.pre.parts), c1 = min(seen, share_of(chunks, part + 1, a.pre.parts));

  const int codes = D / 2 << a.lpage;
  const int64_t block = (int64_t)codes + (D / 32 << a.lpage), stride = 2 * a.Hkv * block;
  const uint8_t *head = a.cache + hk * block;
  // (the table's entries of a chunk are asked for a turn before its keys)
  int entry[TILES];
  auto ask = [&](int c) {
#pragma unroll
    for (int i = 0; i < TILES; ++i) entry[i] = entry_of(a.table, (min(c, c1 - 1) * CHUNK + 16 * i) >> a.lpage);
  };
  Offsets<D> where(lane);
  auto load = [&](int c, Stage4<D, VALUES> &x) {
    where.hold();
    x.ok = 0;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int key = c * CHUNK + 16 * i;
      const int page = entry[i];
      const bool ok = page >= 0 && page < a.pages;
      x.at[i] = key;
      x.ok |= ok << i;
      load_tile<D, VALUES>(head + (ok ? page : 0) * stride, a.Hkv * block, key & ((1 << a.lpage) - 1), codes, where, i, x);
    }
  };

  RowConst rc[RT] = {};
  float Mx[RT], Mn[RT];
  if constexpr (PASS == PASS_GRID) {
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      row_extrema(a, hk, min((unsigned)(tile0 + x) * 16 + slot, total - 1), kb, Mx[x], Mn[x]);
      rc[x] = row_const(Mx[x], Mn[x], a.K, CALIB, a.tau, a.scale);
    }
  }
  const float c2 = a.scale * 1.44269504f;

  f32x4 o[RT][VALUES ? NT : 1] = {};
  float m[RT], l[RT], low[RT];
#pragma unroll
  for (int x = 0; x < RT; ++x) m[x] = -INFINITY, l[x] = 0.f, low[x] = INFINITY;
  Stage4<D, VALUES> cur, nxt;
  int c = c0 + wave;
  if (c < c1) {
    ask(c);
    load(c, cur);
    ask(c + NWAVE);
  }
  auto step = [&](Stage4<D, VALUES> &cur, Stage4<D, VALUES> &nxt) __attribute__((always_inline)) {
    // (the last chunk again at the end: behind a branch, the wait for this chunk would be one for
    // what the branch may have asked for too)
    load(min(c + NWAVE, c1 - 1), nxt);
    ask(c + 2 * NWAVE);
    const int j = cur.at[0];
    const bool all = j + CHUNK - 1 <= lo && cur.ok == (1 << TILES) - 1;
    auto sees = [&](int x, int i, int e) { return j + 16 * i + 4 * kb + e <= last[x] && (cur.ok >> i & 1); };
    const bool bad = __any(holds_nan<D, VALUES>(cur));
    // scores of all tiles from the keys' operands
    float S[RT][TILES][4];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const float f = scale_of(cur.ks[i]);
      u32x4 w[N];
#pragma unroll
      for (int y = 0; y < N; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[y][e] = pair_at(e, cur.k[i][y], f);
#pragma unroll
      for (int x = 0; x < RT; ++x) {
        f32x4 acc = {};
#pragma unroll
        for (int p = NP - 1; p >= 0; --p)
#pragma unroll
          for (int y = 0; y < N; ++y) acc = mma16(as_op(w[y]), q[x][p][y], acc);
#pragma unroll
        for (int e = 0; e < 4; ++e) S[x][i][e] = acc[e];
      }
    }
    if (__builtin_expect(bad, 0)) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        uint64_t nan = __ballot(cur.ks[i] == 255);
        nan |= nan >> 32;
        nan |= nan >> 16;
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[x][i][e] = nan >> (4 * kb + e) & 1 ? NAN : S[x][i][e];
      }
    }
    if (!all) {
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[x][i][e] = sees(x, i, e) ? S[x][i][e] : -INFINITY;
    }
    if constexpr (PASS == PASS_EXTREMA) {
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            m[x] = fmaxf(m[x], S[x][i][e]);
            if constexpr (CALIB != CAL_FWM) low[x] = all || sees(x, i, e) ? fminf(low[x], S[x][i][e]) : low[x];
          }
    } else {
      // weights, as operands of the product with the values
      bf16x8 p[RT][NP];
#pragma unroll
      for (int x = 0; x < RT; ++x) {
        float w[TILES][4];
        if constexpr (PASS == PASS_SOFTMAX) {
          softmax_weights<NT>(S[x], w, m[x], l[x], o[x], c2);
        } else {
          grid_weights<CALIB, RECON, 4>(S[x], w, rc[x], Mx[x], Mn[x], a);
          if (!all) {
#pragma unroll
            for (int i = 0; i < TILES; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) w[i][e] = sees(x, i, e) ? w[i][e] : 0.f;
          }
        }
        float y[8];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          l[x] += (w[i][0] + w[i][1]) + (w[i][2] + w[i][3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[4 * i + e] = w[i][e];
        }
        to_pieces<NP>(y, p[x]);
      }
      if (!all) {
        // values of tokens that no row sees (on no page, behind the last row) as zeros
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (j + 16 * i + 4 * kb + e > hi || !(cur.ok >> i & 1)) cur.clear(i, e);
      }
      if (__builtin_expect(bad, 0)) {
        // groups of NaN: their values as zeros here, and NaN for the rows that see them
        bf16x8 is;
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool nan = (cur.vs[i] >> (8 * e) & 255) == 255;
            if (nan) cur.clear(i, e);
            is[4 * i + e] = (__bf16)(nan ? 1.f : 0.f);
          }
#pragma unroll
        for (int x = 0; x < RT; ++x) {
          bf16x8 one;
#pragma unroll
          for (int e = 0; e < 8; ++e) one[e] = (__bf16)(sees(x, e / 4, e % 4) ? 1.f : 0.f);
          f32x4 k = {};
          k = mma16(is, one, k);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int y = 0; y < NT; ++y) o[x][y][e] = k[e] > 0.f ? NAN : o[x][y][e];
        }
      }
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = scale_of(cur.vs[e / 4] >> (8 * (e % 4)) & 255);
#pragma unroll
      for (int y = 0; y < NT / 2; ++y) {
        u32x4 even, odd;
        value_ops<D>(cur, f, 0, y, even, odd);
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
          for (int i = NP - 1; i >= 0; --i) {
            o[x][2 * y] = mma16(as_op(even), p[x][i], o[x][2 * y]);
            o[x][2 * y + 1] = mma16(as_op(odd), p[x][i], o[x][2 * y + 1]);
          }
      }
    }
  };
  for (; c < c1; c += NWAVE) {
    step(cur, nxt);
    if constexpr (PASS == PASS_GRID) {
      cur = nxt;
    } else {
      // (two chunks a turn, for no copies; the registers do not reach for the interval weights)
      c += NWAVE;
      if (c >= c1) break;
      step(nxt, cur);
    }
  }

  // the waves' parts, joined in their order
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    if constexpr (PASS == PASS_EXTREMA) {
      m[x] = fmaxf(m[x], __shfl_xor(m[x], 16)), m[x] = fmaxf(m[x], __shfl_xor(m[x], 32));
      low[x] = fminf(low[x], __shfl_xor(low[x], 16)), low[x] = fminf(low[x], __shfl_xor(low[x], 32));
      if (kb == 0) red[x][wave][slot][0] = m[x], red[x][wave][slot][1] = low[x];
    } else {
      l[x] += __shfl_xor(l[x], 16);
      l[x] += __shfl_xor(l[x], 32);
      if (kb == 0) red[x][wave][slot][0] = m[x], red[x][wave][slot][1] = l[x];
    }
  }
  if constexpr (PASS == PASS_EXTREMA) {
    __syncthreads();
    if (tid < RT * 16) {
      const int x = tid / 16;
      const unsigned row = (tile0 + x) * 16 + slot;
      if (row < total) {
        float mx = red[x][0][slot][0], mn = red[x][0][slot][1];
#pragma unroll
        for (int i = 1; i < NWAVE; ++i) {
          mx = fmaxf(mx, red[x][i][slot][0]);
          mn = fminf(mn, red[x][i][slot][1]);
        }
        float *e = a.pre.ext + (a.pre.slot(hk, row) + 16 * (int64_t)part) * 2;
        e[0] = mx, e[1] = mn;
      }
    }
  } else {
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      // channel (4 kb + e) NT + y of row `slot`
      float *mine = rows + (wave * 16 + slot) * (D + 4);
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int y = 0; y < NT; ++y) mine[(4 * kb + e) * NT + y] = o[x][y][e];
      __syncthreads();
      const int row16 = tid / 16, at = tid % 16;
      const unsigned row = (tile0 + x) * 16 + row16;
      float top = 0.f, sum = 0.f, z[NT] = {};
      if constexpr (PASS == PASS_SOFTMAX) {
        top = red[x][0][row16][0];
#pragma unroll
        for (int i = 1; i < NWAVE; ++i) top = fmaxf(top, red[x][i][row16][0]);
        if (top == -INFINITY) top = 0.f;
      }
#pragma unroll
      for (int i = 0; i < NWAVE; ++i) {
        const float f = PASS == PASS_SOFTMAX ? __builtin_amdgcn_exp2f(red[x][i][row16][0] - top) : 1.f;
        sum = fmaf(red[x][i][row16][1], f, sum);
#pragma unroll
        for (int e = 0; e < NT; ++e) z[e] = fmaf(rows[(i * 16 + row16) * (D + 4) + at * NT + e], f, z[e]);
      }
      if (row < total) {
        const int64_t out = a.pre.slot(hk, row) + 16 * (int64_t)part;
        float *y = a.pre.part + out * D + at * NT;
#pragma unroll
        for (int e = 0; e < NT; ++e) y[e] = z[e];
        if (at == 0) a.pre.stat[out * 2] = top, a.pre.stat[out * 2 + 1] = sum;  // (log2 units)
      }
    }
  }
}

}  // namespace kia
