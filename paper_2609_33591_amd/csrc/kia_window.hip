// kia_window.hip -- softmax attention with a sliding window and visible first
// tokens on gfx950, forward and backward, for one head dimension (KIA_HEAD).
//
// Query i sees key j iff j <= i and (i - j < window or j < sinks). With
// s = q.k / sqrt(d):
//   O_i = sum_j p_ij v_j, p_ij = e^{s_ij - lse_i}, lse_i = ln sum_j e^{s_ij};
//   D_i = dO_i . O_i, dS_ij = p_ij (dO_i . v_j - D_i);
//   dQ = dS K / sqrt(d), dK = dS^T Q / sqrt(d), dV = P^T dO.
// Query heads h share the key head h / (H / Hkv).
//
// Every kernel has the same shape: a wave keeps 32 rows of one side in registers
// (queries; for dK and dV keys) as the B operand, rows of the other side stream
// through LDS, and a 32x32 block of scores is formed with the streamed rows along
// the registers, so that its weights are the B operand of the next product as they
// stand (krel()) and the streamed rows are its A operand, by columns. Row sums and
// maxima of a query are then one lane's (and its partner's, 32 lanes on).
//
// bf16 runs on v_mfma_f32_32x32x16_bf16; the weights p and dS, the products'
// computed operands, are rounded to bf16 (2^-8 of each), all sums and statistics are
// fp32. Over random values such a rounding adds as much again as the output's own: errors
// of sqrt(2) times that one in the 2-norm (1.3 to 1.45 measured), and the goal is 1.5 times.
// With p and dS in two pieces it is 1.0 times, and the training step of win_fwd_kernel's
// figures takes 16% longer, the prompt there 19%. fp32 runs on v_mfma_f32_32x32x2_f32
// throughout: no operand is rounded, sums are fp32.
//
// A key that a query does not see has no influence on it, whatever it holds: its score
// is replaced before it is used, and in tiles where some pair is masked, rows that hold
// infinities or NaNs go to LDS with zeros in their place, and what they do to the rows
// that see them is done apart (add_bad, bad_rows): a branch that few calls ever take,
// kept small because its registers count for the loop it stands in. Rows of no weight
// (past the end, or of no finite score) are masked and set to 0, never multiplied by it.

#include "kia_around.hpp"
#include "kia_host.hpp"

namespace kia {
namespace {

constexpr float LOG2E_F = 1.44269504f;

template <typename TI> constexpr bool is_f32 = sizeof(TI) == 4;

// ---- rows in LDS ---------------------------------------------------------------
// A [ROWS, D] block of rows of any stride, rows at or past `end` as zeros. The row
// stride in LDS is D plus 16 bytes in fp32, whose columns are read one by one, without
// bank conflicts. In bf16, where 16-byte reads of rows and transposing reads meet, it is D
// plus 32 bytes, by measurement: dK and dV at d = 128 take 152 us, with 16 / 48 / 64 bytes
// 155 / 149 / 286, and the forward 4 to 6% more with 16 or 48. Conflicts are still 12 to 14%
// of all cycles there.
template <typename TI, int D, int ROWS, int NT> struct Rows {
  static constexpr int V = 16 / sizeof(TI), RS = D + (is_f32<TI> ? 4 : 16), SIZE = ROWS * RS;
  static constexpr int PER = ROWS * D / V, PF = (PER + NT - 1) / NT, RPP = NT * V / D;
  static_assert(PER % NT == 0 || PF == 1, "whole passes");
  u32x4 x[PF];
  __device__ __forceinline__ void fetch(const TI *slice, int64_t st, int r0, int end, int tid) {
    const int rows = min(ROWS, end - r0);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<TI *>(slice) + (rows > 0 ? r0 : 0) * st, (short)0,
        rows > 0 ? ((rows - 1) * (int)st + D) * (int)sizeof(TI) : 0, 0x00020000);
    const uint32_t row = tid / (D / V) * (uint32_t)st;
    const uint32_t off = PER % NT == 0 || tid < PER
                             ? (row + tid % (D / V) * V) * (uint32_t)sizeof(TI)
                             : 0x80000000u;
    const uint32_t step = RPP * (uint32_t)st * (uint32_t)sizeof(TI);
#pragma unroll
    for (int e = 0; e < PF; ++e)
      x[e] = __builtin_bit_cast(u32x4,
                                __builtin_amdgcn_raw_buffer_load_b128(rs, off + e * step, 0, 0));
  }
  __device__ __forceinline__ void stash(TI *dst, int tid) const {
    if (PER % NT != 0 && tid >= PER) return;
#pragma unroll
    for (int e = 0; e < PF; ++e) {
      const int i = tid + NT * e;
      *reinterpret_cast<u32x4 *>(dst + i / (D / V) * RS + i % (D / V) * V) = x[e];
    }
  }
  // infinities and NaNs as zeros
  __device__ __forceinline__ void clean() {
#pragma unroll
    for (int e = 0; e < PF; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = x[e][i];
        if constexpr (is_f32<TI>) {
          x[e][i] = (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
        } else {
          x[e][i] = ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u) |
                    ((w & 0x00007f80u) == 0x00007f80u ? 0u : w & 0x0000ffffu);
        }
      }
  }
  // whether any of the thread's values is infinite or NaN
  __device__ __forceinline__ bool bad() const {
    bool b = false;
#pragma unroll
    for (int e = 0; e < PF; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (is_f32<TI>) {
          b |= (x[e][i] & 0x7f800000u) == 0x7f800000u;
        } else {
          b |= (x[e][i] & 0x7f800000u) == 0x7f800000u;
          b |= (x[e][i] & 0x00007f80u) == 0x00007f80u;
        }
      }
    return b;
  }
};

// ---- 32 rows in registers -------------------------------------------------------
// Lane l holds of row l % 32 what its half of the matrix instructions takes: bf16,
// channels 16 s + 8 (l / 32) + e; fp32, channels 8 c + 4 (l / 32) + e.
template <typename TI, int D> struct RowReg {
  bf16x8 v[D / 16];
  __device__ __forceinline__ void load(const uint16_t *row, int half, bool ok) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      u32x4 x = *reinterpret_cast<const u32x4 *>(row + 16 * s + 8 * half);
      if (!ok) x = u32x4{0, 0, 0, 0};
      v[s] = as_op(x);
    }
  }
  __device__ __forceinline__ float dot(const RowReg &o) const {
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf((float)v[s][e], (float)o.v[s][e], sum);
    return sum;
  }
};
template <int D> struct RowReg<float, D> {
  float v[D / 2];
  __device__ __forceinline__ void load(const float *row, int half, bool ok) {
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(row + 8 * c + 4 * half);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * c + e] = ok ? x[e] : 0.f;
    }
  }
  __device__ __forceinline__ float dot(const RowReg &o) const {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < D / 2; ++e) sum = fmaf(v[e], o.v[e], sum);
    return sum;
  }
};

// Products of 32 streamed rows (at `t`, row stride RS) with the 32 rows of b:
// register r of lane l is the pair (streamed row krel(r, l / 32), row l % 32 of b).
template <int D, int RS>
__device__ __forceinline__ f32x16 dots(const uint16_t *t, const RowReg<uint16_t, D> &b, int lane) {
  f32x16 c = {};
  const uint16_t *p = t + (lane & 31) * RS + 8 * (lane >> 5);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) c = mfma16(row_op(p + 16 * s), b.v[s], c);
  return c;
}
template <int D, int RS>
__device__ __forceinline__ f32x16 dots(const float *t, const RowReg<float, D> &b, int lane) {
  f32x16 c = {};
  const float *p = t + (lane & 31) * RS + 4 * (lane >> 5);
#pragma unroll
  for (int s = 0; s < D / 8; ++s) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + 8 * s);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = mfma32(x[e], b.v[4 * s + e], c);
  }
  return c;
}

// The same with b's rows in LDS too.
template <int D, int RS>
__device__ __forceinline__ f32x16 dots(const uint16_t *t, const uint16_t *b, int lane) {
  f32x16 c = {};
  const int at = (lane & 31) * RS + 8 * (lane >> 5);
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    c = mfma16(row_op(t + at + 16 * s), row_op(b + at + 16 * s), c);
  return c;
}

template <int D, int RS>
__device__ __forceinline__ f32x16 dots(const float *t, const float *b, int lane) {
  f32x16 c = {};
  const int at = (lane & 31) * RS + 4 * (lane >> 5);
#pragma unroll
  for (int s = 0; s < D / 8; ++s) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(t + at + 8 * s);
    const f32x4 y = *reinterpret_cast<const f32x4 *>(b + at + 8 * s);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = mfma32(x[e], y[e], c);
  }
  return c;
}

// acc[c][channel][row of b's side] += sum over the 32 streamed rows of their
// channels 32 c .. times the weights w (register r: streamed row krel(r, half)).
// REST: bf16 weights in two pieces, what the rounding leaves multiplied too.
template <int D, int RS, bool REST = false, int NC>
__device__ __forceinline__ void mul_rows(f32x16 (&acc)[NC], const uint16_t *t, const float (&w)[16],
                                         int lane) {
  const uint16_t *p = t + tr_base<D, RS>(lane);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    u32x4 x, y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = w[8 * s + 2 * e], b = w[8 * s + 2 * e + 1];
      x[e] = cvt_bf16x2(a, b);
      if constexpr (REST)
        y[e] = cvt_bf16x2(a - __uint_as_float(x[e] << 16), b - __uint_as_float(x[e] & 0xffff0000u));
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bf16x8 r = tr_op<RS>(p + 16 * s * RS + 32 * c);
      if constexpr (REST) acc[c] = mfma16(r, as_op(y), acc[c]);
      acc[c] = mfma16(r, as_op(x), acc[c]);
    }
  }
}
template <int D, int RS, bool REST = false, int NC>
__device__ __forceinline__ void mul_rows(f32x16 (&acc)[NC], const float *t, const float (&w)[16],
                                         int lane) {
  const float *p = t + 4 * (lane >> 5) * RS + (lane & 31) % D;
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] = mfma32(p[krel0(r) * RS + 32 * c], w[r], acc[c]);
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }
// The infinities and NaNs of the 32 streamed rows at `rows` (stride st, only the first
// `count`), which mul_rows took as zeros: added to the lane's row where see(i) says
// that streamed row i counts for it, times f (0: as NaN).
template <int D, int NC, typename TI, class See>
__device__ __forceinline__ void add_bad(f32x16 (&acc)[NC], const TI *rows, int64_t st, int count,
                                        int lane, float f, See see) {
#pragma unroll 1
  for (int i = 0; i < min(32, count); ++i) {
    const bool ok = see(i);
    const TI *row = rows + i * st + 4 * (lane >> 5);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int g = 0; g < (D < 32 ? D / 8 : 4); ++g) {
        const f32x4 x = load4(row + 32 * c + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[c][4 * g + e] += ok && !finite(x[e]) ? x[e] * f : 0.f;
      }
  }
}
// Which of those rows hold any (bit i: row i).
template <int D, typename TI>
__device__ __forceinline__ uint32_t bad_rows(const TI *rows, int64_t st, int count, int lane) {
  bool bad = false;
  if ((lane & 31) < count) {
    const TI *row = rows + (lane & 31) * st + (lane >> 5) * (D / 2);
#pragma unroll 1
    for (int c = 0; c < D / 2; ++c) bad |= !finite(load1(row + c));
  }
  const uint64_t x = __ballot(bad);
  return (uint32_t)x | (uint32_t)(x >> 32);
}

// One lane's row from accumulators (register r of block c: channel
// 32 c + 8 (r / 4) + 4 half + r % 4), times f.
template <int D, int NC>
__device__ __forceinline__ void store_row(float *row, const f32x16 (&acc)[NC], int half, float f) {
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int g = 0; g < (D < 32 ? D / 8 : 4); ++g) {
      const f32x4 x = {acc[c][4 * g] * f, acc[c][4 * g + 1] * f, acc[c][4 * g + 2] * f,
                       acc[c][4 * g + 3] * f};
      *reinterpret_cast<f32x4 *>(row + 32 * c + 8 * g + 4 * half) = x;
    }
}
template <int D, int NC>
__device__ __forceinline__ void store_row(uint16_t *row, const f32x16 (&acc)[NC], int half,
                                          float f) {
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int g = 0; g < (D < 32 ? D / 8 : 4); ++g) {
      const u32x2 x = {cvt_bf16x2(acc[c][4 * g] * f, acc[c][4 * g + 1] * f),
                       cvt_bf16x2(acc[c][4 * g + 2] * f, acc[c][4 * g + 3] * f)};
      *reinterpret_cast<u32x2 *>(row + 32 * c + 8 * g + 4 * half) = x;
    }
}

template <int NC> __device__ __forceinline__ void clear(f32x16 (&acc)[NC]) {
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[c][r] = 0.f;
}

__device__ __forceinline__ int length_of(const WinArgs &a, int b) {
  return a.lengths ? max(0, min(a.lengths[b], a.T)) : a.T;
}
__device__ __forceinline__ bool sees(const WinArgs &a, int i, int j) {
  return j <= i && (i - j < a.window || j < a.sinks);
}
// whether some pair, every pair, of queries i .. i + ni - 1 and keys j .. j + nj - 1 counts
__device__ __forceinline__ bool sees_some(const WinArgs &a, int i, int ni, int j, int nj) {
  return j <= i + ni - 1 && (i - (j + nj - 1) < a.window || j < a.sinks);
}
__device__ __forceinline__ bool sees_all(const WinArgs &a, int i, int ni, int j, int nj) {
  return j + nj - 1 <= i && (i + ni - 1 - j < a.window || j + nj - 1 < a.sinks);
}

// The key tiles of KT keys that queries i0 .. i1 - 1 see: the first tokens', then the
// window's.
template <int KT> struct KeyTiles {
  int sink, low, count;
  __device__ __forceinline__ KeyTiles(const WinArgs &a, int i0, int i1) {
    const int lo = max(0, i0 - a.window + 1);
    low = lo / KT;
    sink = min((min(a.sinks, lo) + KT - 1) / KT, low);
    count = sink + (i1 - 1) / KT + 1 - low;
  }
  __device__ __forceinline__ int at(int n) const { return (n < sink ? n : low + n - sink) * KT; }
};

// Launch shapes of the forward and dQ: a workgroup's four waves are RG groups of 32
// queries times KP parts of each step's 32 KP keys. Large grids take 4 x 1: every staged
// tile serves 128 queries, and registers that leave room for a third wave a SIMD in bf16
// at d = 128 (168; with 64 keys a step 256). Grids too small to fill the chip give up
// row groups for key parts, whose sums are joined in order through LDS.
template <typename TI, int D, int RG> struct Shape {
  static constexpr int KP = 4 / RG, KT = 32 * KP;
  using R = Rows<TI, D, KT, 256>;
  static constexpr int NC = D >= 32 ? D / 32 : 1;
  static constexpr int BUF = 2 * R::SIZE * (int)sizeof(TI);  // keys and values of a step
  static constexpr int NBUF = 2 * BUF <= 140 * 1024 ? 2 : 1;
  static constexpr int JOIN = KP > 1 ? RG * (KP - 1) * 64 * (NC * 16 + 2) * 4 : 0;
  static constexpr int SMEM = (NBUF * BUF > JOIN ? NBUF * BUF : JOIN) + 64;
  static constexpr int WGS = 160 * 1024 / (SMEM + 64);  // that fit a CU's LDS
  static constexpr int FWD = RG < 4 ? 2 : is_f32<TI> ? (D == 128 ? 2 : 3) : D == 128 ? 3 : 4;
  // (fp32, d = 128: two waves a SIMD spill 45 registers, 595 us against 559 with one)
  static constexpr int DQ = is_f32<TI> && D == 128                              ? 1
                            : RG < 4 || D == 128 || (is_f32<TI> && D == 64) ? 2
                                                                            : 3;
  static constexpr int FWD_OCC = FWD < WGS ? FWD : WGS;
  static constexpr int DQ_OCC = DQ < WGS ? DQ : WGS;
};

// Key parts 1 .. hand their sums (and x, y of each lane) to part 0, through LDS.
template <int RG, int KP, int NC, class Take>
__device__ __forceinline__ void join_parts(char *smem, const f32x16 (&acc)[NC], float x, float y,
                                           int rg, int kp, int lane, Take take) {
  constexpr int W = NC * 16 + 2;
  __syncthreads();
  float *mine = reinterpret_cast<float *>(smem) + lane;
  if (kp > 0) {
    float *p = mine + (rg * (KP - 1) + kp - 1) * W * 64;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) p[(16 * c + r) * 64] = acc[c][r];
    p[(W - 2) * 64] = x;
    p[(W - 1) * 64] = y;
  }
  __syncthreads();
  if (kp > 0) return;
#pragma unroll
  for (int k = 1; k < KP; ++k) {
    const float *p = mine + (rg * (KP - 1) + k - 1) * W * 64;
    take(p[(W - 2) * 64], p[(W - 1) * 64], [&](int c, int r) { return p[(16 * c + r) * 64]; });
  }
}

// One workgroup: RG groups of 32 queries of one head, over the key tiles that any of
// them sees. Keys and values of the next tile are fetched into registers while a tile
// is worked on, and stored to the other of two buffers: one barrier a tile.
// The running maximum of a row moves (and its sums are scaled) only when a score
// passes it by 2^8: sums of weights up to 2^8 lose nothing in fp32.
// bf16, d = 128, 4 x 16 heads over 4, T = 2048, window 512: 66 us, 460 TFLOP/s; one prompt of
// 8192, 16 heads, window 1024: 106 us, 620 TFLOP/s (of a large matrix product's 1200), whose
// 1024 workgroups fill the 768 places 1.3 times: four such prompts together reach 700.
template <typename TI, int D, int RG>
__global__ __launch_bounds__(256, (Shape<TI, D, RG>::FWD_OCC)) void win_fwd_kernel(WinArgs a) {
  using C = Shape<TI, D, RG>;
  using R = typename C::R;
  constexpr int KP = C::KP, KT = C::KT, NBUF = C::NBUF, NC = C::NC, RS = R::RS;
  __shared__ __attribute__((aligned(16))) char smem[C::SMEM];
  __shared__ int flag[2][4];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rg = wave % RG, kp = wave / RG;
  const int G = a.H / a.Hkv, kvs = a.B * a.Hkv;
  const int s = blockIdx.x % kvs, b = s / a.Hkv, hk = s % a.Hkv;
  const int h = hk * G + (int)(blockIdx.x / kvs) % G;
  const int nqb = (a.T + 32 * RG - 1) / (32 * RG);
  const int i0 = (nqb - 1 - (int)(blockIdx.x / (kvs * G))) * 32 * RG;
  const int n = length_of(a, b);
  const int iw = i0 + 32 * rg, row = iw + l32;
  f32x16 acc[NC];
  clear(acc);
  float m = -INFINITY, l = 0.f;
  const float c2 = a.scale * LOG2E_F;
  if (i0 < n) {
    RowReg<TI, D> q;
    q.load(slice_of<TI>(a.q, b, h) + min(row, n - 1) * a.q.st, half, row < n);
    const KeyTiles<KT> tiles(a, i0, min(i0 + 32 * RG, n));
    const TI *ks = slice_of<TI>(a.k, b, hk), *vs = slice_of<TI>(a.v, b, hk);
    R fk, fv;
    auto buf = [&](int p) {
      return reinterpret_cast<TI *>(smem) + (NBUF == 2 ? p & 1 : 0) * 2 * R::SIZE;
    };
    auto fetch = [&](int p) {
      fk.fetch(ks, a.k.st, tiles.at(p), n, tid);
      fv.fetch(vs, a.v.st, tiles.at(p), n, tid);
    };
    auto stage = [&](int p) {
      TI *kb = buf(p);
      if (NBUF == 1 && p > 0) lds_barrier();
      const bool part = !sees_all(a, i0, 32 * RG, tiles.at(p), KT);
      if (part) {
        const bool bad = __any(fv.bad());
        if (__builtin_expect(bad, 0)) fv.clean();
        if (lane == 0) flag[p & 1][wave] = bad;
      }
      fk.stash(kb, tid);
      fv.stash(kb + R::SIZE, tid);
      if (p + 1 < tiles.count) fetch(p + 1);
      lds_barrier();
      return part && any_flag<4>(flag[p & 1]);
    };
    auto compute = [&](int p, bool bad) {
      const int j = tiles.at(p) + 32 * kp;
      const TI *kb = buf(p) + 32 * kp * RS, *vb = kb + R::SIZE;
      if (iw >= n || !sees_some(a, iw, 32, j, 32)) return;
      f32x16 S = dots<D, RS>(kb, q, lane);
      if (!sees_all(a, iw, 32, j, 32)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = sees(a, row, j + krel(r, half)) ? S[r] : -INFINITY;
      }
      float top = S[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, S[r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      // (row by row: no row's bits depend on another's)
      const bool up = (top - m) * c2 > 8.f;
      if (__any(up)) {
        const float f = up ? __builtin_amdgcn_exp2f((m - top) * c2) : 1.f;
        m = up ? top : m;
        l *= f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[c][r] *= f;
      }
      const float mm = m == -INFINITY ? 0.f : m;
      float w[16], sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        // (fp32: the difference first, so that the error is its own and not the score's)
        if constexpr (is_f32<TI>) w[r] = __builtin_amdgcn_exp2f((S[r] - mm) * c2);
        else w[r] = __builtin_amdgcn_exp2f(fmaf(S[r], c2, -mm * c2));
        sum += w[r];
      }
      l += sum;
      mul_rows<D, RS>(acc, vb, w, lane);
      if (__builtin_expect(bad, 0))
        add_bad<D>(acc, vs + j * a.v.st, a.v.st, n - j, lane, 1.f,
                   [&](int i) { return sees(a, row, j + i); });
    };
    fetch(0);
    for (int p = 0; p < tiles.count; ++p) {
      const bool bad = stage(p);
      compute(p, bad);
    }
  }
  if constexpr (KP > 1) {
    join_parts<RG, KP>(smem, acc, m, l, rg, kp, lane, [&](float pm, float pl, auto part) {
      const float to = fmaxf(m, pm);
      const float f = m == to ? 1.f : __builtin_amdgcn_exp2f((m - to) * c2);
      const float g = pm == to ? 1.f : __builtin_amdgcn_exp2f((pm - to) * c2);
      m = to;
      l = l * f + pl * g;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = acc[c][r] * f + part(c, r) * g;
    });
    if (kp > 0) return;
  }
  if (row >= a.T) return;
  l += __shfl_xor(l, 32);
  const bool none = l == 0.f || row >= n;
  // (not by a factor of 0: what such a row met on its way may be infinite or NaN)
  if (none) clear(acc);
  store_row<D, NC>(slice_of<TI>(a.o, b, h) + row * a.o.st, acc, half, none ? 0.f : 1.f / l);
  if (half == 0)
    a.lse[((int64_t)b * a.H + h) * a.T + row] = none ? -INFINITY : fmaf(m, a.scale, logf(l));
}

// dQ, and D for the key gradients. The same walk as the forward's, with the scores
// formed again and p from lse. In bf16 the D at hand, dO . O of the rounded output, is
// off by a rounding of every term. The weights of a row add up to the D that they should
// have been taken with less that one: the key gradients get the D so corrected, and
// query blocks whose rows see few keys, where the error would pass all others, walk
// their keys once before for that sum alone. (2-norm errors of dQ and dK against 64 bits at
// d = 128: window 2 4.5e-3 -> 2.4e-3, window 512 2.6e-3 -> 2.4e-3; the output's rounding
// alone is 1.65e-3.) dQ of longer rows takes D as it is: with scores of a standard deviation
// of 1 its error is lost in the others; where few keys take such a row, dS is small beside
// D's error, and dQ is off by more (deviations of 2 / 4 / 9 / 25: at most 1.8 / 2.4 / 3.8 / 4.8
// times the output's own rounding). Two walks for every row would hold that at 1.5, with 1.6
// times the time of dQ.
// In small heads a score has a large share of each key (q / sqrt(d) of it on average), and
// the roundings of a row's dS, which add up to 0 without them, carry that share into dQ:
// up to 32 channels dS goes in two bf16 pieces (window 217, 100 first tokens, T = 4531: d =
// 16 2.51e-3 -> 1.76e-3 for 111 -> 127 us with 128 heads, d = 32 2.42e-3 -> 1.71e-3 for 117
// -> 134; d = 64 has 2.37e-3 and would pay 163 -> 191).
// The training step above: 89 us, 510 TFLOP/s.
template <typename TI, int D, int RG>
__global__ __launch_bounds__(256, (Shape<TI, D, RG>::DQ_OCC)) void win_dq_kernel(WinArgs a) {
  using C = Shape<TI, D, RG>;
  using R = typename C::R;
  constexpr int KP = C::KP, KT = C::KT, NBUF = C::NBUF, NC = C::NC, RS = R::RS;
  constexpr bool FIX = !is_f32<TI>, REST = FIX && D <= 32;
  __shared__ __attribute__((aligned(16))) char smem[C::SMEM];
  __shared__ float offs[4][64];
  __shared__ int flag[2][4];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rg = wave % RG, kp = wave / RG;
  const int G = a.H / a.Hkv, kvs = a.B * a.Hkv;
  const int s = blockIdx.x % kvs, b = s / a.Hkv, hk = s % a.Hkv;
  const int h = hk * G + (int)(blockIdx.x / kvs) % G;
  const int nqb = (a.T + 32 * RG - 1) / (32 * RG);
  const int i0 = (nqb - 1 - (int)(blockIdx.x / (kvs * G))) * 32 * RG;
  const int n = length_of(a, b);
  const int iw = i0 + 32 * rg, row = iw + l32;
  const int64_t srow = ((int64_t)b * a.H + h) * a.T + row;
  f32x16 acc[NC];
  clear(acc);
  float off = 0.f, delta = 0.f;  // off: sum of the row's weights
  float lse = INFINITY;          // (of a row of nothing too: no weight anywhere)
  if (i0 < n) {
    RowReg<TI, D> q, g;
    const int at = min(row, n - 1);
    q.load(slice_of<TI>(a.q, b, h) + at * a.q.st, half, row < n);
    g.load(slice_of<TI>(a.dO, b, h) + at * a.dO.st, half, row < n);
    {
      RowReg<TI, D> o;
      o.load(slice_of<TI>(a.o, b, h) + at * a.o.st, half, row < n);
      delta = g.dot(o);
      delta += __shfl_xor(delta, 32);
    }
    if (row < n) lse = a.lse[srow];
    if (lse == -INFINITY) lse = INFINITY;
    const float c2 = a.scale * LOG2E_F, lse2 = lse * LOG2E_F;
    const KeyTiles<KT> tiles(a, i0, min(i0 + 32 * RG, n));
    const TI *ks = slice_of<TI>(a.k, b, hk), *vs = slice_of<TI>(a.v, b, hk);
    R fk, fv;
    auto buf = [&](int p) {
      return reinterpret_cast<TI *>(smem) + (NBUF == 2 ? p & 1 : 0) * 2 * R::SIZE;
    };
    auto fetch = [&](int p) {
      fk.fetch(ks, a.k.st, tiles.at(p), n, tid);
      fv.fetch(vs, a.v.st, tiles.at(p), n, tid);
    };
    auto stage = [&](int p) {
      TI *kb = buf(p);
      if (NBUF == 1 && p > 0) lds_barrier();
      const bool part = !sees_all(a, i0, 32 * RG, tiles.at(p), KT);
      if (part) {
        const bool bad = __any(fk.bad());
        if (__builtin_expect(bad, 0)) fk.clean();
        if (lane == 0) flag[p & 1][wave] = bad;
      }
      fk.stash(kb, tid);
      fv.stash(kb + R::SIZE, tid);
      if (p + 1 < tiles.count) fetch(p + 1);
      lds_barrier();
      return part && any_flag<4>(flag[p & 1]);
    };
    auto compute = [&](int p, bool bad, bool only_sum) {
      const int j = tiles.at(p) + 32 * kp;
      const TI *kb = buf(p) + 32 * kp * RS, *vb = kb + R::SIZE;
      if (iw >= n || !sees_some(a, iw, 32, j, 32)) return;
      const f32x16 S = dots<D, RS>(kb, q, lane);
      const f32x16 P = dots<D, RS>(vb, g, lane);
      float w[16], sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = is_f32<TI> ? fmaf(S[r], a.scale, -lse) * LOG2E_F : fmaf(S[r], c2, -lse2);
        w[r] = __builtin_amdgcn_exp2f(e) * (P[r] - delta);
      }
      if (__builtin_expect(bad, 0)) {
        // (a score of -infinity, weight 0, or a row of NaN, D among it)
        const uint32_t rows = bad_rows<D>(ks + j * a.k.st, a.k.st, n - j, lane);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          w[r] = rows >> krel(r, half) & 1 ? 0.f * (P[r] - delta) : w[r];
      }
      if (!sees_all(a, iw, 32, j, 32)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) w[r] = sees(a, row, j + krel(r, half)) ? w[r] : 0.f;
      }
      if constexpr (FIX) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += w[r];
        off += sum;
        if (only_sum) return;
      }
      mul_rows<D, RS, REST>(acc, kb, w, lane);
      if (__builtin_expect(bad, 0))
        add_bad<D>(acc, ks + j * a.k.st, a.k.st, n - j, lane, 0.f,
                   [&](int i) { return sees(a, row, j + i); });
    };
    auto all_tiles = [&](bool only_sum) {
      fetch(0);
      for (int p = 0; p < tiles.count; ++p) {
        const bool bad = stage(p);
        compute(p, bad, only_sum);
      }
    };
    if (FIX && min((int64_t)i0 + 32 * RG, (int64_t)a.window + a.sinks) <= 128) {
      all_tiles(true);
      offs[wave][lane] = off;
      __syncthreads();
      off = 0.f;
#pragma unroll
      for (int k = 0; k < KP; ++k) off += offs[k * RG + rg][lane];
      off += __shfl_xor(off, 32);
      delta += off;
      off = 0.f;
    }
    all_tiles(false);
  }
  if constexpr (KP > 1) {
    join_parts<RG, KP>(smem, acc, off, 0.f, rg, kp, lane, [&](float po, float, auto part) {
      off += po;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] += part(c, r);
    });
    if (kp > 0) return;
  }
  if constexpr (FIX) {
    off += __shfl_xor(off, 32);
    delta += off;
  }
  if (row >= a.T) return;
  if (half == 0 && row < n) a.delta[srow] = delta;
  if (lse == INFINITY) clear(acc);
  store_row<D, NC>(slice_of<TI>(a.dq, b, h) + row * a.dq.st, acc, half, a.scale);
}

// The key block, the part of its query range and the number of parts of a workgroup.
struct KeyPart {
  int kb, part, parts, slot;  // slot: of its partial sums, -1 if it leaves none
  __device__ __forceinline__ KeyPart(const WinArgs &a, int y) {
    const int first = a.sink_blocks * a.parts_a;
    const bool A = y < first;
    parts = A ? a.parts_a : a.parts_b;
    const int z = A ? y : y - first;
    kb = (A ? 0 : a.sink_blocks) + z / parts;
    part = z % parts;
    slot = parts == 1 ? -1 : z + (!A && a.parts_a > 1 ? first : 0);
  }
};

// dK and dV. One workgroup: 64 keys of one key head, over a part of the 64-query tiles
// that see any of them, of every query head that shares the key head; its four waves
// are two halves of the keys times two halves of each tile's queries, whose sums are
// added at the end through LDS. Blocks whose tiles are many (those of the first
// tokens, which every query sees) are cut into parts, whose sums win_sum_kernel adds in
// order: no atomics, so that the gradients repeat bit for bit.
// At d = 128 the keys and values stay in LDS: with them in registers the sums (128) leave
// too few (fp32, 16 heads, T = 2048, window 512: 76 spilled, 350 us against 212; in bf16
// one wave a SIMD, with room for all, takes 271 us where two take 151). The training step
// above: 150 us, 400 TFLOP/s, bound by two workgroups a CU that wait for LDS and for each
// other (matrix unit busy 18%, vector unit 23%, LDS 36% of the time).
template <typename TI, int D>
__global__ __launch_bounds__(256, is_f32<TI> && D == 128 ? 1 : 2) void win_dkv_kernel(WinArgs a) {
  constexpr int NT = 256, NC = D >= 32 ? D / 32 : 1;
  constexpr bool KV = D == 128;
  using R = Rows<TI, D, WIN_QT, NT>;
  constexpr int RS = R::RS;
  // queries and dO (and keys and values); then the second half's sums
  constexpr int ROWS = (KV ? 4 : 2) * R::SIZE * sizeof(TI) + 64;
  constexpr int RED = 2 * 64 * 2 * NC * 16 * 4;
  __shared__ __attribute__((aligned(16))) char smem[ROWS > RED ? ROWS : RED];
  __shared__ __attribute__((aligned(16))) float stat[2][WIN_QT];  // lse and D of the tile's rows
  __shared__ int flag[4];
  TI *qb = reinterpret_cast<TI *>(smem), *gb = qb + R::SIZE, *kb = gb + R::SIZE, *vb = kb + R::SIZE;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave & 1, qg = wave >> 1;
  const int G = a.H / a.Hkv, kvs = a.B * a.Hkv;
  const int s = blockIdx.x % kvs, b = s / a.Hkv, hk = s % a.Hkv;
  const KeyPart kp(a, blockIdx.x / kvs);
  const int n = length_of(a, b);
  const int j0 = kp.kb * WIN_KB, jw = j0 + 32 * kg, key = jw + l32;
  // queries j0 .. iend - 1 see some key of the block
  const int64_t far = j0 < a.sinks ? n : (int64_t)j0 + WIN_KB - 1 + a.window;
  const int iend = (int)min((int64_t)n, far);
  const int per = iend > j0 ? (iend - j0 + WIN_QT - 1) / WIN_QT : 0, total = per * G;
  const int it0 = (int)((int64_t)total * kp.part / kp.parts);
  const int it1 = (int)((int64_t)total * (kp.part + 1) / kp.parts);
  f32x16 dk[NC], dv[NC];
  clear(dk);
  clear(dv);
  if (it0 < it1) {
    RowReg<TI, D> k, v;
    const TI *ks = slice_of<TI>(a.k, b, hk), *vs = slice_of<TI>(a.v, b, hk);
    R fq, fg;
    if constexpr (KV) {
      fq.fetch(ks, a.k.st, j0, n, tid);
      fg.fetch(vs, a.v.st, j0, n, tid);
      fq.stash(kb, tid);
      fg.stash(vb, tid);
    } else {
      const int at = min(key, n - 1);
      k.load(ks + at * a.k.st, half, key < n);
      v.load(vs + at * a.v.st, half, key < n);
    }
    const float c2 = a.scale * LOG2E_F;
    float lse = 0.f, dd = 0.f;  // of the tile's rows, a lane each (D: the second wave's)
    auto fetch = [&](int it) {
      const int h = hk * G + it / per, i = j0 + it % per * WIN_QT;
      fq.fetch(slice_of<TI>(a.q, b, h), a.q.st, i, n, tid);
      fg.fetch(slice_of<TI>(a.dO, b, h), a.dO.st, i, n, tid);
      const int64_t r = ((int64_t)b * a.H + h) * a.T + i + lane;
      lse = INFINITY, dd = 0.f;
      if (i + lane < n) {
        lse = a.lse[r];
        if (wave == 1) dd = a.delta[r];
      }
    };
    bool none = false;
    auto stage = [&](int it) {
      const int i = j0 + it % per * WIN_QT;
      // rows of no weight, past the end or of no finite score, add nothing: their own
      // infinities and NaNs are zeros in LDS too, and what they make of a key's is masked
      if (lse == -INFINITY) lse = INFINITY;
      none = __any(lse == INFINITY);
      const bool part = none || !sees_all(a, i, WIN_QT, j0, WIN_KB);
      bool bad = false;
      if (part) {
        bad = __any(fq.bad() | fg.bad());
        if (__builtin_expect(bad, 0)) fq.clean(), fg.clean();
      }
      if (it > it0) lds_barrier();
      fq.stash(qb, tid);
      fg.stash(gb, tid);
      if (wave == 0) stat[0][lane] = is_f32<TI> ? lse : lse * LOG2E_F;
      if (wave == 1) stat[1][lane] = dd;
      if (part && lane == 0) flag[wave] = bad;
      if (it + 1 < it1) fetch(it + 1);
      lds_barrier();
      return part && any_flag<4>(flag);
    };
    auto compute = [&](int it, bool bad) {
      const int iw = j0 + it % per * WIN_QT + 32 * qg;
      if (jw >= n || iw >= n || !sees_some(a, iw, 32, jw, 32)) return;
      const TI *qt = qb + 32 * qg * RS, *gt = gb + 32 * qg * RS;
      f32x16 S, P;
      if constexpr (KV) {
        S = dots<D, RS>(qt, kb + 32 * kg * RS, lane);
        P = dots<D, RS>(gt, vb + 32 * kg * RS, lane);
      } else {
        S = dots<D, RS>(qt, k, lane);
        P = dots<D, RS>(gt, v, lane);
      }
      float w[16], ds[16];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 L = *reinterpret_cast<const f32x4 *>(&stat[0][32 * qg + 8 * g + 4 * half]);
        const f32x4 E = *reinterpret_cast<const f32x4 *>(&stat[1][32 * qg + 8 * g + 4 * half]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          const float x = is_f32<TI> ? fmaf(S[r], a.scale, -L[e]) * LOG2E_F
                                     : fmaf(S[r], c2, -L[e]);
          w[r] = __builtin_amdgcn_exp2f(x);
          ds[r] = w[r] * (P[r] - E[e]);
        }
      }
      if (!sees_all(a, iw, 32, jw, 32)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool ok = sees(a, iw + krel(r, half), key);
          w[r] = ok ? w[r] : 0.f;
          ds[r] = ok ? ds[r] : 0.f;
        }
      }
      if (__builtin_expect(none, 0)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool ok = stat[0][32 * qg + krel(r, half)] != INFINITY;
          w[r] = ok ? w[r] : 0.f;
          ds[r] = ok ? ds[r] : 0.f;
        }
      }
      mul_rows<D, RS>(dv, gt, w, lane);
      mul_rows<D, RS>(dk, qt, ds, lane);
      // (a query with such a value has lse or D that makes its weights NaN)
      if (__builtin_expect(bad, 0))
        add_bad<D>(dv, slice_of<TI>(a.dO, b, hk * G + it / per) + iw * a.dO.st, a.dO.st, n - iw,
                   lane, 1.f, [&](int r) {
                     return sees(a, iw + r, key) && stat[0][32 * qg + r] != INFINITY;
                   });
    };
    fetch(it0);
    for (int it = it0; it < it1; ++it) {
      const bool bad = stage(it);
      compute(it, bad);
    }
  }
  // the halves of the queries: the second hands its sums over
  __syncthreads();
  f32x4 *red = reinterpret_cast<f32x4 *>(smem) + kg * 64 * 2 * NC * 4 + lane;
  if (qg == 1) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        red[64 * (8 * c + g)] = f32x4{dk[c][4 * g], dk[c][4 * g + 1], dk[c][4 * g + 2], dk[c][4 * g + 3]};
        red[64 * (8 * c + 4 + g)] = f32x4{dv[c][4 * g], dv[c][4 * g + 1], dv[c][4 * g + 2], dv[c][4 * g + 3]};
      }
  }
  __syncthreads();
  if (qg == 1) return;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = red[64 * (8 * c + g)], y = red[64 * (8 * c + 4 + g)];
#pragma unroll
      for (int e = 0; e < 4; ++e) dk[c][4 * g + e] += x[e], dv[c][4 * g + e] += y[e];
    }
  if (kp.slot < 0) {
    if (key < a.T) {
      store_row<D, NC>(slice_of<TI>(a.dk, b, hk) + key * a.dk.st, dk, half, key < n ? a.scale : 0.f);
      store_row<D, NC>(slice_of<TI>(a.dv, b, hk) + key * a.dv.st, dv, half, key < n ? 1.f : 0.f);
    }
    return;
  }
  const int nkb = (a.T + WIN_KB - 1) / WIN_KB;
  const int64_t slot = (int64_t)s * win_slots(nkb, a.sink_blocks, a.parts_a, a.parts_b) + kp.slot;
  float *out = a.part + (slot * 2 * WIN_KB + 32 * kg + l32) * D;
  store_row<D, NC>(out, dk, half, key < n ? a.scale : 0.f);
  store_row<D, NC>(out + WIN_KB * D, dv, half, key < n ? 1.f : 0.f);
}

// The parts' sums of the blocks that have several, in order of the parts.
template <typename TI, int D> __global__ __launch_bounds__(256) void win_sum_kernel(WinArgs a) {
  const int kvs = a.B * a.Hkv, s = blockIdx.x % kvs, b = s / a.Hkv, hk = s % a.Hkv;
  const int nkb = (a.T + WIN_KB - 1) / WIN_KB;
  constexpr int PER = WIN_KB * D / 4, WGS = (2 * PER + 255) / 256;
  const int y = blockIdx.x / kvs / WGS, z = (int)(blockIdx.x / kvs) % WGS * 256 + threadIdx.x;
  // blocks with several parts: those of the first tokens, the others, or both
  const int kb = a.parts_a > 1 ? y : a.sink_blocks + y;
  const bool A = kb < a.sink_blocks;
  const int parts = A ? a.parts_a : a.parts_b;
  if (kb >= nkb || parts == 1 || z >= 2 * PER) return;
  const int first = a.parts_a > 1 ? a.sink_blocks * a.parts_a : 0;
  const int slot = A ? kb * parts : first + (kb - a.sink_blocks) * parts;
  const float *p = a.part + ((int64_t)s * win_slots(nkb, a.sink_blocks, a.parts_a, a.parts_b) + slot)
                              * 2 * WIN_KB * D + 4 * z;
  f32x4 x = *reinterpret_cast<const f32x4 *>(p);
#pragma unroll 8
  for (int i = 1; i < parts; ++i)
    x += *reinterpret_cast<const f32x4 *>(p + (int64_t)i * 2 * WIN_KB * D);
  const int key = kb * WIN_KB + z % PER / (D / 4), c = z % (D / 4) * 4;
  if (key >= a.T) return;
  const View &out = z < PER ? a.dk : a.dv;
  TI *dst = slice_of<TI>(out, b, hk) + key * out.st + c;
  if constexpr (is_f32<TI>) *reinterpret_cast<f32x4 *>(dst) = x;
  else *reinterpret_cast<u32x2 *>(dst) = u32x2{cvt_bf16x2(x[0], x[1]), cvt_bf16x2(x[2], x[3])};
}

template <typename TI, int D, int RG> void launch_fwd(const WinArgs &a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.B * a.H) * ((a.T + 32 * RG - 1) / (32 * RG));
  hipLaunchKernelGGL((win_fwd_kernel<TI, D, RG>), dim3(grid), dim3(256), 0, s, a);
}
template <typename TI, int D, int RG> void launch_dq(const WinArgs &a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.B * a.H) * ((a.T + 32 * RG - 1) / (32 * RG));
  hipLaunchKernelGGL((win_dq_kernel<TI, D, RG>), dim3(grid), dim3(256), 0, s, a);
}
// Two row groups times two key parts up to a number of 128-query blocks, four row groups
// above. Measured, forward and dQ (us, 2 x 2 / 4 x 1; sinks of 4):
//   bf16 d = 64, T = 1024, window 256   96 blocks 12.7 / 18.9, 14.0 / 20.9; 384 17.6 / 21.3,
//                                       20.8 / 24.5; 768 27.5 / 26.6, 33.1 / 32.3
//   bf16 d = 128, T = 2048, window 512  256 blocks 27.6 / 33.5, 33.5 / 36.4; 512 44.7 / 40.9,
//                                       53.6 / 49.5
//   fp32 d = 64, T = 1024, window 256   96 blocks 24 / 42, 30 / 53; 768 90 / 91, 123 / 134
//   fp32 d = 128, T = 1024, window 256  128 blocks 44 / 69, 58 / 98; 256 82 / 71, 111 / 102
// (1 x 4, with 128 keys a step, gains 1 us on grids of a few blocks and loses above.)
template <typename TI, int D> bool two_groups(const WinArgs &a, int cus) {
  const int64_t blocks = (int64_t)a.B * a.H * ((a.T + 127) / 128);
  return blocks <= (D == 128 ? (is_f32<TI> ? cus / 2 : cus) : is_f32<TI> ? 3 * cus : 2 * cus);
}

template <typename TI, int D> void fwd(const WinArgs &a, int cus, hipStream_t s) {
  timed_call("kia_window_fwd", s, [&] {
    if (two_groups<TI, D>(a, cus)) launch_fwd<TI, D, 2>(a, s);
    else launch_fwd<TI, D, 4>(a, s);
  });
}

template <typename TI, int D> void bwd(const WinArgs &a, int cus, hipStream_t s) {
  timed_call("kia_window_dq", s, [&] {
    if (two_groups<TI, D>(a, cus)) launch_dq<TI, D, 2>(a, s);
    else launch_dq<TI, D, 4>(a, s);
  });
  const int nkb = (a.T + WIN_KB - 1) / WIN_KB, sb = a.sink_blocks;
  const unsigned kvs = a.B * a.Hkv;
  timed_call("kia_window_dkv", s, [&] {
    hipLaunchKernelGGL((win_dkv_kernel<TI, D>),
                       dim3(kvs * (sb * a.parts_a + (nkb - sb) * a.parts_b)), dim3(256), 0, s, a);
  });
  const int blocks = (a.parts_a > 1 ? sb : 0) + (a.parts_b > 1 ? nkb - sb : 0);
  if (blocks) {
    timed_call("kia_window_sum", s, [&] {
      hipLaunchKernelGGL((win_sum_kernel<TI, D>),
                         dim3(kvs * blocks * ((2 * WIN_KB * D / 4 + 255) / 256)), dim3(256), 0, s,
                         a);
    });
  }
}

}  // namespace

template <> void launch_win_fwd<KIA_HEAD>(const WinArgs &a, int dtype, int cus, hipStream_t s) {
  if (dtype == KIA_F32) fwd<float, KIA_HEAD>(a, cus, s);
  else fwd<uint16_t, KIA_HEAD>(a, cus, s);
}
template <> void launch_win_bwd<KIA_HEAD>(const WinArgs &a, int dtype, int cus, hipStream_t s) {
  if (dtype == KIA_F32) bwd<float, KIA_HEAD>(a, cus, s);
  else bwd<uint16_t, KIA_HEAD>(a, cus, s);
}

}  // namespace kia
