// kia_select.hip -- the pages that attention over a long cache reads: for every new token
// and key head those whose keys could score highest.
//
// A page's keys lie between its bounds lo and hi in every channel c, so no score q.k of the
// page is above sum_c max(q_c lo_c, q_c hi_c). The largest of that over the key head's query
// heads ranks the page. Pages are ranked in 64 bits: of bf16 queries the terms and nearly
// every sum are exact there, so that the order depends on no order of summation.
//
// Scores are bound by memory, 4 d bytes a page and head, and by the vector unit, which the sums
// in 64 bits keep busy for as long. D / 8 lanes take a page, eight channels each.
// A selection is one workgroup's: the count-th largest score is found digit by digit of its
// bits (eight at a time, from the first one in which the scores differ), and the pages
// above it are written in their order, of pages with that score the first ones.
#include "kia_around.hpp"
#include "kia_host.hpp"

namespace kia {
namespace {

constexpr int NT = 256;
constexpr uint64_t ALWAYS = ~0ull;  // the rank of first and last pages; 0: no candidate

// A double's place in their order as an integer (not 0 and not ALWAYS); NaN ranks as infinity.
__device__ __forceinline__ uint64_t rank_of(double x) {
  if (x != x) x = INFINITY;
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | 1ull << 63;
}

template <int CTRL> __device__ __forceinline__ double moved(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = __builtin_amdgcn_mov_dpp((int)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(b >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// The sum over the D / 8 lanes of a page.
template <int D> __device__ __forceinline__ double page_sum(double x) {
  x += moved<0xb1>(x);                              // quad_perm 1 0 3 2
  x += moved<0x4e>(x);                              // quad_perm 2 3 0 1
  if constexpr (D >= 64) x += moved<0x141>(x);      // row_half_mirror
  if constexpr (D >= 128) x += moved<0x140>(x);     // row_mirror
  return x;
}

// Pages a workgroup ranks.
template <int D> struct Batch { static constexpr int N = 8 * NT / D; };

template <typename TI, int D> __global__ __launch_bounds__(NT) void score_kernel(SelectArgs a) {
  constexpr int OCTS = D / 8;
  extern __shared__ __attribute__((aligned(16))) float rows[];  // [tokens x heads of the group][D]
  const int tid = threadIdx.x, oct = tid % OCTS, G = a.H / a.Hkv;
  const int hk = blockIdx.x % a.Hkv, b = (int)(blockIdx.x / a.Hkv) % a.B;
  const int w = (int)(blockIdx.x / a.Hkv / a.B) * Batch<D>::N + tid / OCTS;  // this lane's page
  const int64_t length = min((int64_t)a.lengths[b], (int64_t)a.width << a.lpage);
  if ((int64_t)(w - tid / OCTS) << a.lpage >= length) return;
  const int page = w < a.width ? a.table[(int64_t)b * a.width + w] : -1;
  const bool ok = page >= 0 && page < a.pages;
  u32x4 lo = {}, hi = {};
  if (ok) {
    const u32x4 *p = reinterpret_cast<const u32x4 *>(a.bounds + ((int64_t)page * a.Hkv + hk) * D) + oct;
    lo = p[0], hi = p[OCTS];
  }
  const int t0 = blockIdx.y * a.tokens, t1 = min(t0 + a.tokens, a.T);
  for (int e = tid; e < (t1 - t0) * G * OCTS; e += NT) {
    const int r = e / OCTS, o = e % OCTS;
    const TI *q = slice_of<TI>(a.q, b, hk * G + r % G) + (t0 + r / G) * a.q.st + 8 * o;
#pragma unroll
    for (int i = 0; i < 8; i += 4)
      *reinterpret_cast<f32x4 *>(rows + r * D + 8 * o + i) = load4(q + i);
  }
  __syncthreads();
  double l[8], h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    l[e] = __uint_as_float(e % 2 ? lo[e / 2] & 0xffff0000u : lo[e / 2] << 16);
    h[e] = __uint_as_float(e % 2 ? hi[e / 2] & 0xffff0000u : hi[e / 2] << 16);
  }
  for (int t = t0; t < t1; ++t) {
    uint64_t top = 0;
    for (int g = 0; g < G; ++g) {
      const float *q = rows + ((t - t0) * G + g) * D + 8 * oct;
      double s = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // (NaN: either way)
        s = fma((double)q[e], q[e] > 0.f ? h[e] : l[e], s);
      }
      top = max(top, rank_of(page_sum<D>(s)));
    }
    const int64_t pos = length - a.T + t, at = pos >> a.lpage;
    if (oct == 0 && w < a.width) {
      const bool always = w < a.first || w > at - a.last;
      a.score[(((int64_t)b * a.Hkv + hk) * a.T + t) * a.width + w] = !ok || w > at ? 0 : always ? ALWAYS : top;
    }
  }
}

// The ranks of a selection: in registers up to 8 x 256, read again and again beyond.
__global__ __launch_bounds__(NT) void select_kernel(SelectArgs a) {
  constexpr int KEEP = 8;
  __shared__ uint32_t bins[256], sums[8];
  __shared__ uint64_t ends[8];
  __shared__ int pick[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t = blockIdx.x % a.T, b = blockIdx.x / a.T / a.Hkv;
  const int64_t length = min((int64_t)a.lengths[b], (int64_t)a.width << a.lpage);
  const int64_t pos = length - a.T + t;
  const int n = pos < 0 ? 0 : (int)(pos >> a.lpage) + 1;
  const uint64_t *score = a.score + (int64_t)blockIdx.x * a.width;
  int *list = a.list + (int64_t)blockIdx.x * a.count;
  uint64_t mine[KEEP];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) mine[i] = tid + i * NT < n ? score[tid + i * NT] : 0;
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < KEEP; ++i) f(mine[i]);
    for (int i = tid + KEEP * NT; i < n; i += NT) f(score[i]);
  };
  // candidates, pages taken in any case, least and largest rank of the others
  uint32_t all = 0, must = 0;
  uint64_t least = ALWAYS, most = 0;
  each([&](uint64_t x) {
    all += x != 0;
    must += x == ALWAYS;
    if (x && x != ALWAYS) least = min(least, x), most = max(most, x);
  });
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    all += __shfl_xor(all, i);
    must += __shfl_xor(must, i);
    least = min(least, (uint64_t)__shfl_xor((unsigned long long)least, i));
    most = max(most, (uint64_t)__shfl_xor((unsigned long long)most, i));
  }
  if (lane == 0) sums[wave] = all, sums[4 + wave] = must, ends[wave] = least, ends[4 + wave] = most;
  __syncthreads();
  all = sums[0] + sums[1] + sums[2] + sums[3];
  must = sums[4] + sums[5] + sums[6] + sums[7];
  least = min(min(ends[0], ends[1]), min(ends[2], ends[3]));
  most = max(max(ends[4], ends[5]), max(ends[6], ends[7]));
  // taken of the others: ranks with (rank & mask) > cut, and of those equal to it the first
  // `equal`. (must <= first + last <= count)
  const bool every = (int)all <= a.count;
  uint64_t cut = ALWAYS, mask = ALWAYS;
  uint32_t equal = every ? 0 : a.count - must;
  if (equal) {
    int bits = least == most ? 0 : 64 - __builtin_clzll(least ^ most);  // undecided low bits
    mask = bits > 63 ? 0 : ALWAYS << bits;
    cut = most & mask;
    while (bits > 0) {
      const int shift = max(bits - 8, 0);
      const uint32_t digit = (1u << (bits - shift)) - 1;
      __syncthreads();
      bins[tid] = 0;
      __syncthreads();
      each([&](uint64_t x) {
        if (x && x != ALWAYS && (x & mask) == cut) atomicAdd(&bins[(uint32_t)(x >> shift) & digit], 1u);
      });
      __syncthreads();
      // from the top: bin 255 - tid, and how many lie above it
      const uint32_t v = bins[255 - tid];
      uint32_t to = v;
#pragma unroll
      for (int i = 1; i < 64; i *= 2) {
        const uint32_t y = __shfl_up(to, i);
        if (lane >= i) to += y;
      }
      if (lane == 63) sums[wave] = to;
      __syncthreads();
      for (int i = 0; i < wave; ++i) to += sums[i];
      if (to >= equal && to - v < equal) pick[0] = 255 - tid, pick[1] = (int)(equal - (to - v));
      __syncthreads();
      cut |= (uint64_t)pick[0] << shift;
      equal = (uint32_t)pick[1];
      const bool whole = equal == bins[pick[0]];
      bits = shift;
      mask = ALWAYS << bits;
      if (whole) break;  // every rank with these digits is taken
    }
  }
  // written in order, 256 pages at a time
  uint32_t done = 0, same = 0;
  for (int i0 = 0; i0 < n; i0 += NT) {
    const uint64_t x = i0 + tid < n ? score[i0 + tid] : 0;
    const bool eq = equal && x && x != ALWAYS && (x & mask) == cut;
    const uint64_t below = (1ull << lane) - 1, qs = __ballot(eq);
    __syncthreads();
    if (lane == 0) sums[wave] = __popcll(qs);
    __syncthreads();
    uint32_t rank = same + __popcll(qs & below);
    for (int i = 0; i < 4; ++i) {
      if (i < wave) rank += sums[i];
      same += sums[i];
    }
    const bool take = x && (every || x == ALWAYS || (eq ? rank < equal : (x & mask) > cut));
    const uint64_t ts = __ballot(take);
    if (lane == 0) sums[4 + wave] = __popcll(ts);
    __syncthreads();
    uint32_t at = done + __popcll(ts & below);
    for (int i = 0; i < 4; ++i) {
      if (i < wave) at += sums[4 + i];
      done += sums[4 + i];
    }
    if (take && at < (uint32_t)a.count) list[at] = i0 + tid;
  }
  for (int i = done + tid; i < a.count; i += NT) list[i] = -1;
}

template <typename TI, int D> void run(const SelectArgs &a, hipStream_t s) {
  const unsigned batches = (a.width + Batch<D>::N - 1) / Batch<D>::N;
  const size_t lds = (size_t)a.tokens * (a.H / a.Hkv) * D * sizeof(float);
  const dim3 grid(batches * a.B * a.Hkv, (a.T + a.tokens - 1) / a.tokens);
  timed_call("kia_cache4_score", s, [&] {
    hipLaunchKernelGGL((score_kernel<TI, D>), grid, dim3(NT), lds, s, a);
  });
  timed_call("kia_cache4_select", s, [&] {
    hipLaunchKernelGGL(select_kernel, dim3((unsigned)a.B * a.Hkv * a.T), dim3(NT), 0, s, a);
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
