// kia_rotary.hip -- rotary positions of query and key heads on gfx950.
//
// Pair n of a head (channels n and n + rot/2, or 2n and 2n + 1) turns by the
// angle p f_n for position p: (a, b) -> m (a cos - b sin, b cos + a sin). The
// gradient is the same with the other sign, the transpose.
//
// Bound by memory: every value is read once and written once, three operations
// each. The angle is shared by all heads of a token, so a workgroup takes a few
// tokens and all their heads (or a share of them, on small grids): cos and sin of
// its tokens go to LDS once, and each thread keeps those of its pairs in registers
// while it walks the heads. Angles are taken in 64 bits, to a quarter turn, and the
// sine and cosine of what is left in 32: a position of 10^6 keeps every digit.
// Queries and keys of 4 x 16 heads of 128 at T = 2048 in bf16, 134 MB in and out: 26 us, 5.2
// TB/s, what a large copy reaches too.
#include "kia_around.hpp"

namespace kia {


template <typename TI, int VW> struct RotVec {
  typedef TI vec __attribute__((ext_vector_type(VW)));
};
template <typename TI> struct RotVec<TI, 1> { typedef TI vec; };

__device__ __forceinline__ uint16_t to_type(float x, uint16_t) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ float to_type(float x, float) { return x; }

// VW: values of one access. A chunk is 2 VW channels of one head: two accesses,
// VW pairs.
template <typename TI, int VW>
__global__ __launch_bounds__(ROT_NT) void rotary_kernel(RotArgs a) {
  typedef typename RotVec<TI, VW>::vec vec;
  extern __shared__ float2 turn[];  // [token][pair]
  const int tid = threadIdx.x, n = a.rot / 2;
  const int nb = (a.T + a.tokens - 1) / a.tokens;
  const int b = blockIdx.x / nb, t0 = (int)(blockIdx.x % nb) * a.tokens;

  for (int e = tid; e < a.tokens * n; e += ROT_NT) {
    const int t = t0 + e / n;
    float s = 0.f, c = 0.f;
    if (t < a.T) {
      const int p = a.pos ? a.pos[(int64_t)b * a.pos_sb + t] : a.first + t;
      // quarter turns: q whole ones and a rest of at most a half
      const double x = (double)p * a.freq[e % n] * 0.63661977236758134308;
      const double q = rint(x);
      sincospif(0.5f * (float)(x - q), &s, &c);
      // (a large q is a multiple of 4 plus these bits whatever its size)
      const int k = (int)(q - 4.0 * floor(q * 0.25));
      if (k & 1) { const float y = s; s = c; c = -y; }
      if (k & 2) { s = -s; c = -c; }
    }
    turn[e] = make_float2(c * a.factor, a.back ? -(s * a.factor) : s * a.factor);
  }
  __syncthreads();

  // thread: chunk, token and the first of its heads
  const int chunks = a.d / (2 * VW);
  const int ch = tid % chunks, tl = tid / chunks % a.tokens, hs = tid / (chunks * a.tokens);
  const int slots = ROT_NT / (chunks * a.tokens), t = t0 + tl;
  if (hs >= slots || t >= a.T) return;
  const int first = blockIdx.y * a.per * slots + hs;
  const int last = min(first - hs + a.per * slots, a.H + a.Hkv);
  const bool turns = ch < n / VW;
  const bool half = a.layout == KIA_ROTARY_HALF;
  // channels of the two accesses
  const int c0 = !turns || !half ? 2 * VW * ch : VW * ch;
  const int c1 = turns && half ? c0 + n : c0 + VW;
  float cs[VW], sn[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    const float2 w = turns ? turn[tl * n + VW * ch + e] : make_float2(1.f, 0.f);
    cs[e] = w.x, sn[e] = w.y;
  }
  for (int h = first; h < last; h += slots) {
    const bool key = h >= a.H;
    const RotSide &s = key ? a.k : a.q;
    const int hh = key ? h - a.H : h;
    const TI *x = (const TI *)s.x + b * s.xb + hh * s.xh + t * s.xt;
    TI *y = (TI *)s.y + b * s.yb + hh * s.yh + t * s.yt;
    vec u = *(const vec *)(x + c0), v = *(const vec *)(x + c1);
    if (turns) {
      float p[2 * VW];
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        if constexpr (VW == 1) p[0] = load1(&u), p[1] = load1(&v);
        else {
          const TI ue = u[e], ve = v[e];
          p[e] = load1(&ue), p[VW + e] = load1(&ve);
        }
      }
      float r[2 * VW];
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        const int ia = half ? e : 2 * e, ib = half ? VW + e : 2 * e + 1;
        const float pa = p[ia], pb = p[ib];
        r[ia] = fmaf(pa, cs[e], -(pb * sn[e]));
        r[ib] = fmaf(pb, cs[e], pa * sn[e]);
      }
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        if constexpr (VW == 1) u = to_type(r[0], TI()), v = to_type(r[1], TI());
        else u[e] = to_type(r[e], TI()), v[e] = to_type(r[VW + e], TI());
      }
    }
    *(vec *)(y + c0) = u;
    *(vec *)(y + c1) = v;
  }
}

template <typename TI, int VW> static void launch(const RotArgs &a, dim3 grid, hipStream_t s) {
  hipLaunchKernelGGL((rotary_kernel<TI, VW>), grid, dim3(ROT_NT),
                     a.tokens * (a.rot / 2) * sizeof(float2), s, a);
}

// The grid: workgroups of `tokens` tokens, and the heads in as many shares as it takes to
// reach four workgroups per CU.
void launch_rotary(RotArgs a, int dtype, int cus, hipStream_t s) {
  int vw;
  a.tokens = rotary_tokens(a.T, a.d, a.rot, dtype, vw);
  const int chunks = a.d / (2 * vw);
  const int slots = ROT_NT / (chunks * a.tokens);
  const int rounds = (a.H + a.Hkv + slots - 1) / slots;
  const unsigned nb = (unsigned)a.B * ((a.T + a.tokens - 1) / a.tokens);
  int shares = (int)((4u * cus + nb - 1) / nb);
  shares = shares < 1 ? 1 : shares > rounds ? rounds : shares;
  a.per = (rounds + shares - 1) / shares;
  const dim3 grid(nb, (rounds + a.per - 1) / a.per);
  if (dtype == KIA_F32) {
    if (vw == 4) launch<float, 4>(a, grid, s);
    else if (vw == 2) launch<float, 2>(a, grid, s);
    else launch<float, 1>(a, grid, s);
  } else {
    if (vw == 8) launch<uint16_t, 8>(a, grid, s);
    else if (vw == 4) launch<uint16_t, 4>(a, grid, s);
    else if (vw == 2) launch<uint16_t, 2>(a, grid, s);
    else launch<uint16_t, 1>(a, grid, s);
  }
}

}  // namespace kia
