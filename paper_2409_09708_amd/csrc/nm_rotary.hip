// Rotary positions with several axes: the pairs of a head are divided among the axes of a token's position (one for text,
// height and width for an image, time too for a video), and pair i, of axis x(i), is turned by the angle
//
//   a = position[t, x(i)] * freq[i]   (a 32-bit product):   (u, v) -> (u cos a - v sin a, v cos a + u sin a).
//
// The backward pass is the same turn by -a.  Elements of a head past the rotated ones are copied.
//
// Bound by memory (3 flops per element): every element is read and written once.  The cosines and sines of a block's tokens
// are computed once into LDS and serve all heads; then the block's lanes take both members of eight pairs, in memory order
// over the heads of a token, so that loads and stores run along whole lines.
// Measured: 12608 tokens of 24 heads of 64 inside a joint projection's output, two axes, bfloat16: 14.4 us, 5.4 TB/s; 16399 tokens of
// 10 heads of 128, 96 of them turned, interleaved, float to bfloat16: 20.5 us, 6.1 TB/s.  Both at the rate of a large copy.
#include "nm_device.h"
#include "nm_launch.h"
#include "nm_rows.h"

namespace nm {

namespace {

constexpr int kRotThreads = 256;  // (flat_grid_256)
constexpr int kRotPairs = 512;    // cosines and sines that a block keeps: 4 KiB

struct RotArgs {
  RotaryCall c;
  int tokens;  // per block
  int pairs;   // R / 2
};

// i / d for 0 <= i < 2^21, from 1 / d: the quotient is at least 0.5 / d away from the next integer, the product off by less
__device__ __forceinline__ int quotient(int i, float inverse) { return (int)(((float)i + 0.5f) * inverse); }

template <bool XF32, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const RotArgs a) {
  __shared__ float2 turn[kRotPairs];
  const RotaryCall& c = a.c;
  const int64_t t0 = flat_lane_256() / kRotThreads * a.tokens;
  if (t0 >= c.T) return;
  const int n_tokens = (int)(c.T - t0 < a.tokens ? c.T - t0 : a.tokens);
  for (int p0 = 0; p0 < a.pairs; p0 += kRotPairs) {  // (heads of over 1024 rotated elements: a run of pairs at a time)
    const int n_pairs = a.pairs - p0 < kRotPairs ? a.pairs - p0 : kRotPairs;
    // pieces of a head: its pairs of this run, eight (interleaved: four) at a time, and with the last run what lies behind the
    // rotated elements
    constexpr int PER_PIECE = INTERLEAVED ? 4 : 8;
    const int rotate = (n_pairs + PER_PIECE - 1) / PER_PIECE;
    const int rest = p0 + n_pairs == a.pairs ? ((int)c.D - 2 * a.pairs + 7) / 8 : 0;
    const int per_head = rotate + rest, per_token = per_head * (int)c.H, n_pieces = n_tokens * per_token;
    const float by_token = 1.f / (float)per_token, by_head = 1.f / (float)per_head;
    struct Place { int tok, head, k, at, n; };  // at: its first element in the head, n: how many (of pairs: of their first members)
    auto place = [&](int i) {
      Place p;
      p.tok = quotient(i, by_token);
      const int j = i - p.tok * per_token;
      p.head = quotient(j, by_head);
      p.k = j - p.head * per_head;
      if (p.k >= rotate) {
        p.at = 2 * a.pairs + (p.k - rotate) * 8;
        p.n = (int)c.D - p.at;
      } else {
        p.at = INTERLEAVED ? 2 * p0 + p.k * 8 : p0 + p.k * 8;
        p.n = INTERLEAVED ? 2 * (n_pairs - p.k * 4) : n_pairs - p.k * 8;
      }
      return p;
    };
    Raw8<XF32> u, v;
    auto fetch = [&](int i) {
      if (i >= n_pieces) return;
      const Place p = place(i);
      const int64_t x = (t0 + p.tok) * c.x_token + p.head * c.x_head + p.at;
      u.load(c.X, x, p.n);
      if (!INTERLEAVED && p.k < rotate) v.load(c.X, x + a.pairs, p.n);
    };
    fetch(threadIdx.x);  // (on its way while the angles are computed)
    if (p0) __syncthreads();
    for (int i = threadIdx.x; i < n_tokens * n_pairs; i += kRotThreads) {
      const int64_t t = t0 + i / n_pairs;
      const int pair = p0 + i % n_pairs;
      int axis = 0;
#pragma unroll
      for (int x = 0; x < kMaxRotaryAxes - 1; ++x) axis += pair >= c.section_end[x] ? 1 : 0;
      const int64_t at = t * c.axes + axis;
      const float pos = c.positions_f32 ? static_cast<const float*>(c.positions)[at]
                                        : (float)static_cast<const int32_t*>(c.positions)[at];
      float sn, cs;
      sincosf(pos * c.freqs[pair], &sn, &cs);
      turn[i] = float2{cs, c.inverse ? -sn : sn};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_pieces; i += kRotThreads) {
      const Place p = place(i);
      const int64_t y = (t0 + p.tok) * c.y_token + p.head * c.y_head + p.at;
      const float2* w = turn + p.tok * n_pairs + p.k * PER_PIECE;
      float y0[8], y1[8];
      if (p.k >= rotate) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y0[e] = u[e];
      } else if constexpr (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 cw = 2 * e < p.n ? w[e] : float2{1.f, 0.f};
          y0[2 * e] = u[2 * e] * cw.x - u[2 * e + 1] * cw.y;
          y0[2 * e + 1] = u[2 * e + 1] * cw.x + u[2 * e] * cw.y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 cw = e < p.n ? w[e] : float2{1.f, 0.f};
          y0[e] = u[e] * cw.x - v[e] * cw.y;
          y1[e] = v[e] * cw.x + u[e] * cw.y;
        }
      }
      fetch(i + kRotThreads);
      store8(c.Y, y, p.n, y0, !c.y_f32);
      if (!INTERLEAVED && p.k < rotate) store8(c.Y, y + a.pairs, p.n, y1, !c.y_f32);
    }
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryCall& c, hipStream_t s) {
  RotArgs a;
  a.c = c;
  a.pairs = (int)(c.R / 2);
  // tokens per block: two pieces for each of its lanes, as far as their cosines fit, ...
  const int64_t per_token = c.H * c.D / (c.interleaved ? 8 : 16), pieces = per_token > 0 ? per_token : 1;
  int64_t tokens = (2 * kRotThreads + pieces - 1) / pieces;
  const int64_t room = kRotPairs / (a.pairs < kRotPairs ? a.pairs : kRotPairs);
  tokens = tokens < room ? tokens : room;
  const int64_t spread = (c.T + 511) / 512;  // ... and blocks enough for the chip
  tokens = tokens < spread ? tokens : spread;
  a.tokens = (int)tokens;
  const dim3 grid = flat_grid_256((c.T + a.tokens - 1) / a.tokens * kRotThreads);
  if (c.interleaved) {
    if (c.x_f32) rotary_kernel<true, true><<<grid, kRotThreads, 0, s>>>(a);
    else rotary_kernel<false, true><<<grid, kRotThreads, 0, s>>>(a);
  } else {
    if (c.x_f32) rotary_kernel<true, false><<<grid, kRotThreads, 0, s>>>(a);
    else rotary_kernel<false, false><<<grid, kRotThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace nm
