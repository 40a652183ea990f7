// Rotary positions with several axes: the pairs of a head are divided among the axes of a token's position (one for text,
// height and width for an image, time too for a video), and pair i, of axis x(i), is turned by the angle
//
//   a = position[t, x(i)] * freq[i]   (a 32-bit product):   (u, v) -> (u cos a - v sin a, v cos a + u sin a).
//
// The backward pass is the same turn by -a.  Elements of a head past the rotated ones are copied.
//
// Bound by memory (3 flops per element): every element is read and written once.  The cosines and sines of a block's tokens
// are computed once into LDS and serve all heads; then the block's lanes take 16-byte pieces of both members of eight pairs,
// in memory order over the heads of a token, so that loads and stores run along whole lines.
#include "nm_device.h"
#include "nm_launch.h"
#include "nm_rows.h"

namespace nm {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotPairs = 512;  // cosines and sines that a block keeps: 4 KiB

struct RotArgs {
  RotaryCall c;
  int tokens;   // per block
  int pairs;    // R / 2
};

// N = 8: pairs and the elements behind them in 16-byte pieces; N = 1: any alignment, one pair or one element per lane.
template <bool XF32, int N>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const RotArgs a) {
  __shared__ float2 turn[kRotPairs];
  const RotaryCall& c = a.c;
  const int64_t t0 = flat_lane_256() / kRotThreads * a.tokens;
  if (t0 >= c.T) return;
  const int n_tokens = (int)(c.T - t0 < a.tokens ? c.T - t0 : a.tokens);
  for (int p0 = 0; p0 < a.pairs; p0 += kRotPairs) {  // (heads of over 1024 rotated elements: a run of pairs at a time)
    const int n_pairs = a.pairs - p0 < kRotPairs ? a.pairs - p0 : kRotPairs;
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
    const bool last = p0 + n_pairs == a.pairs;
    // lanes of a head: its pairs of this run, and with the last run what lies behind the rotated elements
    const int rotate = n_pairs / (c.interleaved ? (N == 8 ? 4 : 1) : N);
    const int rest = last ? (int)(c.D - 2 * a.pairs) / N : 0;
    const int per_head = rotate + rest, per_token = per_head * (int)c.H;
    for (int i = threadIdx.x; i < n_tokens * per_token; i += kRotThreads) {
      const int tok = i / per_token, j = i % per_token, head = j / per_head, k = j % per_head;
      const int64_t xb = (t0 + tok) * c.x_token + head * c.x_head, yb = (t0 + tok) * c.y_token + head * c.y_head;
      const float2* w = turn + tok * n_pairs;
      if (k >= rotate) {
        const int at = 2 * a.pairs + (k - rotate) * N;
        float v[N];
        load_vec<XF32, N>(c.X, xb + at, v);
        store_vec<N>(c.Y, yb + at, v, !c.y_f32);
      } else if (c.interleaved) {
        if constexpr (N == 8) {
          float v[8], y[8];
          const int at = 2 * p0 + k * 8;
          load_vec<XF32, 8>(c.X, xb + at, v);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 cw = w[k * 4 + e];
            y[2 * e] = v[2 * e] * cw.x - v[2 * e + 1] * cw.y;
            y[2 * e + 1] = v[2 * e + 1] * cw.x + v[2 * e] * cw.y;
          }
          store_vec<8>(c.Y, yb + at, y, !c.y_f32);
        } else {
          float u[1], v[1];
          const int at = 2 * (p0 + k);
          load_vec<XF32, 1>(c.X, xb + at, u);
          load_vec<XF32, 1>(c.X, xb + at + 1, v);
          const float2 cw = w[k];
          const float y0[1] = {u[0] * cw.x - v[0] * cw.y}, y1[1] = {v[0] * cw.x + u[0] * cw.y};
          store_vec<1>(c.Y, yb + at, y0, !c.y_f32);
          store_vec<1>(c.Y, yb + at + 1, y1, !c.y_f32);
        }
      } else {
        float u[N], v[N], y0[N], y1[N];
        const int at = p0 + k * N;
        load_vec<XF32, N>(c.X, xb + at, u);
        load_vec<XF32, N>(c.X, xb + a.pairs + at, v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 cw = w[k * N + e];
          y0[e] = u[e] * cw.x - v[e] * cw.y;
          y1[e] = v[e] * cw.x + u[e] * cw.y;
        }
        store_vec<N>(c.Y, yb + at, y0, !c.y_f32);
        store_vec<N>(c.Y, yb + a.pairs + at, y1, !c.y_f32);
      }
    }
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryCall& c, hipStream_t s) {
  RotArgs a;
  a.c = c;
  a.pairs = (int)(c.R / 2);
  const bool pieces = (c.D | c.R | c.x_token | c.x_head | c.y_token | c.y_head) % 8 == 0 &&
                      (c.interleaved || a.pairs % 8 == 0) && ((uintptr_t)c.X & 15) == 0 && ((uintptr_t)c.Y & 15) == 0;
  // tokens per block: enough work for its lanes (a few pieces each), as far as their cosines fit
  const int64_t lanes = (c.H * c.D / (pieces ? 16 : 2) > 0) ? c.H * c.D / (pieces ? 16 : 2) : 1;
  int64_t tokens = (4 * kRotThreads + lanes - 1) / lanes;
  const int64_t room = kRotPairs / (a.pairs < kRotPairs ? a.pairs : kRotPairs);
  tokens = tokens < room ? tokens : room;
  const int64_t spread = (c.T + 511) / 512;  // ... and blocks enough for the chip
  tokens = tokens < spread ? tokens : spread;
  a.tokens = (int)(tokens > 0 ? tokens : 1);
  const dim3 grid = flat_grid_256((c.T + a.tokens - 1) / a.tokens * kRotThreads);
  if (pieces) {
    if (c.x_f32) rotary_kernel<true, 8><<<grid, kRotThreads, 0, s>>>(a);
    else rotary_kernel<false, 8><<<grid, kRotThreads, 0, s>>>(a);
  } else {
    if (c.x_f32) rotary_kernel<true, 1><<<grid, kRotThreads, 0, s>>>(a);
    else rotary_kernel<false, 1><<<grid, kRotThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace nm
