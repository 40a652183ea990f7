// Norm of each head of each token over its own D elements, then the rotary turn of its pairs, and the backward pass of both.
//
//   c = x - mean(x) (layer norm: centred) or x (root mean square),  rstd = 1 / sqrt(mean(c^2) + eps),  n = c rstd,
//   y = turn(n w),   pair i of axis x(i) turned by a = position[t, x(i)] freq[i]:  (u, v) -> (u cos a - v sin a, v cos a + u sin a)
//
// and with d = turn^-1(dy), g = d w:   dx = rstd (g (- mean(g)) - n mean(g n)),   dw = sum over tokens and heads of d n.
// The first `heads` heads (queries) take one row of weights, the others (keys) the second.
//
// A head is held by LANES lanes, each with two runs of eight elements: both members of eight pairs, or sixteen elements in a row of
// neighbouring pairs and of what is not turned.  So a norm is a few exchanges between lanes, a turn none, and rstd is computed again
// in the backward pass rather than kept.  The angles of a block's tokens go to LDS once for all heads, reduced to half a turn either way
// in 64 bits: a 32-bit product of position 65536 is off by up to 2^-9 of a radian, as much as a rounding to bfloat16.
// Sums and statistics are 32-bit floats; the mean is corrected by the mean difference to it, as large offsets need.
//
// Bound by memory: 10 flops per element forward, 18 backward, for 4 to 12 bytes.  12608 tokens of 24 heads of 64, bfloat16, two axes: 15.8 to 17.8 us
// (by the card, and by how much of its 78 MB the last level of cache still has; under the profiler 16.8), 4.4 to 4.9 TB/s, where a copy of 1 GiB has
// 5.5; gradients of 8191 x 40 x 128, bfloat16, 56.5 to 60.8 us and of 16399 x 10 x 80, float, 42.8, each with 5 for the second launch; one token 3.2
// and the host's side of a call.
#include "nm_device.h"
#include "nm_launch.h"
#include "nm_rows.h"

#include <type_traits>

namespace nm {

namespace {

constexpr int kHeadThreads = 256;  // (flat_grid_256)
constexpr int kHeadPairs = 1024;   // cosines and sines that a block keeps: 8 KiB
constexpr int kGradPairs = 4096;   // ... of the backward pass: 32 KiB, for one run of tokens a block (with 1024 the two above took 64.4 and 46.0 us)
constexpr int kHeadMost = 512;     // elements of a head

// The heads that share a row of weights: a block takes those of a run of tokens.
struct HeadSet {
  int first, count;  // heads
  int tokens;        // of a block at a time
  int splits;        // blocks that share a token's heads (few tokens)
  int64_t blocks;
};
struct HeadArgs {
  HeadNormCall c;
  HeadSet set[2];   // queries and keys (the latter with no blocks where all heads share their weights)
  int pairs;        // R / 2
  int rotate;       // pieces of a head with pairs that are turned
  float* partial;   // backward: [blocks][D], those of the first set before those of the second; NULL: no gradient of the weights
};

// i / d for 0 <= i < 2^21, from 1 / d: the quotient is at least 0.5 / d away from the next integer, the product off by less
constexpr int64_t kHeadMostUnits = 1 << 20;  // (a token has no more heads)
__device__ __forceinline__ int head_quotient(int i, float inverse) { return (int)(((float)i + 0.5f) * inverse); }

// Sum over the LANES lanes of a head.  Up to 16 lanes the exchanges are operands of the additions: neighbours, pairs, then the halves of
// eight and of 16 lanes mirrored, which are all the same by then.  (Gradients of 8191 x 40 x 128: 77.5 us with exchanges through LDS.)
template <int CONTROL>
__device__ __forceinline__ float lane_moved(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CONTROL, 0xF, 0xF, true));
}
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
  v += lane_moved<0xB1>(v);
  v += lane_moved<0x4E>(v);
  if constexpr (LANES >= 8) v += lane_moved<0x141>(v);
  if constexpr (LANES >= 16) v += lane_moved<0x140>(v);
#pragma unroll
  for (int m = 16; m < LANES; m <<= 1) v += __shfl_xor(v, m, 64);
  return v;
}

// Where unit i of a run of tokens lies: its token in the run, its head, and the element at which they begin (strides fit 32 bits).
struct HeadUnit {
  int tok, head;
  __device__ __forceinline__ HeadUnit(const HeadSet& s, int i, float by_count) {
    tok = head_quotient(i, by_count);
    head = s.first + i - tok * s.count;
  }
  __device__ __forceinline__ int64_t at(int64_t run, int token, int heads) const { return run + (int64_t)tok * token + (int64_t)head * heads; }
};

// The two runs of eight elements that lane k of a head holds: where they begin, how many there are (<= 0: none), and the first of their
// pairs in the table of a token's turns.  Lanes side by side hold runs side by side, so that an access covers whole lines.
struct HeadPiece {
  int at[2], n[2], pair[2];
  bool turned;
};
template <bool INTERLEAVED>
__device__ __forceinline__ HeadPiece head_piece(const HeadArgs& a, int k) {
  HeadPiece p;
  const int D = (int)a.c.D;
  p.turned = k < a.rotate;
  if (!INTERLEAVED && p.turned) {  // both members of eight pairs
    p.pair[0] = p.pair[1] = p.at[0] = k * 8;
    p.at[1] = a.pairs + k * 8;
    p.n[0] = p.n[1] = a.pairs - k * 8;
  } else {                         // twice four pairs, or what is not turned
    const int from = p.turned ? 0 : 2 * a.pairs, to = p.turned ? 2 * a.pairs : D, lanes = p.turned ? a.rotate : (D - from + 15) / 16;
    const int i = p.turned ? k : k - a.rotate;
    p.at[0] = from + i * 8;
    p.at[1] = from + (lanes + i) * 8;
    p.n[0] = i < lanes ? to - p.at[0] : 0;
    p.n[1] = i < lanes ? to - p.at[1] : 0;
    p.pair[0] = p.at[0] / 2;
    p.pair[1] = p.at[1] / 2;
  }
  return p;
}

// A lane's two runs.  WHOLE: each has eight elements or none (left as it was then, which is zeros), so nothing is read or written singly.
template <bool F32, bool WHOLE>
struct HeadRaw {
  Raw8<F32> r[2];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int v = 0; v < (F32 ? 2 : 1); ++v) r[i].v[v] = u32x4_t{0, 0, 0, 0};
  }
  __device__ __forceinline__ void load(const void* base, int64_t row, const HeadPiece& p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (WHOLE) {
        if (p.n[i] > 0) r[i].load(base, row + p.at[i], 8);
      } else {
        r[i].load(base, row + p.at[i], p.n[i]);
      }
    }
  }
};
template <bool WHOLE>
__device__ __forceinline__ void head_store(void* base, int64_t row, const HeadPiece& p, const float (&u)[8], const float (&v)[8], bool f32) {
  if (p.n[0] > 0) store8(base, row + p.at[0], WHOLE ? 8 : p.n[0], u, !f32);
  if (p.n[1] > 0) store8(base, row + p.at[1], WHOLE ? 8 : p.n[1], v, !f32);
}

// The turn of a lane's pairs, back where `back`; w: the token's cosines and sines.
template <bool INTERLEAVED, bool WHOLE>
__device__ __forceinline__ void head_turn(float (&u)[8], float (&v)[8], const float2* w, const HeadPiece& p, bool back) {
  if (!p.turned) return;
  if constexpr (INTERLEAVED) {
    auto run = [&](float (&q)[8], int r) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 cs = (WHOLE ? 0 : 2 * e) < p.n[r] ? w[p.pair[r] + e] : float2{1.f, 0.f};
        const float sn = back ? -cs.y : cs.y, x = q[2 * e], y = q[2 * e + 1];
        q[2 * e] = x * cs.x - y * sn;
        q[2 * e + 1] = y * cs.x + x * sn;
      }
    };
    run(u, 0);
    run(v, 1);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 cs = WHOLE || e < p.n[0] ? w[p.pair[0] + e] : float2{1.f, 0.f};
      const float sn = back ? -cs.y : cs.y, x = u[e], y = v[e];
      u[e] = x * cs.x - y * sn;
      v[e] = y * cs.x + x * sn;
    }
  }
}

// Cosines and sines of the pairs of n_tokens tokens from t0 on, in two halves: what they are computed from is asked for before the heads'
// elements are, since loads come back in order (64 images 17.3 us, 18.1 asked for after them), where registers allow.
struct HeadAngle {
  uint32_t position;
  float freq;
  __device__ __forceinline__ void load(const HeadArgs& a, int64_t t0, int i, float by_pairs) {
    const HeadNormCall& c = a.c;
    const int tok = head_quotient(i, by_pairs), pair = i - tok * a.pairs;
    int axis = 0;
#pragma unroll
    for (int x = 0; x < kMaxRotaryAxes - 1; ++x) axis += pair >= c.section_end[x] ? 1 : 0;
    position = static_cast<const uint32_t*>(c.positions)[(t0 + tok) * c.axes + axis];
    freq = c.freqs[pair];
  }
  __device__ __forceinline__ void store(const HeadArgs& a, int i, float2* turn) const {
    const double pos = a.c.positions_f32 ? (double)__uint_as_float(position) : (double)(int32_t)position;
    const double turns = pos * (double)freq * 0.15915494309189533577;  // (1 / 2 pi)
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    turn[i] = float2{cs, sn};
  }
};
template <bool EARLY>
struct HeadAngles {
  static constexpr int kMost = kHeadPairs / kHeadThreads;
  HeadAngle each[EARLY ? kMost : 1];
  __device__ __forceinline__ bool early(const HeadArgs& a, int n_tokens) const { return EARLY && n_tokens * a.pairs <= kHeadPairs; }
  __device__ __forceinline__ void load(const HeadArgs& a, int64_t t0, int n_tokens) {
    if (a.pairs == 0 || !early(a, n_tokens)) return;
#pragma unroll
    for (int k = 0; k < kMost; ++k) {
      const int i = k * kHeadThreads + threadIdx.x;
      if (i < n_tokens * a.pairs) each[k].load(a, t0, i, 1.f / (float)a.pairs);
    }
  }
  __device__ __forceinline__ void store(const HeadArgs& a, int64_t t0, int n_tokens, float2* turn) {
    if (early(a, n_tokens)) {
#pragma unroll
      for (int k = 0; k < (EARLY ? kMost : 1); ++k) {
        const int i = k * kHeadThreads + threadIdx.x;
        if (i < n_tokens * a.pairs) each[k].store(a, i, turn);
      }
    } else {
#pragma unroll 1
      for (int i = threadIdx.x; i < n_tokens * a.pairs; i += kHeadThreads) {
        each[0].load(a, t0, i, 1.f / (float)a.pairs);
        each[0].store(a, i, turn);
      }
    }
  }
};

// c = x (- mean) and 1 / sqrt(mean(c^2) + eps) of a head; elements past it stay zero.
template <int LANES, bool WHOLE>
__device__ __forceinline__ float head_stats(float (&u)[8], float (&v)[8], const HeadPiece& p, bool centred, float inv, float eps) {
  if (centred) {
    float first = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) first += u[e] + v[e];
    first = head_sum<LANES>(first) * inv;
    float off = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = (WHOLE ? 0 : e) < p.n[0] ? u[e] - first : 0.f;
      v[e] = (WHOLE ? 0 : e) < p.n[1] ? v[e] - first : 0.f;
      off += u[e] + v[e];
    }
    off = head_sum<LANES>(off) * inv;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if ((WHOLE ? 0 : e) < p.n[0]) u[e] -= off;
      if ((WHOLE ? 0 : e) < p.n[1]) v[e] -= off;
    }
  }
  float sq = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sq = fmaf(u[e], u[e], fmaf(v[e], v[e], sq));
  return rsqrtf(head_sum<LANES>(sq) * inv + eps);
}

__device__ __forceinline__ void head_weight(const HeadArgs& a, int set, const HeadPiece& p, float (&wu)[8], float (&wv)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) wu[e] = wv[e] = 1.f;
  if (a.c.w == nullptr) return;
  HeadRaw<true, false> r;
  r.load(a.c.w, (int64_t)set * a.c.D, p);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    wu[e] = r.r[0][e];
    wv[e] = r.r[1][e];
  }
}

template <bool XF32, bool INTERLEAVED, int LANES, bool WHOLE>
__global__ void __launch_bounds__(kHeadThreads) head_norm_kernel(const HeadArgs a) {
  __shared__ __attribute__((aligned(16))) float2 turn[kHeadPairs];
  constexpr int GROUPS = kHeadThreads / LANES;
  const HeadNormCall& c = a.c;
  int64_t block = flat_lane_256() / kHeadThreads;
  const int which = block >= a.set[0].blocks;
  if (which) block -= a.set[0].blocks;
  const HeadSet& set = a.set[which];
  if (block >= set.blocks) return;
  const int splits = set.splits, count = set.count;
  const int64_t t0 = block / splits * set.tokens;
  const int n_tokens = (int)(c.T - t0 < set.tokens ? c.T - t0 : set.tokens);
  const HeadPiece p = head_piece<INTERLEAVED>(a, threadIdx.x % LANES);
  const float inv = 1.f / (float)c.D, by_count = 1.f / (float)count;
  const int units = n_tokens * count, step = GROUPS * splits;
  int i = (int)(block % splits) * GROUPS + threadIdx.x / LANES;
  HeadRaw<XF32, WHOLE> in;
  in.clear();
  const int64_t x_run = t0 * c.x_token, y_run = t0 * c.y_token;
  auto fetch = [&](int at) {
    if (at < units) in.load(c.X, HeadUnit(set, at, by_count).at(x_run, (int)c.x_token, (int)c.x_head), p);
  };
  HeadAngles<true> angles;
  angles.load(a, t0, n_tokens);
  fetch(i);  // (on its way while the angles are computed; two units ahead took 19.5 us for 18.1 of 64 images)
  float wu[8], wv[8];
  head_weight(a, which, p, wu, wv);
  angles.store(a, t0, n_tokens, turn);
  __syncthreads();
  for (; i < units; i += step) {
    const HeadUnit unit(set, i, by_count);
    float u[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = in.r[0][e];
      v[e] = in.r[1][e];
    }
    fetch(i + step);
    const float rstd = head_stats<LANES, WHOLE>(u, v, p, c.centred, inv, c.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = u[e] * rstd * wu[e];
      v[e] = v[e] * rstd * wv[e];
    }
    head_turn<INTERLEAVED, WHOLE>(u, v, turn + unit.tok * a.pairs, p, false);
    head_store<WHOLE>(c.Y, unit.at(y_run, (int)c.y_token, (int)c.y_head), p, u, v, c.y_f32);
  }
}

// A block keeps its share of dw in registers over its runs of tokens; at the end the lane groups of a wave add theirs by exchanges and the
// waves in LDS, in an order that does not change, and a second launch adds the blocks'.
template <bool YF32, bool XF32, bool INTERLEAVED, int LANES, bool WHOLE>
__global__ void __launch_bounds__(kHeadThreads, 3) head_norm_grad_kernel(const HeadArgs a) {
  __shared__ __attribute__((aligned(16))) float2 turn[kGradPairs];
  __shared__ float totals[kHeadThreads / 64][kHeadMost];
  constexpr int GROUPS = kHeadThreads / LANES;
  const HeadNormCall& c = a.c;
  const int which = blockIdx.x >= a.set[0].blocks;
  const HeadSet& set = a.set[which];
  const int count = set.count;
  const HeadPiece p = head_piece<INTERLEAVED>(a, threadIdx.x % LANES);
  const float inv = 1.f / (float)c.D, by_count = 1.f / (float)count;
  float wu[8], wv[8], dw[2][8];
  head_weight(a, which, p, wu, wv);
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[0][e] = dw[1][e] = 0.f;
  HeadRaw<XF32, WHOLE> x_in;
  HeadRaw<YF32, WHOLE> y_in;
  x_in.clear();
  y_in.clear();
  for (int64_t t0 = (blockIdx.x - (which ? a.set[0].blocks : 0)) * set.tokens; t0 < c.T; t0 += set.blocks * set.tokens) {
    const int n_tokens = (int)(c.T - t0 < set.tokens ? c.T - t0 : set.tokens), units = n_tokens * count;
    const int64_t x_run = t0 * c.x_token, dy_run = t0 * c.dy_token, y_run = t0 * c.y_token;
    auto fetch = [&](int at) {
      if (at >= units) return;
      const HeadUnit unit(set, at, by_count);
      x_in.load(c.X, unit.at(x_run, (int)c.x_token, (int)c.x_head), p);
      y_in.load(c.dY, unit.at(dy_run, (int)c.dy_token, (int)c.dy_head), p);
    };
    int i = threadIdx.x / LANES;
    HeadAngles<!XF32 && !YF32> angles;
    angles.load(a, t0, n_tokens);
    fetch(i);
    __syncthreads();  // (the last run's angles have been read)
    angles.store(a, t0, n_tokens, turn);
    __syncthreads();
    for (; i < units; i += GROUPS) {
      const HeadUnit unit(set, i, by_count);
      float u[8], v[8], du[8], dv[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = x_in.r[0][e];
        v[e] = x_in.r[1][e];
        du[e] = y_in.r[0][e];
        dv[e] = y_in.r[1][e];
      }
      fetch(i + GROUPS);
      const float rstd = head_stats<LANES, WHOLE>(u, v, p, c.centred, inv, c.eps);
      head_turn<INTERLEAVED, WHOLE>(du, dv, turn + unit.tok * a.pairs, p, true);
      float sum_g = 0.f, sum_gn = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // (elements past the head: n and d are zero)
        u[e] *= rstd;
        v[e] *= rstd;
        dw[0][e] = fmaf(du[e], u[e], dw[0][e]);
        dw[1][e] = fmaf(dv[e], v[e], dw[1][e]);
        du[e] *= wu[e];
        dv[e] *= wv[e];
        sum_g += du[e] + dv[e];
        sum_gn = fmaf(du[e], u[e], fmaf(dv[e], v[e], sum_gn));
      }
      sum_gn = head_sum<LANES>(sum_gn) * inv;
      sum_g = c.centred ? head_sum<LANES>(sum_g) * inv : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        du[e] = rstd * (du[e] - sum_g - u[e] * sum_gn);
        dv[e] = rstd * (dv[e] - sum_g - v[e] * sum_gn);
      }
      head_store<WHOLE>(c.Y, unit.at(y_run, (int)c.y_token, (int)c.y_head), p, du, dv, c.y_f32);
    }
  }
  if (a.partial == nullptr) return;
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int m = LANES; m < 64; m <<= 1) dw[i / 8][i % 8] += __shfl_xor(dw[i / 8][i % 8], m, 64);
  if ((threadIdx.x & 63) < LANES) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i % 8 < p.n[i / 8]) totals[wave][p.at[i / 8] + i % 8] = dw[i / 8][i % 8];
  }
  __syncthreads();
  float* out = a.partial + (int64_t)blockIdx.x * c.D;
  for (int d = threadIdx.x; d < (int)c.D; d += kHeadThreads) out[d] = (totals[0][d] + totals[1][d]) + (totals[2][d] + totals[3][d]);
}

// The blocks' sums in order: 16 columns of a set to a block, the rows shared by 64 lanes per column, then a tree over the 64.
constexpr int kHeadSumCols = 16, kHeadSumRows = 64;
__global__ void __launch_bounds__(kHeadSumCols * kHeadSumRows) head_norm_sum_kernel(const HeadArgs a) {
  __shared__ float part[kHeadSumRows][kHeadSumCols + 1];
  const int col = threadIdx.x % kHeadSumCols, r = threadIdx.x / kHeadSumCols, cols = (int)a.c.D;
  const int at = blockIdx.x * kHeadSumCols + col, set = blockIdx.y, blocks = (int)a.set[set].blocks;
  const float* partial = a.partial + (set ? a.set[0].blocks * cols : 0);
  float v = 0.f;
  if (at < cols) {
#pragma unroll 8
    for (int k = r; k < blocks; k += kHeadSumRows) v += partial[(int64_t)k * cols + at];
  }
  part[r][col] = v;
  __syncthreads();
  for (int half = kHeadSumRows / 2; half > 0; half >>= 1) {
    if (r < half) part[r][col] += part[r + half][col];
    __syncthreads();
  }
  if (r == 0 && at < cols) a.c.dw[(int64_t)set * cols + at] = part[0][col];
}

// Lanes that hold a head, 16 elements each.
int head_lanes(int64_t D, int64_t R) {
  const int64_t pieces = (R / 2 + 7) / 8 + (D - R + 15) / 16;
  return pieces <= 4 ? 4 : pieces <= 8 ? 8 : pieces <= 16 ? 16 : 64;  // (at most 34 pieces)
}
// Whether all runs of eight elements are whole.
bool head_whole(const HeadNormCall& c) { return (c.interleaved ? c.R : c.R / 2) % 8 == 0 && (c.D - c.R) % 8 == 0; }
template <int N> struct Lanes { static constexpr int value = N; };
template <class F>
void with_lanes(int lanes, F&& f) {
  if (lanes == 4) f(Lanes<4>{});
  else if (lanes == 8) f(Lanes<8>{});
  else if (lanes == 16) f(Lanes<16>{});
  else f(Lanes<64>{});
}
template <class F>
void with_flag(bool on, F&& f) {
  if (on) f(std::true_type{});
  else f(std::false_type{});
}

// How a set's heads go to blocks: kHeadTurns of them to each lane group of a block at a time (64 images 17.0 us with three, 17.4 with four
// and six), as far as its tokens' cosines fit and blocks are left for the chip.
constexpr int64_t kHeadTurns = 3, kHeadBlocks = 1024, kHeadGradBlocks = 768;
HeadSet head_set(int64_t T, int first, int count, int lanes, int64_t pairs) {
  HeadSet s = {first, count, 1, 1, 0};
  if (count == 0) return s;
  const int64_t groups = kHeadThreads / lanes;
  int64_t tokens = kHeadTurns * groups / count;
  if (pairs > 0 && tokens > kHeadPairs / pairs) tokens = kHeadPairs / pairs;
  const int64_t spread = (T * count + kHeadBlocks * groups - 1) / (kHeadBlocks * groups) * groups / count;  // (whole turns of the groups)
  if (tokens > spread) tokens = spread;
  s.tokens = (int)(tokens > 1 ? tokens : 1);
  s.blocks = (T + s.tokens - 1) / s.tokens;
  return s;
}
HeadArgs head_args(int64_t T, int64_t H, int64_t heads, int64_t D, int64_t R) {
  HeadArgs a = {};
  a.pairs = (int)(R / 2);
  a.rotate = (a.pairs + 7) / 8;
  const int lanes = head_lanes(D, R);
  a.set[0] = head_set(T, 0, (int)heads, lanes, a.pairs);
  a.set[1] = head_set(T, (int)heads, (int)(H - heads), lanes, a.pairs);
  return a;
}
// Blocks of the backward pass, each with a row of sums: no more than the chip holds, by the sets' heads.
HeadArgs head_grad_args(int64_t T, int64_t H, int64_t heads, int64_t D, int64_t R) {
  HeadArgs a = head_args(T, H, heads, D, R);
  for (HeadSet& s : a.set) {
    const int64_t most = (kHeadGradBlocks * s.count + H - 1) / H;
    if (s.blocks <= most) continue;
    // tokens of a run: their cosines fit, and its heads are no more than head_quotient counts
    const int64_t fit = a.pairs > 0 ? kGradPairs / a.pairs : kGradPairs, counted = kHeadMostUnits / s.count, room = fit < counted ? fit : counted;
    const int64_t runs = (T + most * room - 1) / (most * room);  // of each block, all as long
    s.tokens = (int)((T + most * runs - 1) / (most * runs));
    s.blocks = (T + s.tokens * runs - 1) / (s.tokens * runs);
  }
  return a;
}

}  // namespace

hipError_t launch_head_norm(const HeadNormCall& c, hipStream_t s) {
  const int lanes = head_lanes(c.D, c.R);
  HeadArgs a = head_args(c.T, c.H, c.heads, c.D, c.R);
  a.c = c;
  const int64_t groups = kHeadThreads / lanes;
  for (HeadSet& set : a.set)
    if (set.tokens == 1 && set.blocks < kHeadBlocks) {  // few tokens: a head to a lane group
      const int64_t splits = (set.count + groups - 1) / groups;
      set.splits = (int)(splits < 16 ? splits : 16);
      set.blocks *= set.splits;
    }
  const dim3 grid = flat_grid_256((a.set[0].blocks + a.set[1].blocks) * kHeadThreads);
  with_lanes(lanes, [&](auto l) {
    with_flag(c.interleaved, [&](auto i) {
      with_flag(c.x_f32, [&](auto x) {
        with_flag(head_whole(c), [&](auto w) {
          head_norm_kernel<decltype(x)::value, decltype(i)::value, decltype(l)::value, decltype(w)::value><<<grid, kHeadThreads, 0, s>>>(a);
        });
      });
    });
  });
  return hipGetLastError();
}

size_t head_norm_grad_workspace_bytes(int64_t T, int64_t H, int64_t heads, int64_t D, int64_t R) {
  const HeadArgs a = head_grad_args(T, H, heads, D, R);
  return (size_t)(a.set[0].blocks + a.set[1].blocks) * (size_t)D * sizeof(float);
}

hipError_t launch_head_norm_grad(const HeadNormCall& c, hipStream_t s) {
  const int lanes = head_lanes(c.D, c.R);
  HeadArgs a = head_grad_args(c.T, c.H, c.heads, c.D, c.R);
  a.c = c;
  const unsigned blocks = (unsigned)(a.set[0].blocks + a.set[1].blocks);
  if (c.dw != nullptr) a.partial = blocks > 1 ? static_cast<float*>(c.workspace) : c.dw;
  with_lanes(lanes, [&](auto l) {
    with_flag(c.interleaved, [&](auto i) {
      with_flag(c.x_f32, [&](auto x) {
        with_flag(c.dy_f32, [&](auto y) {
          with_flag(head_whole(c), [&](auto w) {
            head_norm_grad_kernel<decltype(y)::value, decltype(x)::value, decltype(i)::value, decltype(l)::value, decltype(w)::value>
                <<<dim3(blocks), kHeadThreads, 0, s>>>(a);
          });
        });
      });
    });
  });
  if (c.dw != nullptr && blocks > 1) {
    const dim3 grid((unsigned)((c.D + kHeadSumCols - 1) / kHeadSumCols), c.heads < c.H ? 2 : 1);
    head_norm_sum_kernel<<<grid, kHeadSumCols * kHeadSumRows, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace nm
