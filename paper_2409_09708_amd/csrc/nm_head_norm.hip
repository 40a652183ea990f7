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
// Bound by memory: 10 flops per element forward, 18 backward, for 4 to 12 bytes.
#include "nm_device.h"
#include "nm_launch.h"
#include "nm_rows.h"

#include <type_traits>

namespace nm {

namespace {

constexpr int kHeadThreads = 256;  // (flat_grid_256)
constexpr int kHeadPairs = 512;    // cosines and sines that a block keeps: 4 KiB
constexpr int kHeadMost = 512;     // elements of a head

struct HeadArgs {
  HeadNormCall c;
  int tokens;       // per block and turn
  int splits;       // blocks that share a token's heads (forward, few tokens)
  int pairs;        // R / 2
  int rotate;       // pieces of a head with pairs that are turned
  int64_t groups;   // of tokens
  float* partial;   // backward: [blocks][sets][D], or NULL: one block, which writes dw itself
};

// i / d for 0 <= i < 2^21, from 1 / d: the quotient is at least 0.5 / d away from the next integer, the product off by less
__device__ __forceinline__ int head_quotient(int i, float inverse) { return (int)(((float)i + 0.5f) * inverse); }

// Sum over the LANES lanes of a head.
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int m = 1; m < LANES; m <<= 1) v += __shfl_xor(v, m, 64);
  return v;
}

// The two runs of eight elements that lane k of a head holds: where they begin, how many there are (<= 0: none), and the first of its
// pairs in the table of a token's turns.
struct HeadPiece {
  int at[2], n[2], pair;
  bool turned;
};
template <bool INTERLEAVED>
__device__ __forceinline__ HeadPiece head_piece(const HeadArgs& a, int k) {
  HeadPiece p;
  const int D = (int)a.c.D;
  p.turned = k < a.rotate;
  p.pair = k * 8;
  if (!INTERLEAVED && p.turned) {
    p.at[0] = k * 8;
    p.at[1] = a.pairs + k * 8;
    p.n[0] = p.n[1] = a.pairs - k * 8;
  } else {
    p.at[0] = p.turned ? k * 16 : 2 * a.pairs + (k - a.rotate) * 16;
    p.at[1] = p.at[0] + 8;
    p.n[0] = (p.turned ? 2 * a.pairs : D) - p.at[0];
    p.n[1] = p.n[0] - 8;
  }
  return p;
}

template <bool F32>
struct HeadRaw {
  Raw8<F32> r[2];
  __device__ __forceinline__ void load(const void* base, int64_t row, const HeadPiece& p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) r[i].load(base, row + p.at[i], p.n[i]);  // (n <= 0: zeros, nothing read)
  }
};

// The turn of a lane's pairs, back where `back`.
template <bool INTERLEAVED>
__device__ __forceinline__ void head_turn(float (&u)[8], float (&v)[8], const float2* w, const HeadPiece& p, bool back) {
  if (!p.turned) return;
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float* q = e < 4 ? u + 2 * e : v + 2 * e - 8;
      const float2 cs = 2 * e < p.n[0] ? w[e] : float2{1.f, 0.f};
      const float sn = back ? -cs.y : cs.y, x = q[0], y = q[1];
      q[0] = x * cs.x - y * sn;
      q[1] = y * cs.x + x * sn;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 cs = e < p.n[0] ? w[e] : float2{1.f, 0.f};
      const float sn = back ? -cs.y : cs.y, x = u[e], y = v[e];
      u[e] = x * cs.x - y * sn;
      v[e] = y * cs.x + x * sn;
    }
  }
}

// Cosines and sines of the pairs of n_tokens tokens from t0 on.
__device__ __forceinline__ void head_angles(const HeadArgs& a, int64_t t0, int n_tokens, float2* turn) {
  const HeadNormCall& c = a.c;
  if (a.pairs == 0) return;
  const float by_pairs = 1.f / (float)a.pairs;
  for (int i = threadIdx.x; i < n_tokens * a.pairs; i += kHeadThreads) {
    const int tok = head_quotient(i, by_pairs), pair = i - tok * a.pairs;
    int axis = 0;
#pragma unroll
    for (int x = 0; x < kMaxRotaryAxes - 1; ++x) axis += pair >= c.section_end[x] ? 1 : 0;
    const int64_t at = (t0 + tok) * c.axes + axis;
    const double pos = c.positions_f32 ? (double)static_cast<const float*>(c.positions)[at]
                                       : (double)static_cast<const int32_t*>(c.positions)[at];
    constexpr double kTurn = 6.283185307179586476925;
    const double angle = pos * (double)c.freqs[pair];
    float sn, cs;
    sincosf((float)(angle - kTurn * rint(angle * (1.0 / kTurn))), &sn, &cs);
    turn[i] = float2{cs, sn};
  }
}

// c = x (- mean) and 1 / sqrt(mean(c^2) + eps) of a head; elements past it stay zero.
template <int LANES>
__device__ __forceinline__ float head_stats(float (&u)[8], float (&v)[8], const HeadPiece& p, bool centred, float inv, float eps) {
  if (centred) {
    float first = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) first += u[e] + v[e];
    first = head_sum<LANES>(first) * inv;
    float off = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = e < p.n[0] ? u[e] - first : 0.f;
      v[e] = e < p.n[1] ? v[e] - first : 0.f;
      off += u[e] + v[e];
    }
    off = head_sum<LANES>(off) * inv;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e < p.n[0]) u[e] -= off;
      if (e < p.n[1]) v[e] -= off;
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
  HeadRaw<true> r;
  r.load(a.c.w, (int64_t)set * a.c.D, p);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    wu[e] = r.r[0][e];
    wv[e] = r.r[1][e];
  }
}

template <bool XF32, bool INTERLEAVED, int LANES>
__global__ void __launch_bounds__(kHeadThreads) head_norm_kernel(const HeadArgs a) {
  __shared__ __attribute__((aligned(16))) float2 turn[kHeadPairs];
  constexpr int GROUPS = kHeadThreads / LANES;
  const HeadNormCall& c = a.c;
  const int64_t block = flat_lane_256() / kHeadThreads;
  const int64_t t0 = block / a.splits * a.tokens;
  if (t0 >= c.T) return;
  const int split = (int)(block % a.splits);
  const int n_tokens = (int)(c.T - t0 < a.tokens ? c.T - t0 : a.tokens);
  const int k = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const HeadPiece p = head_piece<INTERLEAVED>(a, k);
  const float inv = 1.f / (float)c.D;
  bool ready = false;
  for (int set = 0; set < 2; ++set) {
    const int first = set ? (int)c.heads : 0, count = set ? (int)(c.H - c.heads) : (int)c.heads;  // the set's heads
    if (count == 0) continue;
    const float by_count = 1.f / (float)count;
    const int units = n_tokens * count, step = GROUPS * a.splits;
    HeadRaw<XF32> in;
    auto fetch = [&](int i) {
      if (i >= units) return;
      const int tok = head_quotient(i, by_count);
      in.load(c.X, (t0 + tok) * c.x_token + (int64_t)(first + i - tok * count) * c.x_head, p);
    };
    fetch(split * GROUPS + group);  // (on its way while the angles are computed)
    float wu[8], wv[8];
    head_weight(a, set, p, wu, wv);
    if (!ready) {
      head_angles(a, t0, n_tokens, turn);
      __syncthreads();
      ready = true;
    }
    for (int i = split * GROUPS + group; i < units; i += step) {
      const int tok = head_quotient(i, by_count);
      const int64_t y = (t0 + tok) * c.y_token + (int64_t)(first + i - tok * count) * c.y_head;
      float u[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = in.r[0][e];
        v[e] = in.r[1][e];
      }
      fetch(i + step);
      const float rstd = head_stats<LANES>(u, v, p, c.centred, inv, c.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = u[e] * rstd * wu[e];
        v[e] = v[e] * rstd * wv[e];
      }
      head_turn<INTERLEAVED>(u, v, turn + tok * a.pairs + p.pair, p, false);
      if (p.n[0] > 0) store8(c.Y, y + p.at[0], p.n[0], u, !c.y_f32);
      if (p.n[1] > 0) store8(c.Y, y + p.at[1], p.n[1], v, !c.y_f32);
    }
  }
}

// Blocks walk over groups of tokens and keep their shares of dw in registers; at the end the lane groups of a wave add theirs by
// exchanges and the waves in LDS, in an order that does not change, and a second launch adds the blocks'.
template <bool YF32, bool XF32, bool INTERLEAVED, int LANES>
__global__ void __launch_bounds__(kHeadThreads) head_norm_grad_kernel(const HeadArgs a) {
  __shared__ __attribute__((aligned(16))) float2 turn[kHeadPairs];
  __shared__ float totals[kHeadThreads / 64][kHeadMost];
  constexpr int GROUPS = kHeadThreads / LANES;
  const HeadNormCall& c = a.c;
  const int k = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const HeadPiece p = head_piece<INTERLEAVED>(a, k);
  const float inv = 1.f / (float)c.D;
  float dw[2][2][8];
#pragma unroll
  for (int i = 0; i < 32; ++i) dw[i / 16][i / 8 % 2][i % 8] = 0.f;
  for (int64_t g0 = blockIdx.x; g0 < a.groups; g0 += gridDim.x) {
    const int64_t t0 = g0 * a.tokens;
    const int n_tokens = (int)(c.T - t0 < a.tokens ? c.T - t0 : a.tokens);
    __syncthreads();  // (the last group's angles have been read)
    head_angles(a, t0, n_tokens, turn);
    __syncthreads();
#pragma unroll
    for (int set = 0; set < 2; ++set) {
      const int first = set ? (int)c.heads : 0, count = set ? (int)(c.H - c.heads) : (int)c.heads;
      if (count == 0) continue;
      const float by_count = 1.f / (float)count;
      const int units = n_tokens * count;
      HeadRaw<XF32> x_in;
      HeadRaw<YF32> y_in;
      auto fetch = [&](int i) {
        if (i >= units) return;
        const int tok = head_quotient(i, by_count);
        const int64_t head = first + i - tok * count;
        x_in.load(c.X, (t0 + tok) * c.x_token + head * c.x_head, p);
        y_in.load(c.dY, (t0 + tok) * c.dy_token + head * c.dy_head, p);
      };
      fetch(group);
      float wu[8], wv[8];
      head_weight(a, set, p, wu, wv);
      for (int i = group; i < units; i += GROUPS) {
        const int tok = head_quotient(i, by_count);
        const int64_t out = (t0 + tok) * c.y_token + (int64_t)(first + i - tok * count) * c.y_head;
        float u[8], v[8], du[8], dv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] = x_in.r[0][e];
          v[e] = x_in.r[1][e];
          du[e] = y_in.r[0][e];
          dv[e] = y_in.r[1][e];
        }
        fetch(i + GROUPS);
        const float rstd = head_stats<LANES>(u, v, p, c.centred, inv, c.eps);
        head_turn<INTERLEAVED>(du, dv, turn + tok * a.pairs + p.pair, p, true);
        float sum_g = 0.f, sum_gn = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {  // (elements past the head: n and d are zero)
          u[e] *= rstd;
          v[e] *= rstd;
          dw[set][0][e] = fmaf(du[e], u[e], dw[set][0][e]);
          dw[set][1][e] = fmaf(dv[e], v[e], dw[set][1][e]);
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
        if (p.n[0] > 0) store8(c.Y, out + p.at[0], p.n[0], du, !c.y_f32);
        if (p.n[1] > 0) store8(c.Y, out + p.at[1], p.n[1], dv, !c.y_f32);
      }
    }
  }
  if (c.dw == nullptr) return;
  const int sets = c.heads < c.H ? 2 : 1, wave = threadIdx.x >> 6;
#pragma unroll
  for (int set = 0; set < 2; ++set) {
    if (set >= sets) break;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int m = LANES; m < 64; m <<= 1) dw[set][i / 8][i % 8] += __shfl_xor(dw[set][i / 8][i % 8], m, 64);
    if ((threadIdx.x & 63) < LANES) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i % 8 < p.n[i / 8]) totals[wave][p.at[i / 8] + i % 8] = dw[set][i / 8][i % 8];
    }
    __syncthreads();
    float* out = (a.partial ? a.partial + (int64_t)blockIdx.x * sets * c.D : c.dw) + set * c.D;
    for (int d = threadIdx.x; d < (int)c.D; d += kHeadThreads) out[d] = (totals[0][d] + totals[1][d]) + (totals[2][d] + totals[3][d]);
    __syncthreads();
  }
}

// The blocks' sums in order: 16 columns to a block, the rows shared by 64 lanes per column, then a tree over the 64.
constexpr int kHeadSumCols = 16, kHeadSumRows = 64;
__global__ void __launch_bounds__(kHeadSumCols * kHeadSumRows) head_norm_sum_kernel(const float* partial, int blocks, int cols, float* dw) {
  __shared__ float part[kHeadSumRows][kHeadSumCols + 1];
  const int col = threadIdx.x % kHeadSumCols, r = threadIdx.x / kHeadSumCols;
  const int at = blockIdx.x * kHeadSumCols + col;
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
  if (r == 0 && at < cols) dw[at] = part[0][col];
}

// Lanes that hold a head, 16 elements each.
int head_lanes(int64_t D, int64_t R) {
  const int64_t pieces = (R / 2 + 7) / 8 + (D - R + 15) / 16;
  return pieces <= 4 ? 4 : pieces <= 8 ? 8 : pieces <= 16 ? 16 : 64;  // (at most 34 pieces)
}
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

// Tokens that a block takes at a time: two heads for each of its lane groups, as far as their cosines fit and blocks are left for the chip.
int head_tokens(int64_t T, int64_t H, int lanes, int64_t pairs) {
  const int64_t groups = kHeadThreads / lanes;
  int64_t tokens = (2 * groups + H - 1) / H;
  if (pairs > 0 && tokens > kHeadPairs / pairs) tokens = kHeadPairs / pairs;
  const int64_t spread = (T + 1023) / 1024;
  return (int)(tokens < spread ? tokens : spread);
}
constexpr int64_t kHeadGradBlocks = 1024;  // which keep sums of dw
int64_t head_grad_blocks(int64_t T, int64_t H, int64_t D, int64_t R) {
  const int64_t tokens = head_tokens(T, H, head_lanes(D, R), R / 2), groups = (T + tokens - 1) / tokens;
  return groups < kHeadGradBlocks ? groups : kHeadGradBlocks;
}
HeadArgs head_args(const HeadNormCall& c, int lanes) {
  HeadArgs a = {};
  a.c = c;
  a.pairs = (int)(c.R / 2);
  a.rotate = (a.pairs + 7) / 8;
  a.tokens = head_tokens(c.T, c.H, lanes, a.pairs);
  a.groups = (c.T + a.tokens - 1) / a.tokens;
  a.splits = 1;
  return a;
}

}  // namespace

hipError_t launch_head_norm(const HeadNormCall& c, hipStream_t s) {
  const int lanes = head_lanes(c.D, c.R);
  HeadArgs a = head_args(c, lanes);
  const int64_t groups = kHeadThreads / lanes, most = (c.H + groups - 1) / groups;
  if (a.tokens == 1 && a.groups < 1024) a.splits = (int)(most < 16 ? most : 16);
  const dim3 grid = flat_grid_256(a.groups * a.splits * kHeadThreads);
  with_lanes(lanes, [&](auto l) {
    with_flag(c.interleaved, [&](auto i) {
      with_flag(c.x_f32, [&](auto x) {
        head_norm_kernel<decltype(x)::value, decltype(i)::value, decltype(l)::value><<<grid, kHeadThreads, 0, s>>>(a);
      });
    });
  });
  return hipGetLastError();
}

size_t head_norm_grad_workspace_bytes(int64_t T, int64_t H, int64_t D, int64_t R, int sets) {
  const int64_t blocks = head_grad_blocks(T, H, D, R);
  return blocks > 1 ? (size_t)blocks * sets * (size_t)D * sizeof(float) : 0;
}

hipError_t launch_head_norm_grad(const HeadNormCall& c, hipStream_t s) {
  const int lanes = head_lanes(c.D, c.R);
  HeadArgs a = head_args(c, lanes);
  const int64_t blocks = head_grad_blocks(c.T, c.H, c.D, c.R);
  a.partial = c.dw != nullptr && blocks > 1 ? static_cast<float*>(c.workspace) : nullptr;
  with_lanes(lanes, [&](auto l) {
    with_flag(c.interleaved, [&](auto i) {
      with_flag(c.x_f32, [&](auto x) {
        with_flag(c.dy_f32, [&](auto y) {
          head_norm_grad_kernel<decltype(y)::value, decltype(x)::value, decltype(i)::value, decltype(l)::value>
              <<<dim3((unsigned)blocks), kHeadThreads, 0, s>>>(a);
        });
      });
    });
  });
  if (a.partial != nullptr) {
    const int cols = (int)(c.heads < c.H ? 2 * c.D : c.D);
    head_norm_sum_kernel<<<dim3((unsigned)((cols + kHeadSumCols - 1) / kHeadSumCols)), kHeadSumCols * kHeadSumRows, 0, s>>>(
        a.partial, (int)blocks, cols, c.dw);
  }
  return hipGetLastError();
}

}  // namespace nm
