// Layer norm of rows, optionally of the sum of two inputs, and its backward pass.
//
//   s = x (+ r),  mu = mean(s),  rstd = 1 / sqrt(mean((s - mu)^2) + eps),  y = (s - mu) rstd w + b
//
// and with n = (s - mu) rstd, g = dy w, for each row
//
//   ds = rstd (g - mean(g) - n mean(g n)) (+ the gradient that reaches s by its other use),
//   dw = sum over rows of dy n,  db = sum over rows of dy.
//
// All sums, statistics and the normalised values are 32-bit floats; a value is rounded once, when it is stored as
// bfloat16.  The mean m of one sum is off by the roundings of that sum, for rows with a large common offset by more than their
// spread.  So with the squares of the differences to it goes their sum (the row lies in registers: no memory traffic):
//
//   e = mean(s - m),  mu = m + e,  variance = mean((s - m)^2) - e^2,  y = ((s - m) - e) rstd w + b
//
// where s - m is exact once m is close.  (Rows of 768 times 10000.1, eps 1e-6: y was -0.7, and is 0 to 10^-5.)
//
// Bound by memory at any width: 8 flops per element forward, 14 backward, against 4 to 16 bytes.  A row is held by
// LANES lanes (16 for the narrowest, a wave, or a block of four waves), 8 consecutive elements (one 16-byte piece of
// bfloat16) per lane and step, so that a wave's load covers whole 128-byte lines, at any width and alignment.  Rows above
// 8192 elements are read again for each sum.
// Measured: 200704 x 128, float in with the sum kept, 361 MB in 65 us, 5.6 TB/s, what a large copy reaches; backward 50432 x 768 of
// bfloat16, 310 MB in 60 us and 5 for the sums of dw and db; 4099 x 5003 of float, rows 5008 apart, 246 MB in 67 and 8 (a row of a block
// pays a barrier for each of its two sums); one row 3 us, a launch.  The second sum of the forward pass costs 8192 x 2048 of bfloat16 in
// and out 16.0 us where 15.3 were without; elsewhere at most one part in a hundred.
#include "nm_device.h"
#include "nm_launch.h"
#include "nm_rows.h"

namespace nm {

namespace {

struct NormArgs {
  const void* X;
  const void* R;  // nullable
  const float* w;
  const float* b;
  void* Y;
  void* S;       // nullable
  float* stats;  // nullable: (mean, rstd) per row
  int64_t T, C, ldx, ldr, ldy, lds;
  float eps;
  int y_bf16;
};

struct NormGradArgs {
  const void* dY;
  const void* S;
  const float* stats;
  const float* w;   // nullable
  const void* dS;   // nullable, type of dY
  void* dX;
  float* dw;        // nullable, with db
  float* db;
  float* partial;   // [blocks][2][C], or NULL: one block, which writes dw and db itself
  int64_t T, C, lddy, lds, ldds, lddx;
  int dx_bf16;
};

constexpr int kNormThreads = 256;  // (flat_grid_256)

// Sum over the LANES lanes of a row (every lane receives it).  `slot` is LDS of at least 4 floats, used by rows of a
// whole block only; consecutive calls need different slots.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* slot) {
#pragma unroll
  for (int m = 1; m < (LANES < 64 ? LANES : 64); m <<= 1) v += __shfl_xor(v, m, 64);
  if constexpr (LANES > 64) {
    static_assert(LANES == kNormThreads, "a row of a block");
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (slot[0] + slot[1]) + (slot[2] + slot[3]);
  }
  return v;
}

// Two sums at once; `slots` of at least 8 floats.
template <int LANES>
__device__ __forceinline__ void row_sums(float& u, float& v, float* slots) {
#pragma unroll
  for (int m = 1; m < (LANES < 64 ? LANES : 64); m <<= 1) {
    u += __shfl_xor(u, m, 64);
    v += __shfl_xor(v, m, 64);
  }
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) *reinterpret_cast<float2*>(slots + 2 * (threadIdx.x >> 6)) = float2{u, v};
    __syncthreads();
    u = (slots[0] + slots[2]) + (slots[4] + slots[6]);
    v = (slots[1] + slots[3]) + (slots[5] + slots[7]);
  }
}

// What the differences to a first mean, their sum and that of their squares, say of a row of 1 / inv elements.
struct RowStats {
  float e, mean, rstd;
};
__device__ __forceinline__ RowStats row_stats(float first, float sum, float sq, float inv, float eps) {
  const float e = sum * inv, var = sq * inv - e * e;
  return {e, first + e, rsqrtf((var < 0.f ? 0.f : var) + eps)};  // (a NaN stays one)
}

template <bool XF32, int LANES, int CH>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const NormArgs a) {
  __shared__ __attribute__((aligned(8))) float slots[12];
  const int lane = threadIdx.x % LANES;
  const int64_t row = flat_lane_256() / LANES;
  const bool live = row < a.T;
  const int C = (int)a.C;
  float x[CH][8];
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * LANES + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[c][e] = 0.f;
    if (live && at < C) {
      Raw8<XF32> raw;
      raw.load(a.X, row * a.ldx + at, C - at);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = raw[e];
      if (a.R != nullptr) {
        raw.load(a.R, row * a.ldr + at, C - at);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] += raw[e];
        if (a.S != nullptr) store8(a.S, row * a.lds + at, C - at, x[c], !XF32);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[c][e];
    }
  }
  const float inv = 1.f / (float)C, first = row_sum<LANES>(sum, slots + 8) / (float)C;
  float off = 0.f, sq = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int n = C - (c * LANES + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[c][e] -= first;
      if (e < n) {
        off += x[c][e];
        sq = fmaf(x[c][e], x[c][e], sq);
      }
    }
  }
  row_sums<LANES>(off, sq, slots);
  const RowStats st = row_stats(first, off, sq, inv, a.eps);
  if (!live) return;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * LANES + lane) * 8;
    if (at < C) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (x[c][e] - st.e) * st.rstd;
      Raw8<true> p;
      if (a.w != nullptr) {
        p.load(a.w, at, C - at);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= p[e];
      }
      if (a.b != nullptr) {
        p.load(a.b, at, C - at);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += p[e];
      }
      store8(a.Y, row * a.ldy + at, C - at, y, a.y_bf16);
    }
  }
  if (a.stats != nullptr && lane == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = float2{st.mean, st.rstd};
}

// Rows of any length: one block each, read once for every sum.
template <bool XF32>
__global__ void __launch_bounds__(kNormThreads) norm_long_kernel(const NormArgs a) {
  __shared__ __attribute__((aligned(8))) float slots[12];
  const int64_t row = flat_lane_256() / kNormThreads;
  if (row >= a.T) return;
  auto value = [&](int64_t at) {
    const float x = load1<XF32>(a.X, row * a.ldx + at);
    return a.R == nullptr ? x : x + load1<XF32>(a.R, row * a.ldr + at);
  };
  float sum = 0.f;
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) sum += value(at);
  const float inv = 1.f / (float)a.C, first = row_sum<kNormThreads>(sum, slots + 8) / (float)a.C;
  float off = 0.f, sq = 0.f;
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) {
    const float d = value(at) - first;
    off += d;
    sq = fmaf(d, d, sq);
  }
  row_sums<kNormThreads>(off, sq, slots);
  const RowStats st = row_stats(first, off, sq, inv, a.eps);
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) {
    const float s = value(at);
    if (a.R != nullptr && a.S != nullptr) store1(a.S, row * a.lds + at, s, !XF32);
    store1(a.Y, row * a.ldy + at, fmaf((s - first - st.e) * st.rstd, a.w ? a.w[at] : 1.f, a.b ? a.b[at] : 0.f), a.y_bf16);
  }
  if (a.stats != nullptr && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = float2{st.mean, st.rstd};
}

// A block walks over rows, LANES lanes to each, and keeps its share of dw and db in registers; at the end the row groups of
// the block add theirs in LDS, and the blocks' sums are added in order by a second launch (norm_grad_sum_kernel): the result
// does not depend on scheduling.  A row's operands are loaded while the row before it is reduced.
template <bool YF32, bool SF32, int LANES, int CH>
__global__ void __launch_bounds__(kNormThreads) norm_grad_kernel(const NormGradArgs a) {
  __shared__ float slots[2][8];
  constexpr int ROWS = kNormThreads / LANES;
  constexpr int W = CH * LANES * 8;  // columns held, >= C
  constexpr bool ROOM = CH <= 2;     // registers enough to keep w, and to load dS ahead
  __shared__ float totals[ROWS > 1 ? 2 * W : 1];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int C = (int)a.C;
  const float inv = 1.f / (float)C;
  float dw[CH][8], db[CH][8], w[ROOM ? CH : 1][8];
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[c][e] = db[c][e] = 0.f;
  auto weight = [&](int c, float (&v)[8]) {
    const int at = (c * LANES + lane) * 8;
    Raw8<true> p;
    if (a.w != nullptr && at < C) p.load(a.w, at, C - at);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = a.w != nullptr && at < C ? p[e] : 1.f;
  };
  if constexpr (ROOM) {
#pragma unroll
    for (int c = 0; c < CH; ++c) weight(c, w[c]);
  }
  Raw8<SF32> s_in[CH];
  Raw8<YF32> g_in[CH], r_in[ROOM ? CH : 1];
  float2 st_in = {0.f, 0.f};
  const int64_t step = (int64_t)gridDim.x * ROWS;
  auto fetch = [&](int64_t row) {
    if (row >= a.T) return;
    st_in = *reinterpret_cast<const float2*>(a.stats + 2 * row);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LANES + lane) * 8;
      if (at < C) {
        s_in[c].load(a.S, row * a.lds + at, C - at);
        g_in[c].load(a.dY, row * a.lddy + at, C - at);
        if constexpr (ROOM)
          if (a.dS != nullptr) r_in[c].load(a.dS, row * a.ldds + at, C - at);
      }
    }
  };
  int turn = 0;
  int64_t first = (int64_t)blockIdx.x * ROWS;
  fetch(first + group);
  for (; first < a.T; first += step, turn ^= 1) {
    const int64_t row = first + group;
    const bool live = row < a.T;
    const float2 st = st_in;
    float n[CH][8], g[CH][8];
    Raw8<YF32> r[ROOM ? CH : 1];
    float sum_g = 0.f, sum_gn = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LANES + lane) * 8;
      if (live && at < C) {
        float wc[8];
        if constexpr (ROOM) {
          r[c] = r_in[c];
#pragma unroll
          for (int e = 0; e < 8; ++e) wc[e] = w[c][e];
        } else {
          weight(c, wc);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {  // (elements past the row: dY is zero, and so is all that they add)
          n[c][e] = (s_in[c][e] - st.x) * st.y;
          g[c][e] = g_in[c][e];
          dw[c][e] = fmaf(g[c][e], n[c][e], dw[c][e]);
          db[c][e] += g[c][e];
          g[c][e] *= wc[e];
          sum_g += g[c][e];
          sum_gn = fmaf(g[c][e], n[c][e], sum_gn);
        }
      }
    }
    fetch(row + step);
    sum_g = row_sum<LANES>(sum_g, slots[turn]) * inv;
    sum_gn = row_sum<LANES>(sum_gn, slots[turn] + 4) * inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LANES + lane) * 8;
      if (live && at < C) {
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = st.y * (g[c][e] - sum_g - n[c][e] * sum_gn);
        if (a.dS != nullptr) {
          Raw8<YF32> now;
          if constexpr (ROOM) now = r[c];
          else now.load(a.dS, row * a.ldds + at, C - at);
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] += now[e];
        }
        store8(a.dX, row * a.lddx + at, C - at, d, a.dx_bf16);
      }
    }
  }
  if (a.dw == nullptr) return;
  float* out_w = a.partial ? a.partial + (int64_t)blockIdx.x * 2 * C : a.dw;
  float* out_b = a.partial ? out_w + C : a.db;
  if constexpr (ROWS > 1) {
    for (int q = 0; q < ROWS; ++q) {  // one row group after another adds its share: an order that does not change
      if (group == q) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int i = (c * 8 + e) * LANES + lane;  // consecutive lanes on consecutive banks
            totals[i] = q ? totals[i] + dw[c][e] : dw[c][e];
            totals[W + i] = q ? totals[W + i] + db[c][e] : db[c][e];
          }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < W; i += kNormThreads) {
      const int l = i % LANES, ce = i / LANES;
      const int at = ((ce / 8) * LANES + l) * 8 + ce % 8;
      if (at < C) { out_w[at] = totals[i]; out_b[at] = totals[W + i]; }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LANES + lane) * 8;
      if (at < C) {
        store8(out_w, at, C - at, dw[c], false);
        store8(out_b, at, C - at, db[c], false);
      }
    }
  }
}

// dw and db from the blocks' sums: 32 columns per block, the rows of the partial sums shared by 32 lanes per column, each
// adding every 32nd in order, then a tree over the 32.
constexpr int kSumCols = 32, kSumRows = 32;
__global__ void __launch_bounds__(kSumCols * kSumRows) norm_grad_sum_kernel(const float* partial, int blocks, int64_t C,
                                                                            float* dw, float* db) {
  __shared__ float part[kSumRows][kSumCols + 1];
  const int col = threadIdx.x % kSumCols, r = threadIdx.x / kSumCols;
  const int64_t at = (int64_t)blockIdx.x * kSumCols + col;  // of the 2 C columns
  float v = 0.f;
  if (at < 2 * C) {
#pragma unroll 8
    for (int k = r; k < blocks; k += kSumRows) v += partial[(int64_t)k * 2 * C + at];
  }
  part[r][col] = v;
  __syncthreads();
  for (int half = kSumRows / 2; half > 0; half >>= 1) {
    if (r < half) part[r][col] += part[r + half][col];
    __syncthreads();
  }
  if (r == 0 && at < 2 * C) (at < C ? dw + at : db + (at - C))[0] = part[0][col];
}

// Rows of any length: the input's gradient, one block per row ...
template <bool YF32, bool SF32>
__global__ void __launch_bounds__(kNormThreads) norm_grad_long_kernel(const NormGradArgs a) {
  __shared__ float slots[8];
  const int64_t row = flat_lane_256() / kNormThreads;
  if (row >= a.T) return;
  const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
  auto value = [&](int64_t at, float* g) {
    const float d = load1<YF32>(a.dY, row * a.lddy + at);
    *g = a.w ? d * a.w[at] : d;
    return (load1<SF32>(a.S, row * a.lds + at) - st.x) * st.y;
  };
  float sum_g = 0.f, sum_gn = 0.f;
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) {
    float g;
    const float n = value(at, &g);
    sum_g += g;
    sum_gn = fmaf(g, n, sum_gn);
  }
  sum_g = row_sum<kNormThreads>(sum_g, slots) / (float)a.C;
  sum_gn = row_sum<kNormThreads>(sum_gn, slots + 4) / (float)a.C;
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) {
    float g;
    const float n = value(at, &g);
    const float d = st.y * (g - sum_g - n * sum_gn);
    store1(a.dX, row * a.lddx + at, a.dS ? d + load1<YF32>(a.dS, row * a.ldds + at) : d, a.dx_bf16);
  }
}
// ... and dw, db: a wave on 64 columns of every (4 gridDim.y)-th row, partial sums as above.
template <bool YF32, bool SF32>
__global__ void __launch_bounds__(kNormThreads) norm_grad_columns_kernel(const NormGradArgs a) {
  __shared__ float part[2][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at = (int64_t)blockIdx.x * 64 + lane;
  float dw = 0.f, db = 0.f;
  if (at < a.C)
    for (int64_t row = (int64_t)blockIdx.y * 4 + wave; row < a.T; row += (int64_t)gridDim.y * 4) {
      const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
      const float d = load1<YF32>(a.dY, row * a.lddy + at);
      dw = fmaf(d, (load1<SF32>(a.S, row * a.lds + at) - st.x) * st.y, dw);
      db += d;
    }
  part[0][wave][lane] = dw;
  part[1][wave][lane] = db;
  __syncthreads();
  if (wave < 2 && at < a.C) {
    float* out = a.partial ? a.partial + ((int64_t)blockIdx.y * 2 + wave) * a.C : (wave ? a.db : a.dw);
    out[at] = (part[wave][0][lane] + part[wave][1][lane]) + (part[wave][2][lane] + part[wave][3][lane]);
  }
}

// How a row of C elements is held: lanes per row, steps of eight elements per lane (0: not in registers).
struct RowForm { int lanes, steps; };
RowForm row_form(int64_t C) {
  if (C <= 128) return {16, 1};
  if (C <= 512) return {64, 1};
  if (C <= 1024) return {64, 2};
  if (C <= 2048) return {256, 1};
  if (C <= 4096) return {256, 2};
  if (C <= 6144) return {256, 3};
  if (C <= 8192) return {256, 4};
  return {0, 0};
}

// calls f(lanes, steps as integral constants) for the form
template <int N> struct Int { static constexpr int value = N; };
template <class F>
void with_form(const RowForm& r, F&& f) {
  if (r.lanes == 16) f(Int<16>{}, Int<1>{});
  else if (r.lanes == 64) r.steps == 1 ? f(Int<64>{}, Int<1>{}) : f(Int<64>{}, Int<2>{});
  else if (r.steps == 1) f(Int<256>{}, Int<1>{});
  else if (r.steps == 2) f(Int<256>{}, Int<2>{});
  else if (r.steps == 3) f(Int<256>{}, Int<3>{});
  else f(Int<256>{}, Int<4>{});
}

// Blocks that walk the rows of the backward pass, each with 2 C partial sums that are written and read once more; fewer where there
// are fewer rows.  Rows of a wave: what a compute unit's registers hold of them in bfloat16, three; rows of a block: two.  The whole
// call with 256, 512, 768 and 1024 blocks: 50432 x 768 of bfloat16 76, 65, 64 and 75 us; 4099 x 5003 of float 93, 75, 87 and 86.  By the
// width alone, since the workspace's size knows no types: of rows of a wave with float on a side two fit, and 768 are too many
// there (50432 x 768 of float 118, 121, 134 and 124; float rows with gradients in bfloat16 90, 90, 105 and 95).
constexpr int64_t kWaveRowBlocks = 768, kBlockRowBlocks = 512;
int64_t grad_blocks(int64_t T, const RowForm& r) {
  const int64_t per_block = r.lanes ? kNormThreads / r.lanes : 4, all = (T + per_block - 1) / per_block;
  const int64_t most = r.lanes == kNormThreads ? kBlockRowBlocks : kWaveRowBlocks;
  return all < most ? all : most;
}

}  // namespace

hipError_t launch_norm(const NormCall& c, hipStream_t s) {
  NormArgs a;
  a.X = c.X; a.R = c.R; a.w = c.w; a.b = c.b; a.Y = c.Y; a.S = c.S; a.stats = c.stats;
  a.T = c.T; a.C = c.C; a.ldx = c.ldx; a.ldr = c.ldr; a.ldy = c.ldy; a.lds = c.lds; a.eps = c.eps; a.y_bf16 = !c.y_f32;
  const RowForm r = row_form(c.C);
  if (r.lanes == 0) {
    if (c.x_f32) norm_long_kernel<true><<<flat_grid_256(c.T * kNormThreads), kNormThreads, 0, s>>>(a);
    else norm_long_kernel<false><<<flat_grid_256(c.T * kNormThreads), kNormThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  with_form(r, [&](auto lanes, auto steps) {
    constexpr int L = decltype(lanes)::value, CH = decltype(steps)::value;
    const dim3 grid = flat_grid_256(c.T * L);
    if (c.x_f32) norm_kernel<true, L, CH><<<grid, kNormThreads, 0, s>>>(a);
    else norm_kernel<false, L, CH><<<grid, kNormThreads, 0, s>>>(a);
  });
  return hipGetLastError();
}

size_t norm_grad_workspace_bytes(int64_t T, int64_t C) {
  const int64_t blocks = grad_blocks(T, row_form(C));
  return blocks > 1 ? (size_t)blocks * 2 * (size_t)C * sizeof(float) : 0;
}

hipError_t launch_norm_grad(const NormGradCall& c, hipStream_t s) {
  NormGradArgs a;
  a.dY = c.dY; a.S = c.S; a.stats = c.stats; a.w = c.w; a.dS = c.dS; a.dX = c.dX; a.dw = c.dw; a.db = c.db;
  a.T = c.T; a.C = c.C; a.lddy = c.lddy; a.lds = c.lds; a.ldds = c.ldds; a.lddx = c.lddx; a.dx_bf16 = !c.dx_f32;
  const RowForm r = row_form(c.C);
  auto typed = [&](auto f) {
    if (c.dy_f32) c.s_f32 ? f(Int<1>{}, Int<1>{}) : f(Int<1>{}, Int<0>{});
    else c.s_f32 ? f(Int<0>{}, Int<1>{}) : f(Int<0>{}, Int<0>{});
  };
  const int64_t blocks = grad_blocks(c.T, r);
  if (r.lanes == 0) {
    a.partial = blocks > 1 ? static_cast<float*>(c.workspace) : nullptr;
    typed([&](auto y, auto x) {
      constexpr bool YF = decltype(y)::value, SF = decltype(x)::value;
      norm_grad_long_kernel<YF, SF><<<flat_grid_256(c.T * kNormThreads), kNormThreads, 0, s>>>(a);
      if (c.dw != nullptr)
        norm_grad_columns_kernel<YF, SF><<<dim3((unsigned)((c.C + 63) / 64), (unsigned)blocks), kNormThreads, 0, s>>>(a);
    });
  } else {
    a.partial = blocks > 1 ? static_cast<float*>(c.workspace) : nullptr;
    with_form(r, [&](auto lanes, auto steps) {
      constexpr int L = decltype(lanes)::value, CH = decltype(steps)::value;
      typed([&](auto y, auto x) {
        norm_grad_kernel<decltype(y)::value, decltype(x)::value, L, CH><<<dim3((unsigned)blocks), kNormThreads, 0, s>>>(a);
      });
    });
  }
  if (c.dw != nullptr && blocks > 1)
    norm_grad_sum_kernel<<<dim3((unsigned)((2 * c.C + kSumCols - 1) / kSumCols)), kSumCols * kSumRows, 0, s>>>(
        a.partial, (int)blocks, c.C, c.dw, c.db);
  return hipGetLastError();
}

}  // namespace nm
