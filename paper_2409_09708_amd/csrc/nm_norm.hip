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
// bfloat16.  The mean is taken first and the variance from the differences to it (the row lies in registers, so the
// second sum costs no memory traffic), which keeps rows with a large common offset exact.
//
// Bound by memory at any width: 8 flops per element forward, 14 backward, against 4 to 16 bytes.  A row is held by
// LANES lanes (16 for the narrowest, a wave, or a block of four waves), 8 consecutive elements (one 16-byte piece of
// bfloat16) per lane and step, so that a wave's load covers whole 128-byte lines; where the width, a leading dimension
// or an address rules that out, one element per lane and step.  Rows above 8192 elements are read again for each sum.
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

template <bool XF32, int LANES, int VEC, int CH>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const NormArgs a) {
  __shared__ float slots[8];
  const int lane = threadIdx.x % LANES;
  const int64_t row = flat_lane_256() / LANES;
  const bool live = row < a.T;
  const int C = (int)a.C;
  float x[CH][VEC];
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * LANES + lane) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[c][e] = 0.f;
    if (live && at < C) {
      load_vec<XF32, VEC>(a.X, row * a.ldx + at, x[c]);
      if (a.R != nullptr) {
        float r[VEC];
        load_vec<XF32, VEC>(a.R, row * a.ldr + at, r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[c][e] += r[e];
        if (a.S != nullptr) store_vec<VEC>(a.S, row * a.lds + at, x[c], !XF32);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum += x[c][e];
    }
  }
  const float inv = 1.f / (float)C;
  const float mean = row_sum<LANES>(sum, slots) * inv;
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if ((c * LANES + lane) * VEC < C) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) sq = fmaf(x[c][e] - mean, x[c][e] - mean, sq);
    }
  const float rstd = rsqrtf(row_sum<LANES>(sq, slots + 4) * inv + a.eps);
  if (!live) return;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * LANES + lane) * VEC;
    if (at < C) {
      float w[VEC], b[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) { w[e] = 1.f; b[e] = 0.f; }
      if (a.w != nullptr) load_vec<true, VEC>(a.w, at, w);
      if (a.b != nullptr) load_vec<true, VEC>(a.b, at, b);
#pragma unroll
      for (int e = 0; e < VEC; ++e) w[e] = fmaf((x[c][e] - mean) * rstd, w[e], b[e]);
      store_vec<VEC>(a.Y, row * a.ldy + at, w, a.y_bf16);
    }
  }
  if (a.stats != nullptr && lane == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = float2{mean, rstd};
}

// Rows of any length: one block each, read once for every sum.
template <bool XF32>
__global__ void __launch_bounds__(kNormThreads) norm_long_kernel(const NormArgs a) {
  __shared__ float slots[8];
  const int64_t row = flat_lane_256() / kNormThreads;
  if (row >= a.T) return;
  auto value = [&](int64_t at) {
    float x[1], r[1];
    load_vec<XF32, 1>(a.X, row * a.ldx + at, x);
    if (a.R == nullptr) return x[0];
    load_vec<XF32, 1>(a.R, row * a.ldr + at, r);
    return x[0] + r[0];
  };
  float sum = 0.f;
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) sum += value(at);
  const float inv = 1.f / (float)a.C;
  const float mean = row_sum<kNormThreads>(sum, slots) * inv;
  float sq = 0.f;
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) {
    const float d = value(at) - mean;
    sq = fmaf(d, d, sq);
  }
  const float rstd = rsqrtf(row_sum<kNormThreads>(sq, slots + 4) * inv + a.eps);
  for (int64_t at = threadIdx.x; at < a.C; at += kNormThreads) {
    const float s[1] = {value(at)};
    const float y[1] = {fmaf((s[0] - mean) * rstd, a.w ? a.w[at] : 1.f, a.b ? a.b[at] : 0.f)};
    if (a.R != nullptr && a.S != nullptr) store_vec<1>(a.S, row * a.lds + at, s, !XF32);
    store_vec<1>(a.Y, row * a.ldy + at, y, a.y_bf16);
  }
  if (a.stats != nullptr && threadIdx.x == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = float2{mean, rstd};
}

// A block walks over rows, LANES lanes to each, and keeps its share of dw and db in registers; at the end the row groups of
// the block add theirs in LDS, and the blocks' sums are added in order by a second launch (norm_grad_sum_kernel): the result
// does not depend on scheduling.
template <bool YF32, bool SF32, int LANES, int VEC, int CH>
__global__ void __launch_bounds__(kNormThreads) norm_grad_kernel(const NormGradArgs a) {
  __shared__ float slots[2][8];
  constexpr int ROWS = kNormThreads / LANES;
  constexpr int W = CH * LANES * VEC;  // columns held, >= C
  __shared__ float totals[ROWS > 1 ? 2 * W : 1];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int C = (int)a.C;
  const float inv = 1.f / (float)C;
  float dw[CH][VEC], db[CH][VEC];
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < VEC; ++e) dw[c][e] = db[c][e] = 0.f;
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.T; first += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    const int64_t row = first + group;
    const bool live = row < a.T;
    const float2 st = live ? *reinterpret_cast<const float2*>(a.stats + 2 * row) : float2{0.f, 0.f};
    float n[CH][VEC], g[CH][VEC];
    float sum_g = 0.f, sum_gn = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LANES + lane) * VEC;
      if (live && at < C) {
        load_vec<SF32, VEC>(a.S, row * a.lds + at, n[c]);
        load_vec<YF32, VEC>(a.dY, row * a.lddy + at, g[c]);
        float w[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = 1.f;
        if (a.w != nullptr) load_vec<true, VEC>(a.w, at, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          n[c][e] = (n[c][e] - st.x) * st.y;
          dw[c][e] = fmaf(g[c][e], n[c][e], dw[c][e]);
          db[c][e] += g[c][e];
          g[c][e] *= w[e];
          sum_g += g[c][e];
          sum_gn = fmaf(g[c][e], n[c][e], sum_gn);
        }
      }
    }
    sum_g = row_sum<LANES>(sum_g, slots[turn]) * inv;
    sum_gn = row_sum<LANES>(sum_gn, slots[turn] + 4) * inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LANES + lane) * VEC;
      if (live && at < C) {
        float d[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) d[e] = st.y * (g[c][e] - sum_g - n[c][e] * sum_gn);
        if (a.dS != nullptr) {
          float r[VEC];
          load_vec<YF32, VEC>(a.dS, row * a.ldds + at, r);
#pragma unroll
          for (int e = 0; e < VEC; ++e) d[e] += r[e];
        }
        store_vec<VEC>(a.dX, row * a.lddx + at, d, a.dx_bf16);
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
          for (int e = 0; e < VEC; ++e) {
            const int i = (c * VEC + e) * LANES + lane;  // consecutive lanes on consecutive banks
            totals[i] = q ? totals[i] + dw[c][e] : dw[c][e];
            totals[W + i] = q ? totals[W + i] + db[c][e] : db[c][e];
          }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < W; i += kNormThreads) {
      const int l = i % LANES, ce = i / LANES;
      const int at = ((ce / VEC) * LANES + l) * VEC + ce % VEC;
      if (at < C) { out_w[at] = totals[i]; out_b[at] = totals[W + i]; }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = (c * LANES + lane) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (at + e < C) { out_w[at + e] = dw[c][e]; out_b[at + e] = db[c][e]; }
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
    float s[1], d[1];
    load_vec<SF32, 1>(a.S, row * a.lds + at, s);
    load_vec<YF32, 1>(a.dY, row * a.lddy + at, d);
    *g = a.w ? d[0] * a.w[at] : d[0];
    return (s[0] - st.x) * st.y;
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
    float g, r[1] = {0.f};
    const float n = value(at, &g);
    if (a.dS != nullptr) load_vec<YF32, 1>(a.dS, row * a.ldds + at, r);
    const float d[1] = {st.y * (g - sum_g - n * sum_gn) + r[0]};
    store_vec<1>(a.dX, row * a.lddx + at, d, a.dx_bf16);
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
      float s[1], d[1];
      load_vec<SF32, 1>(a.S, row * a.lds + at, s);
      load_vec<YF32, 1>(a.dY, row * a.lddy + at, d);
      dw = fmaf(d[0], (s[0] - st.x) * st.y, dw);
      db += d[0];
    }
  part[0][wave][lane] = dw;
  part[1][wave][lane] = db;
  __syncthreads();
  if (wave < 2 && at < a.C) {
    float* out = a.partial ? a.partial + ((int64_t)blockIdx.y * 2 + wave) * a.C : (wave ? a.db : a.dw);
    out[at] = (part[wave][0][lane] + part[wave][1][lane]) + (part[wave][2][lane] + part[wave][3][lane]);
  }
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// How a row of C elements is held: lanes per row, elements per lane and step, steps (0 = not in registers).
struct RowForm { int lanes, vec, steps; };
RowForm row_form(int64_t C, bool pieces) {
  if (pieces) {
    if (C <= 128) return {16, 8, 1};
    if (C <= 512) return {64, 8, 1};
    if (C <= 1024) return {64, 8, 2};
    if (C <= 2048) return {256, 8, 1};
    if (C <= 4096) return {256, 8, 2};
    if (C <= 8192) return {256, 8, 4};
  } else {
    if (C <= 256) return {64, 1, 4};
    if (C <= 1024) return {64, 1, 16};
    if (C <= 4096) return {256, 1, 16};
    if (C <= 8192) return {256, 1, 32};
  }
  return {0, 0, 0};
}

// calls f(lanes, vec, steps as integral constants) for the form
template <int N> struct Int { static constexpr int value = N; };
template <class F>
void with_form(const RowForm& r, F&& f) {
  if (r.vec == 8) {
    if (r.lanes == 16) f(Int<16>{}, Int<8>{}, Int<1>{});
    else if (r.lanes == 64) r.steps == 1 ? f(Int<64>{}, Int<8>{}, Int<1>{}) : f(Int<64>{}, Int<8>{}, Int<2>{});
    else if (r.steps == 1) f(Int<256>{}, Int<8>{}, Int<1>{});
    else if (r.steps == 2) f(Int<256>{}, Int<8>{}, Int<2>{});
    else f(Int<256>{}, Int<8>{}, Int<4>{});
  } else {
    if (r.lanes == 64) r.steps == 4 ? f(Int<64>{}, Int<1>{}, Int<4>{}) : f(Int<64>{}, Int<1>{}, Int<16>{});
    else if (r.steps == 16) f(Int<256>{}, Int<1>{}, Int<16>{});
    else f(Int<256>{}, Int<1>{}, Int<32>{});
  }
}

// Blocks that walk the rows of the backward pass: two per compute unit (each keeps 2 C partial sums, written and read once
// more), fewer where there are fewer rows.
constexpr int64_t kGradBlocks = 512;
int64_t grad_blocks(int64_t T, int rows_per_block) {
  const int64_t all = (T + rows_per_block - 1) / rows_per_block;
  return all < kGradBlocks ? all : kGradBlocks;
}

}  // namespace

hipError_t launch_norm(const NormCall& c, hipStream_t s) {
  NormArgs a;
  a.X = c.X; a.R = c.R; a.w = c.w; a.b = c.b; a.Y = c.Y; a.S = c.S; a.stats = c.stats;
  a.T = c.T; a.C = c.C; a.ldx = c.ldx; a.ldr = c.ldr; a.ldy = c.ldy; a.lds = c.lds; a.eps = c.eps; a.y_bf16 = !c.y_f32;
  const bool pieces = (c.C | c.ldx | c.ldy | (c.R ? c.ldr : 0) | (c.S ? c.lds : 0)) % 8 == 0 && aligned16(c.X) &&
                      aligned16(c.R) && aligned16(c.Y) && aligned16(c.S) && aligned16(c.w) && aligned16(c.b);
  const RowForm r = row_form(c.C, pieces);
  if (r.lanes == 0) {
    if (c.x_f32) norm_long_kernel<true><<<flat_grid_256(c.T * kNormThreads), kNormThreads, 0, s>>>(a);
    else norm_long_kernel<false><<<flat_grid_256(c.T * kNormThreads), kNormThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  with_form(r, [&](auto lanes, auto vec, auto steps) {
    constexpr int L = decltype(lanes)::value, V = decltype(vec)::value, CH = decltype(steps)::value;
    const dim3 grid = flat_grid_256(c.T * L);
    if (c.x_f32) norm_kernel<true, L, V, CH><<<grid, kNormThreads, 0, s>>>(a);
    else norm_kernel<false, L, V, CH><<<grid, kNormThreads, 0, s>>>(a);
  });
  return hipGetLastError();
}

size_t norm_grad_workspace_bytes(int64_t T, int64_t C) {
  // (at most one block per row: a form with several rows to a block takes fewer)
  const int64_t blocks = T < kGradBlocks ? T : kGradBlocks;
  return blocks > 1 ? (size_t)blocks * 2 * (size_t)C * sizeof(float) : 0;
}

hipError_t launch_norm_grad(const NormGradCall& c, hipStream_t s) {
  NormGradArgs a;
  a.dY = c.dY; a.S = c.S; a.stats = c.stats; a.w = c.w; a.dS = c.dS; a.dX = c.dX; a.dw = c.dw; a.db = c.db;
  a.T = c.T; a.C = c.C; a.lddy = c.lddy; a.lds = c.lds; a.ldds = c.ldds; a.lddx = c.lddx; a.dx_bf16 = !c.dx_f32;
  const bool pieces = (c.C | c.lddy | c.lds | c.lddx | (c.dS ? c.ldds : 0)) % 8 == 0 && aligned16(c.dY) && aligned16(c.S) &&
                      aligned16(c.dX) && aligned16(c.dS) && aligned16(c.w);
  const RowForm r = row_form(c.C, pieces);
  auto typed = [&](auto f) {
    if (c.dy_f32) c.s_f32 ? f(Int<1>{}, Int<1>{}) : f(Int<1>{}, Int<0>{});
    else c.s_f32 ? f(Int<0>{}, Int<1>{}) : f(Int<0>{}, Int<0>{});
  };
  int64_t blocks = grad_blocks(c.T, r.lanes ? kNormThreads / r.lanes : 4);
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
    with_form(r, [&](auto lanes, auto vec, auto steps) {
      constexpr int L = decltype(lanes)::value, V = decltype(vec)::value, CH = decltype(steps)::value;
      typed([&](auto y, auto x) {
        norm_grad_kernel<decltype(y)::value, decltype(x)::value, L, V, CH><<<dim3((unsigned)blocks), kNormThreads, 0, s>>>(a);
      });
    });
  }
  if (c.dw != nullptr && blocks > 1)
    norm_grad_sum_kernel<<<dim3((unsigned)((2 * c.C + kSumCols - 1) / kSumCols)), kSumCols * kSumRows, 0, s>>>(
        a.partial, (int)blocks, c.C, c.dw, c.db);
  return hipGetLastError();
}

}  // namespace nm
