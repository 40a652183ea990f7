// Backward pass of the attention.  With p_ij = exp(s_ij - lse_i) recomputed from the saved log-sum and
// D_i = sum_d dO_id O_id:
//
//   dP_ij = dO_i . v_j,  dS_ij = p_ij (dP_ij - D_i),
//   dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i,  dV_j = sum_i p_ij dO_i   (the latter two over the query
//   heads that share the key head as well).
//
// Two kernels, so that every sum is taken in one place and in a fixed order: grad_query_kernel keeps the queries of a block
// and walks over the keys (and leaves D for the other one), grad_key_kernel keeps keys and walks over the queries of the group's
// heads.  That recomputes the scores and dP once more, 7 products instead of 5, and needs no atomics.  Scores, probabilities and sums
// are 32-bit floats; p and dS are rounded to bfloat16 as operands of the products that take them.
#include "nm_attention.h"

namespace nm {

namespace {

struct GradArgs {
  AttentionCall c;
  int group;
  float scale_log2;
  int n_q_tiles, n_k_tiles;
  float* delta;  // D: [Hq, Tq]
};

constexpr int kKeys = 64;              // keys per tile of grad_query_kernel
constexpr int kRows = kWaves * 32;     // queries (keys) that a block keeps
constexpr int kQueries = 32;           // queries per tile of grad_key_kernel

template <int DP, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, 2) grad_query_kernel(const GradArgs a) {
  using Tile = RowTile<DP>;
  constexpr int NB = DP / 32, STEPS = DP / 16, TILE_BYTES = kKeys * Tile::kRowBytes;
  constexpr int LOADS = kKeys * Tile::kPieces / kThreads;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2][2 * TILE_BYTES];
  TilePlace at;
  if (!tile_place(a.c.B, a.c.Hkv, a.group, a.n_q_tiles, true, &at)) return;
  const int head = at.kv_head * a.group + at.sub;
  const int D = a.c.D;
  const Span sq = sequence(a.c.offsets_q, nullptr, at.seq, a.c.Tq);
  const Span sk = sequence(a.c.offsets_k, a.c.lengths_k, at.seq, a.c.Tk);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int shift = sk.len - sq.len;
  const bf16_t* Kh = a.c.K.p + sk.first * a.c.K.token + at.kv_head * a.c.K.head;
  const bf16_t* Vh = a.c.V.p + sk.first * a.c.V.token + at.kv_head * a.c.V.head;

  for (int tile = at.tile; (int64_t)tile * kRows < sq.len; tile += a.n_q_tiles) {
    const int q_wave = tile * kRows + wave * 32;
    const int qi = q_wave + (lane & 31);
    const bool live = qi < sq.len;
    const int64_t tok = sq.first + qi;
    const bf16_t* q_row = a.c.Q.p + tok * a.c.Q.token + head * a.c.Q.head;
    const bf16_t* do_row = a.c.dO.p + tok * a.c.dO.token + head * a.c.dO.head;
    const bf16_t* o_row = a.c.O.p + tok * a.c.O.token + head * a.c.O.head;
    u32x4_t q[STEPS], g[STEPS];
    float delta = 0.f;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      q[st] = load_piece<ALIGNED>(q_row, 16 * st + 8 * half, D, live);
      g[st] = load_piece<ALIGNED>(do_row, 16 * st + 8 * half, D, live);
      const u32x4_t o = load_piece<ALIGNED>(o_row, 16 * st + 8 * half, D, live);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        delta = fmaf(__uint_as_float(g[st][e] << 16), __uint_as_float(o[e] << 16), delta);
        delta = fmaf(__uint_as_float(g[st][e] & 0xFFFF0000u), __uint_as_float(o[e] & 0xFFFF0000u), delta);
      }
    }
    delta = half_sum(delta);
    float lse2 = 0.f;
    if (live) {
      const int64_t n = (int64_t)head * a.c.Tq + tok;
      lse2 = a.c.lse[n] * kLog2e;
      if (lse2 == kMinusInf) lse2 = 0.f;  // a query that sees no key
      if (half == 0) a.delta[n] = delta;
    }

    const int last_q = (tile + 1) * kRows < sq.len ? (tile + 1) * kRows : sq.len;
    int end = sk.len, wave_end = sk.len, first_hidden = sk.len, limit = sk.len;
    if (a.c.causal) {
      auto upto = [&](int i) { const int n = i + shift + 1; return n < 0 ? 0 : n < sk.len ? n : sk.len; };
      end = upto(last_q - 1);
      wave_end = upto(q_wave + 31 < last_q ? q_wave + 31 : last_q - 1);
      first_hidden = upto(q_wave);
      limit = upto(qi);
    }
    if (q_wave >= sq.len) wave_end = 0;

    f32x16_t acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;

    u32x4_t k_in[LOADS], v_in[LOADS];
    auto fetch = [&](int k0) {
#pragma unroll
      for (int n = 0; n < LOADS; ++n) {
        const int i = n * kThreads + tid, row = k0 + i / Tile::kPieces, d = i % Tile::kPieces * 8;
        const bool there = row < sk.len;
        k_in[n] = load_piece<ALIGNED>(Kh + (int64_t)row * a.c.K.token, d, D, there);
        v_in[n] = load_piece<ALIGNED>(Vh + (int64_t)row * a.c.V.token, d, D, there);
      }
    };
    auto settle = [&](int stage) {
#pragma unroll
      for (int n = 0; n < LOADS; ++n) {
        const int i = n * kThreads + tid, to = Tile::place(i / Tile::kPieces, i % Tile::kPieces);
        *reinterpret_cast<u32x4_t*>(smem[stage] + to) = k_in[n];
        *reinterpret_cast<u32x4_t*>(smem[stage] + TILE_BYTES + to) = v_in[n];
      }
    };
    const int n_key_tiles = (end + kKeys - 1) / kKeys;
    __syncthreads();
    if (n_key_tiles > 0) {
      fetch(0);
      settle(0);
    }
    __syncthreads();
    for (int kt = 0; kt < n_key_tiles; ++kt) {
      const int k0 = kt * kKeys;
      if (kt + 1 < n_key_tiles) fetch(k0 + kKeys);
      const unsigned char* k_tile = smem[kt & 1];
      const unsigned char* v_tile = k_tile + TILE_BYTES;
      if (k0 < wave_end) {
#pragma unroll
        for (int kb = 0; kb < kKeys / 32; ++kb) {
          f32x16_t s, dp;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
          for (int st = 0; st < STEPS; ++st) s = mma32(Tile::rows(k_tile, 32 * kb, st, lane), q[st], s);
#pragma unroll
          for (int st = 0; st < STEPS; ++st) dp = mma32(Tile::rows(v_tile, 32 * kb, st, lane), g[st], dp);
          if (k0 + 32 * kb + 32 > first_hidden) hide_rows(s, limit - k0 - 32 * kb - 4 * half);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fast_exp2(fmaf(s[r], a.scale_log2, -lse2)) * (dp[r] - delta);
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            const u32x4_t ds = acc_operand(s, st);
#pragma unroll
            for (int b = 0; b < NB; ++b) acc[b] = mma32(Tile::columns(k_tile, 32 * kb + 16 * st, b, lane), ds, acc[b]);
          }
        }
      }
      if (kt + 1 < n_key_tiles) settle((kt + 1) & 1);
      __syncthreads();
    }
    if (live) store_column<DP, ALIGNED>(a.c.dQ.p + tok * a.c.dQ.token + head * a.c.dQ.head, acc, lane, D, a.c.scale);
  }
}

template <int DP, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, DP == 128 ? 1 : 2) grad_key_kernel(const GradArgs a) {
  using Tile = RowTile<DP>;
  constexpr int NB = DP / 32, STEPS = DP / 16, TILE_BYTES = kQueries * Tile::kRowBytes;
  constexpr int PIECES = kQueries * Tile::kPieces, LOADS = (PIECES + kThreads - 1) / kThreads;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2][2 * TILE_BYTES];  // two stages of queries and dO
  __shared__ __attribute__((aligned(16))) float rows[2][2][kQueries];               // ... and of lse (base 2) and D
  TilePlace at;
  if (!tile_place(a.c.B, a.c.Hkv, 1, a.n_k_tiles, false, &at)) return;
  const int D = a.c.D;
  const Span sq = sequence(a.c.offsets_q, nullptr, at.seq, a.c.Tq);
  const Span sk = sequence(a.c.offsets_k, a.c.lengths_k, at.seq, a.c.Tk);
  const Span room = sequence(a.c.offsets_k, nullptr, at.seq, a.c.Tk);  // rows past the length get zeros
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int shift = sk.len - sq.len;

  for (int tile = at.tile; (int64_t)tile * kRows < room.len; tile += a.n_k_tiles) {
    const int k_wave = tile * kRows + wave * 32;
    const int kj = k_wave + (lane & 31);
    const int64_t tok = sk.first + kj;
    const bf16_t* k_row = a.c.K.p + tok * a.c.K.token + at.kv_head * a.c.K.head;
    const bf16_t* v_row = a.c.V.p + tok * a.c.V.token + at.kv_head * a.c.V.head;
    u32x4_t k[STEPS], v[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      k[st] = load_piece<ALIGNED>(k_row, 16 * st + 8 * half, D, kj < sk.len);
      v[st] = load_piece<ALIGNED>(v_row, 16 * st + 8 * half, D, kj < sk.len);
    }
    f32x16_t dk[NB], dv[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.f;

    // query tiles from the first one that sees a key of the block, for each head of the group: one list
    int first_q = 0;
    if (a.c.causal) first_q = tile * kRows - shift < 0 ? 0 : (tile * kRows - shift) / kQueries * kQueries;
    const int per_head = tile * kRows < sk.len && first_q < sq.len ? (sq.len - first_q + kQueries - 1) / kQueries : 0;
    const int n_steps = per_head * a.group;

    u32x4_t q_in[LOADS], g_in[LOADS];
    float row_in = 0.f;
    auto fetch = [&](int step) {
      const int head = at.kv_head * a.group + step / per_head, q0 = first_q + step % per_head * kQueries;
      const bf16_t* Qh = a.c.Q.p + sq.first * a.c.Q.token + head * a.c.Q.head;
      const bf16_t* Gh = a.c.dO.p + sq.first * a.c.dO.token + head * a.c.dO.head;
#pragma unroll
      for (int n = 0; n < LOADS; ++n) {
        const int i = n * kThreads + tid, row = q0 + i / Tile::kPieces, d = i % Tile::kPieces * 8;
        const bool there = row < sq.len && (PIECES % kThreads == 0 || i < PIECES);
        q_in[n] = load_piece<ALIGNED>(Qh + (int64_t)row * a.c.Q.token, d, D, there);
        g_in[n] = load_piece<ALIGNED>(Gh + (int64_t)row * a.c.dO.token, d, D, there);
      }
      if (tid < 2 * kQueries) {
        const int row = q0 + tid % kQueries;
        const int64_t n = (int64_t)head * a.c.Tq + sq.first + row;
        row_in = row >= sq.len ? 0.f : tid < kQueries ? a.c.lse[n] * kLog2e : a.delta[n];
        if (row_in == kMinusInf) row_in = 0.f;
      }
    };
    auto settle = [&](int stage) {
#pragma unroll
      for (int n = 0; n < LOADS; ++n) {
        const int i = n * kThreads + tid, to = Tile::place(i / Tile::kPieces, i % Tile::kPieces);
        if (PIECES % kThreads == 0 || i < PIECES) {
          *reinterpret_cast<u32x4_t*>(smem[stage] + to) = q_in[n];
          *reinterpret_cast<u32x4_t*>(smem[stage] + TILE_BYTES + to) = g_in[n];
        }
      }
      if (tid < 2 * kQueries) rows[stage][tid / kQueries][tid % kQueries] = row_in;
    };
    __syncthreads();
    if (n_steps > 0) {
      fetch(0);
      settle(0);
    }
    __syncthreads();
    for (int step = 0; step < n_steps; ++step) {
      const int q0 = first_q + step % per_head * kQueries;
      if (step + 1 < n_steps) fetch(step + 1);
      const unsigned char* q_tile = smem[step & 1];
      const unsigned char* g_tile = q_tile + TILE_BYTES;
      // (a wave whose keys none of these queries sees, or without keys)
      if (k_wave < sk.len && (!a.c.causal || q0 + kQueries - 1 + shift >= k_wave)) {
        f32x16_t s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) s = mma32(Tile::rows(q_tile, 0, st, lane), k[st], s);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) dp = mma32(Tile::rows(g_tile, 0, st, lane), v[st], dp);
        const float* row = rows[step & 1][0] + 4 * half;
        if (a.c.causal && q0 + shift < k_wave + 31) {
          const int first = kj - shift - q0 - 4 * half;  // rows before it do not see the lane's key
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = acc_row(r) >= first ? s[r] : kMinusInf;
        }
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4_t lse = *reinterpret_cast<const f32x4_t*>(row + 8 * r4);
          const f32x4_t delta = *reinterpret_cast<const f32x4_t*>(row + kQueries + 8 * r4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * r4 + e;
            s[r] = fast_exp2(fmaf(s[r], a.scale_log2, -lse[e]));
            dp[r] = s[r] * (dp[r] - delta[e]);
          }
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const u32x4_t p = acc_operand(s, st), ds = acc_operand(dp, st);
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            dv[b] = mma32(Tile::columns(g_tile, 16 * st, b, lane), p, dv[b]);
            dk[b] = mma32(Tile::columns(q_tile, 16 * st, b, lane), ds, dk[b]);
          }
        }
      }
      if (step + 1 < n_steps) settle((step + 1) & 1);
      __syncthreads();
    }
    if (kj < room.len) {
      if (kj >= sk.len) {  // (it was multiplied as a row of zeros: what came of that, infinities included, is not its gradient)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.f;
      }
      store_column<DP, ALIGNED>(a.c.dK.p + tok * a.c.dK.token + at.kv_head * a.c.dK.head, dk, lane, D, a.c.scale);
      store_column<DP, ALIGNED>(a.c.dV.p + tok * a.c.dV.token + at.kv_head * a.c.dV.head, dv, lane, D, 1.f);
    }
  }
}

int tiles(int64_t most, int B, int Hkv, int group) {
  int n = (int)((most + kRows - 1) / kRows);
  if (n < 1) n = 1;
  while (tile_blocks(B, Hkv, group, n) >= kMostBlocks) n = (n + 1) / 2;
  return n;
}

}  // namespace

size_t attention_grad_workspace_bytes(int64_t Tq, int Hq) { return (size_t)Tq * Hq * sizeof(float); }

hipError_t launch_attention_grad(const AttentionCall& c, hipStream_t s) {
  GradArgs a = {};
  a.c = c;
  a.group = c.Hq / c.Hkv;
  a.scale_log2 = c.scale * kLog2e;
  a.n_q_tiles = tiles(c.max_q, c.B, c.Hkv, a.group);
  a.n_k_tiles = tiles(c.max_k, c.B, c.Hkv, 1);
  a.delta = static_cast<float*>(c.workspace);
  const bool aligned = c.D % 8 == 0 && head_rows_aligned(c.Q) && head_rows_aligned(c.K) && head_rows_aligned(c.V) &&
                       head_rows_aligned(c.O) && head_rows_aligned(c.dO) && head_rows_aligned(c.dQ) &&
                       head_rows_aligned(c.dK) && head_rows_aligned(c.dV);
  auto launch = [&](auto dp, auto al) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool ALIGNED = decltype(al)::value;
    const int64_t q_blocks = tile_blocks(c.B, c.Hkv, a.group, a.n_q_tiles), k_blocks = tile_blocks(c.B, c.Hkv, 1, a.n_k_tiles);
    grad_query_kernel<DP, ALIGNED><<<dim3((unsigned)q_blocks), kThreads, 0, s>>>(a);
    if (c.Tk > 0) grad_key_kernel<DP, ALIGNED><<<dim3((unsigned)k_blocks), kThreads, 0, s>>>(a);
  };
  if (aligned) with_head<true>(c.D, launch);
  else with_head<false>(c.D, launch);
  return hipGetLastError();
}

}  // namespace nm
