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
//
// Measured: packed causal texts of 4093, 848 and 1393 tokens, 16 heads on 4 of 128: 399 us, of which the queries' kernel has 142, the
// keys' 232 and the joined sums 25; of 199 GFLOP that makes 500 TFLOP/s, 700 of the products there are.  Bound by registers: two
// waves a SIMD, 256 registers each, are too few to keep the matrix cores fed through the exponentials, and the keys' kernel spills 38
// of its own.  64 images of 197 tokens, 12 heads of 64: 34 and 45 us, 155 MB.
#include "nm_attention.h"

#include <algorithm>
#include <iterator>

namespace nm {

namespace {

struct GradArgs {
  AttentionCall c;
  int group;
  float scale_log2;
  int n_q_tiles, n_k_tiles;
  int chunk, n_chunks;  // of a key tile's steps
  float* delta;         // D: [Hq, Tq]
  float* part;          // [chunk][key][key head][dK, dV][DP]
};

constexpr int kKeys = 64;              // keys per tile of grad_query_kernel
constexpr int kRows = kWaves * 32;     // queries (keys) that a block keeps
constexpr int kQueries = 32;           // queries per tile of grad_key_kernel
constexpr int64_t kKeyBlocks = 512;    // blocks that grad_key_kernel's work is cut for

template <int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 2) grad_query_kernel(const GradArgs a) {
  using Tile = RowTile<DP>;
  using Rows = WaveRows<DP>;
  constexpr int NB = DP / 32, STEPS = DP / 16, TILE_BYTES = kKeys * Tile::kRowBytes;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2][2 * TILE_BYTES];
  TilePlace at;
  if (!tile_place(a.c.B, a.c.Hkv, a.group, a.n_q_tiles, true, a.c.causal, &at)) return;
  const int head = at.kv_head * a.group + at.sub;
  const int D = WHOLE ? DP : a.c.D;
  const Sequence of = sequence(a.c, at.seq);
  const Span sq = of.q, sk = of.k;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int shift = sk.len - sq.len;
  TilePair<DP, kKeys, WHOLE, kThreads> load;
  load.base[0] = a.c.K.p + sk.first * a.c.K.token + at.kv_head * a.c.K.head;
  load.base[1] = a.c.V.p + sk.first * a.c.V.token + at.kv_head * a.c.V.head;
  load.stride[0] = a.c.K.token;
  load.stride[1] = a.c.V.token;
  load.rows = sk.len;
  load.D = D;
  load.smem = smem[0];
  load.lds = NM_LDS_ADDRESS(smem[0]);

  for (int tile = at.tile; (int64_t)tile * kRows < sq.len; tile += a.n_q_tiles) {
    const int q_wave = tile * kRows + wave * 32;
    const int qi = q_wave + (lane & 31);
    const bool live = qi < sq.len;
    const int64_t tok = sq.first + qi;
    const bf16_t* q_rows = a.c.Q.p + (sq.first + q_wave) * a.c.Q.token + head * a.c.Q.head;
    const bf16_t* do_rows = a.c.dO.p + (sq.first + q_wave) * a.c.dO.token + head * a.c.dO.head;
    const bf16_t* o_rows = a.c.O.p + (sq.first + q_wave) * a.c.O.token + head * a.c.O.head;
    u32x4_t q[STEPS], g[STEPS];
    float delta = 0.f;
    auto add = [&](u32x4_t x, u32x4_t o) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        delta = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(o[e] << 16), delta);
        delta = fmaf(__uint_as_float(x[e] & 0xFFFF0000u), __uint_as_float(o[e] & 0xFFFF0000u), delta);
      }
    };
    if constexpr (WHOLE) {
      u32x4_t o[STEPS];
      Rows::load(g, do_rows, a.c.dO.token, sq.len - q_wave, lane);
      Rows::load(o, o_rows, a.c.O.token, sq.len - q_wave, lane);
      Rows::load(q, q_rows, a.c.Q.token, sq.len - q_wave, lane);
      Rows::exchange(g);
      Rows::exchange(o);
#pragma unroll
      for (int st = 0; st < STEPS; ++st) add(g[st], o[st]);
      Rows::exchange(q);
    } else {
      const int row = lane & 31;
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        q[st] = load_piece(q_rows + row * a.c.Q.token, 16 * st + 8 * half, D, live);
        g[st] = load_piece(do_rows + row * a.c.dO.token, 16 * st + 8 * half, D, live);
        add(g[st], load_piece(o_rows + row * a.c.O.token, 16 * st + 8 * half, D, live));
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

    const int n_key_tiles = (end + kKeys - 1) / kKeys;
    if constexpr (WHOLE) {
      arrived(q);
      arrived(g);
      asm volatile("" : "+v"(lse2), "+v"(delta));
    }
    __syncthreads();  // (a block's second query tile: the first one's keys are no longer read)
    if (n_key_tiles > 0) load.fetch(0, 0);
    for (int kt = 0; kt < n_key_tiles; ++kt) {
      const int k0 = kt * kKeys;
      load.settle(kt & 1);
      __syncthreads();
      if (kt + 1 < n_key_tiles) load.fetch((kt + 1) & 1, k0 + kKeys);
      if (k0 < wave_end) {
        const uint32_t k_tile = load.lds + (uint32_t)(kt & 1) * 2 * TILE_BYTES;
        const uint32_t row_at = k_tile + Tile::row_base(lane), column_at = k_tile + Tile::column_base(lane);
#pragma unroll
        for (int kb = 0; kb < kKeys / 32; ++kb) {
          auto rows_of = [&](int i) { return Tile::rows(row_at + i % 2 * TILE_BYTES, 32 * kb, i / 2); };
          auto columns_of = [&](int i) { return Tile::columns(column_at, 32 * kb + i / NB * 16, i % NB); };
          f32x16_t s, dp;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
          u32x4_t f[kAhead];
          read_ahead<2 * STEPS>(f, rows_of);
          products<2 * STEPS>(f, rows_of, [&](int i, u32x4_t x) {
            if (i % 2 == 0) s = mma32(x, q[i / 2], s);
            else dp = mma32(x, g[i / 2], dp);
          });
          read_ahead<2 * NB>(f, columns_of);
          if (k0 + 32 * kb + 32 > first_hidden) hide_rows(s, limit - k0 - 32 * kb - 4 * half);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fast_exp2(fmaf(s[r], a.scale_log2, -lse2)) * (dp[r] - delta);
          const u32x4_t ds[2] = {acc_operand(s, 0), acc_operand(s, 1)};
          products<2 * NB>(f, columns_of, [&](int i, u32x4_t x) { acc[i % NB] = mma32(x, ds[i / NB], acc[i % NB]); });
        }
      }
    }
    bf16_t* dq_rows = a.c.dQ.p + (sq.first + q_wave) * a.c.dQ.token + head * a.c.dQ.head;
    if constexpr (WHOLE) Rows::store(dq_rows, a.c.dQ.token, sq.len - q_wave, acc, lane, a.c.scale);
    else if (live) store_column<DP>(dq_rows + (lane & 31) * a.c.dQ.token, acc, lane, D, a.c.scale);
  }
}

// Key tiles differ in how many queries see them, and shared key heads leave few of them, so the (head, query tile) steps of a key
// tile are cut into up to n_chunks for different blocks; where there is more than one, 32-bit sums of each go to the workspace
// and grad_key_sum_kernel adds them in order.  n_chunks is what the longest tile needs; the shorter ones under a causal mask are cut
// as well, down to a quarter of a chunk, since blocks that start later should be the shorter ones: one text of 8192, 16 heads on 4,
// 993 us, 1360 with chunks of one size (three quarters of it for the last tiles' blocks), 970 with all tiles cut alike, which costs
// many short texts more.
constexpr int kCutFiner = 4;
struct KeySteps {
  int first_q, per_head, steps, chunks, share;
};
__device__ __forceinline__ KeySteps key_steps(const GradArgs& a, int tile, int q_len, int k_len) {
  const int shift = k_len - q_len;
  KeySteps s;
  // query tiles from the first one that sees a key of the tile on, for each head of the group: one list
  s.first_q = !a.c.causal || tile * kRows - shift < 0 ? 0 : (tile * kRows - shift) / kQueries * kQueries;
  s.per_head = tile * kRows < k_len && s.first_q < q_len ? (q_len - s.first_q + kQueries - 1) / kQueries : 0;
  s.steps = s.per_head * a.group;
  s.chunks = (kCutFiner * s.steps + a.chunk - 1) / a.chunk;
  if (s.chunks < 1) s.chunks = 1;
  if (s.chunks > a.n_chunks) s.chunks = a.n_chunks;
  s.share = (s.steps + s.chunks - 1) / s.chunks;  // steps of a chunk (the last ones can have fewer)
  return s;
}

template <int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, DP == 128 && !WHOLE ? 1 : 2) grad_key_kernel(const GradArgs a) {
  using Tile = RowTile<DP>;
  using Rows = WaveRows<DP>;
  constexpr int NB = DP / 32, STEPS = DP / 16, TILE_BYTES = kQueries * Tile::kRowBytes;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2][2 * TILE_BYTES];  // two stages of queries and dO
  __shared__ __attribute__((aligned(16))) float rows[2][2][kQueries];               // ... and of lse (base 2) and D
  // Heads of 128 elements: the keys' operands stay in LDS, each wave's its own, since 64 registers of keys and values beside 160 of
  // sums leave too few for two waves a SIMD (65 were spilled; the packed texts above took 638 us, 420 with the keys in LDS, as things
  // were then; 38 still are).
  constexpr bool KEEP = DP == 128;
  __shared__ __attribute__((aligned(1024))) unsigned char kept[KEEP ? kRows * Tile::kRowBytes : 16];
  TilePlace at;
  if (!tile_place(a.c.B, a.c.Hkv, a.n_chunks, a.n_k_tiles, false, a.c.causal, &at)) return;
  const int chunk = at.sub;
  const int D = WHOLE ? DP : a.c.D;
  const Sequence of = sequence(a.c, at.seq);
  const Span sq = of.q, sk = of.k;  // (of.room rows of keys: those past the length get zeros)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int shift = sk.len - sq.len;
  TilePair<DP, kQueries, WHOLE, kThreads> load;
  load.stride[0] = a.c.Q.token;
  load.stride[1] = a.c.dO.token;
  load.rows = sq.len;
  load.D = D;
  load.smem = smem[0];
  load.lds = NM_LDS_ADDRESS(smem[0]);

  for (int tile = at.tile; (int64_t)tile * kRows < of.room; tile += a.n_k_tiles) {
    const KeySteps list = key_steps(a, tile, sq.len, sk.len);
    if (chunk >= list.chunks) continue;
    const int first_step = chunk * list.share < list.steps ? chunk * list.share : list.steps;
    const int end_step = first_step + list.share < list.steps ? first_step + list.share : list.steps;
    const int k_wave = tile * kRows + wave * 32;
    const int kj = k_wave + (lane & 31);
    const int64_t tok = sk.first + kj;
    const bf16_t* k_rows = a.c.K.p + (sk.first + k_wave) * a.c.K.token + at.kv_head * a.c.K.head;
    const bf16_t* v_rows = a.c.V.p + (sk.first + k_wave) * a.c.V.token + at.kv_head * a.c.V.head;
    u32x4_t k[STEPS], v[STEPS];
    unsigned char* own = kept + wave * 32 * Tile::kRowBytes;
    const uint32_t kept_tile = NM_LDS_ADDRESS(kept) + wave * 32 * Tile::kRowBytes;
    if constexpr (WHOLE) {
      Rows::load(k, k_rows, a.c.K.token, sk.len - k_wave, lane);
      Rows::load(v, v_rows, a.c.V.token, sk.len - k_wave, lane);
      if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) *reinterpret_cast<u32x4_t*>(own + Tile::place(Rows::row(i, lane), Rows::piece(i, lane))) = k[i];
      } else {
        Rows::exchange(k);
      }
      Rows::exchange(v);
    } else {
      const int row = lane & 31;
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        k[st] = load_piece(k_rows + row * a.c.K.token, 16 * st + 8 * half, D, kj < sk.len);
        if constexpr (KEEP) *reinterpret_cast<u32x4_t*>(own + Tile::place(row, 2 * st + half)) = k[st];
        v[st] = load_piece(v_rows + row * a.c.V.token, 16 * st + 8 * half, D, kj < sk.len);
      }
    }
    f32x16_t dk[NB], dv[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.f;

    // Of the step whose loads are started next.  Last queries first: under a causal mask the tiles of a head begin together.
    const int last_q = list.first_q + (list.per_head - 1) * kQueries;
    int head = at.kv_head * a.group, q0 = last_q;
    if (list.per_head > 0) {
      head += first_step / list.per_head;
      q0 -= first_step % list.per_head * kQueries;
    }
    float row_in = 0.f;
    auto fetch = [&](int stage) {
      load.base[0] = a.c.Q.p + sq.first * a.c.Q.token + head * a.c.Q.head;
      load.base[1] = a.c.dO.p + sq.first * a.c.dO.token + head * a.c.dO.head;
      if (tid < 2 * kQueries) {  // (looked at when it is stored, a step later)
        const int row = q0 + tid % kQueries, there = row < sq.len ? row : sq.len - 1;
        row_in = (tid < kQueries ? a.c.lse : a.delta)[(int64_t)head * a.c.Tq + sq.first + there];
      }
      load.fetch(stage, q0);
    };
    if constexpr (WHOLE) {
      if constexpr (!KEEP) arrived(k);
      arrived(v);
    }
    __syncthreads();  // (a block's second key tile)
    if (first_step < end_step) fetch(0);
    for (int step = first_step; step < end_step; ++step) {
      const int stage = (step - first_step) & 1, q_now = q0;
      if (tid < 2 * kQueries) {
        // no row: a log-sum of infinity, and so probabilities of zero, and a D of zero; a query that sees no key: any finite log-sum
        const bool there = q_now + tid % kQueries < sq.len;
        const float lse2 = !there ? -kMinusInf : row_in == kMinusInf ? 0.f : row_in * kLog2e;
        rows[stage][tid / kQueries][tid % kQueries] = tid < kQueries ? lse2 : there ? row_in : 0.f;
      }
      load.settle(stage);
      load.clear_past(stage, q_now);
      __syncthreads();
      if (step + 1 < end_step) {
        q0 -= kQueries;
        if (q0 < list.first_q) { q0 = last_q; ++head; }
        fetch(stage ^ 1);
      }
      // (a wave whose keys none of these queries sees, or without keys)
      if (k_wave < sk.len && (!a.c.causal || q_now + kQueries - 1 + shift >= k_wave)) {
        const uint32_t q_tile = load.lds + (uint32_t)stage * 2 * TILE_BYTES;
        int now = lane;
        if constexpr (KEEP) asm volatile("" : "+v"(now));  // (addresses are computed here: held over the loop they would be spilled)
        const uint32_t row_at = q_tile + Tile::row_base(now), column_at = q_tile + Tile::column_base(now);
        // products in pairs: scores and dO V, then dV and dK
        auto rows_of = [&](int i) { return Tile::rows(row_at + i % 2 * TILE_BYTES, 0, i / 2); };
        auto columns_of = [&](int i) { return Tile::columns(column_at + (1 - i % 2) * TILE_BYTES, i / 2 / NB * 16, i / 2 % NB); };
        f32x16_t s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
        u32x4_t f[kAhead];
        read_ahead<2 * STEPS>(f, rows_of);
        if constexpr (KEEP) {
          const uint32_t kept_at = kept_tile + Tile::row_base(now);
          u32x4_t kf[2] = {Tile::rows(kept_at, 0, 0), Tile::rows(kept_at, 0, 1)};
          products<2 * STEPS>(f, rows_of, [&](int i, u32x4_t x) {
            if (i % 2 == 0) {
              s = mma32(x, kf[i / 2 % 2], s);
              if (i / 2 + 2 < STEPS) kf[i / 2 % 2] = Tile::rows(kept_at, 0, i / 2 + 2);
            } else {
              dp = mma32(x, v[i / 2], dp);
            }
          });
        } else {
          products<2 * STEPS>(f, rows_of, [&](int i, u32x4_t x) {
            if (i % 2 == 0) s = mma32(x, k[i / 2], s);
            else dp = mma32(x, v[i / 2], dp);
          });
        }
        read_ahead<4 * NB>(f, columns_of);
        const float* row = rows[stage][0] + 4 * half;
        if (a.c.causal && q_now + shift < k_wave + 31) {
          const int first = k_wave + (now & 31) - shift - q_now - 4 * (now >> 5);  // rows before it do not see the lane's key
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
        const u32x4_t p[2] = {acc_operand(s, 0), acc_operand(s, 1)}, ds[2] = {acc_operand(dp, 0), acc_operand(dp, 1)};
        products<4 * NB>(f, columns_of, [&](int i, u32x4_t x) {
          const int b = i / 2 % NB, st = i / 2 / NB;
          if (i % 2 == 0) dv[b] = mma32(x, p[st], dv[b]);
          else dk[b] = mma32(x, ds[st], dk[b]);
        });
      }
    }
    if (list.chunks > 1) {
      if (kj < sk.len) {
        float* to = a.part + ((((int64_t)chunk * a.c.Tk + tok) * a.c.Hkv + at.kv_head) * 2) * DP + 4 * half;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            *reinterpret_cast<float4*>(to + 32 * b + acc_row(r)) = float4{dk[b][r], dk[b][r + 1], dk[b][r + 2], dk[b][r + 3]};
            *reinterpret_cast<float4*>(to + DP + 32 * b + acc_row(r)) = float4{dv[b][r], dv[b][r + 1], dv[b][r + 2], dv[b][r + 3]};
          }
      }
    } else {
      if (kj >= sk.len) {  // (it was multiplied as a row of zeros: what came of that, infinities included, is not its gradient)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.f;
      }
      bf16_t* dk_rows = a.c.dK.p + (sk.first + k_wave) * a.c.dK.token + at.kv_head * a.c.dK.head;
      bf16_t* dv_rows = a.c.dV.p + (sk.first + k_wave) * a.c.dV.token + at.kv_head * a.c.dV.head;
      if constexpr (WHOLE) {
        Rows::store(dk_rows, a.c.dK.token, of.room - k_wave, dk, lane, a.c.scale);
        Rows::store(dv_rows, a.c.dV.token, of.room - k_wave, dv, lane, 1.f);
      } else if (kj < of.room) {
        store_column<DP>(dk_rows + (lane & 31) * a.c.dK.token, dk, lane, D, a.c.scale);
        store_column<DP>(dv_rows + (lane & 31) * a.c.dV.token, dv, lane, D, 1.f);
      }
    }
  }
}

// dK and dV of the key tiles that were cut: a wave per key and head, four elements a lane (dK on the first half of the lanes of a
// 32-element run, dV on the other).
template <int DP>
__global__ void __launch_bounds__(kThreads) grad_key_sum_kernel(const GradArgs a) {
  const int seq = blockIdx.y;
  const Sequence of = sequence(a.c, seq);
  const Span sq = of.q, sk = of.k;
  constexpr int LANES = 2 * DP / 4, PER_BLOCK = kThreads / LANES;  // lanes and rows of one (key, head)
  const int lane = threadIdx.x % LANES;
  const bool values = lane >= DP / 4;
  const int d = lane % (DP / 4) * 4;
  for (int64_t n = (int64_t)blockIdx.x * PER_BLOCK + threadIdx.x / LANES; n < (int64_t)of.room * a.c.Hkv;
       n += (int64_t)gridDim.x * PER_BLOCK) {
    const int kj = (int)(n / a.c.Hkv), head = (int)(n % a.c.Hkv);
    const int chunks = key_steps(a, kj / kRows, sq.len, sk.len).chunks;
    if (chunks == 1 || d >= a.c.D) continue;  // (written already)
    const int64_t tok = sk.first + kj;
    float4 o = {0.f, 0.f, 0.f, 0.f};
    if (kj < sk.len) {
      const float* from = a.part + ((tok * a.c.Hkv + head) * 2 + (values ? 1 : 0)) * DP + d;
      for (int c = 0; c < chunks; ++c) {
        const float4 x = *reinterpret_cast<const float4*>(from + (int64_t)c * a.c.Tk * a.c.Hkv * 2 * DP);
        o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
      }
      const float by = values ? 1.f : a.c.scale;
      o.x *= by; o.y *= by; o.z *= by; o.w *= by;
    }
    const HeadRows& to = values ? a.c.dV : a.c.dK;
    bf16_t* out = to.p + tok * to.token + head * to.head + d;
    const float v[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d + e < a.c.D) out[e] = (bf16_t)f32_to_bf16_rne(v[e]);
  }
}

// How the key tiles' steps are cut: into about two blocks' worth per compute unit, from what the call says about the lengths;
// not below 16 steps (512 queries), where the sums' way through memory would cost as much as the steps.
constexpr int kLeastSteps = 16, kMostChunks = 32;
struct KeyPlan {
  int chunk, n_chunks;
};
KeyPlan key_plan(int64_t Tk, int B, int Hkv, int group, int64_t max_q, int64_t max_k, bool causal) {
  const int64_t most = max_k > 0 ? (max_q + kQueries - 1) / kQueries * group : 0;  // steps of a key tile
  const int64_t all_tiles = Tk / kRows + B, tiles = all_tiles < (int64_t)B * ((max_k + kRows - 1) / kRows) ? all_tiles : (int64_t)B * ((max_k + kRows - 1) / kRows);
  const int64_t total = tiles * Hkv * (causal ? (most + 1) / 2 : most);
  int64_t chunk = (total + kKeyBlocks - 1) / kKeyBlocks;
  chunk = chunk < kLeastSteps ? kLeastSteps : chunk;
  if ((most + chunk - 1) / chunk > kMostChunks) chunk = (most + kMostChunks - 1) / kMostChunks;
  KeyPlan p;
  p.chunk = (int)(chunk < (1 << 30) ? chunk : 1 << 30);
  p.n_chunks = (int)((most + p.chunk - 1) / p.chunk);
  if (p.n_chunks < 1) p.n_chunks = 1;
  return p;
}

int tiles(int64_t most, int B, int Hkv, int group) {
  int n = (int)((most + kRows - 1) / kRows);
  if (n < 1) n = 1;
  while (tile_blocks(B, Hkv, group, n) >= kMostBlocks) n = (n + 1) / 2;
  return n;
}

}  // namespace

size_t attention_grad_workspace_bytes(int64_t Tq, int64_t Tk, int B, int Hq, int Hkv, int D, int64_t max_q, int64_t max_k,
                                      bool causal) {
  const KeyPlan p = key_plan(Tk, B, Hkv, Hq / Hkv, max_q, max_k, causal);
  const size_t parts = p.n_chunks > 1 ? (size_t)p.n_chunks * Tk * Hkv * 2 * padded_head(D) * sizeof(float) : 0;
  return round256((size_t)Tq * Hq * sizeof(float)) + parts;
}

hipError_t launch_attention_grad(const AttentionCall& c, hipStream_t s) {
  GradArgs a = {};
  a.c = c;
  a.group = c.Hq / c.Hkv;
  a.scale_log2 = c.scale * kLog2e;
  const KeyPlan plan = key_plan(c.Tk, c.B, c.Hkv, a.group, c.max_q, c.max_k, c.causal);
  a.chunk = plan.chunk;
  a.n_chunks = plan.n_chunks;
  a.n_q_tiles = tiles(c.max_q, c.B, c.Hkv, a.group);
  a.n_k_tiles = tiles(c.max_k, c.B, c.Hkv, a.n_chunks);
  a.delta = static_cast<float*>(c.workspace);
  a.part = a.delta + round256((size_t)c.Tq * c.Hq * sizeof(float)) / sizeof(float);
  const HeadRows* all[] = {&c.Q, &c.K, &c.V, &c.O, &c.dO, &c.dQ, &c.dK, &c.dV};
  with_head(c.D, std::all_of(std::begin(all), std::end(all), [](const HeadRows* r) { return whole_rows(*r); }), [&](auto dp, auto whole) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool WHOLE = decltype(whole)::value;
    const int64_t q_blocks = tile_blocks(c.B, c.Hkv, a.group, a.n_q_tiles);
    grad_query_kernel<DP, WHOLE><<<dim3((unsigned)q_blocks), kThreads, 0, s>>>(a);
    if (c.Tk == 0) return;
    const int64_t k_blocks = tile_blocks(c.B, c.Hkv, a.n_chunks, a.n_k_tiles);
    grad_key_kernel<DP, WHOLE><<<dim3((unsigned)k_blocks), kThreads, 0, s>>>(a);
    if (a.n_chunks > 1) {
      constexpr int PER_BLOCK = kThreads / (2 * DP / 4);
      int64_t blocks = (c.max_k * c.Hkv + PER_BLOCK - 1) / PER_BLOCK;
      blocks = blocks < 1 ? 1 : blocks < 4096 ? blocks : 4096;
      grad_key_sum_kernel<DP><<<dim3((unsigned)blocks, (unsigned)c.B), kThreads, 0, s>>>(a);
    }
  });
  return hipGetLastError();
}

}  // namespace nm
