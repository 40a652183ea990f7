// Softmax attention over packed sequences, grouped heads, causal or not.  For query i of a sequence of Lq queries and Lk keys
// and each of the query heads that share key head h
//
//   s_j = scale q_i . k_j for the keys it sees (all, or j <= i + Lk - Lq),  o_i = sum_j exp(s_j - lse_i) v_j,
//   lse_i = log sum_j exp(s_j);   a query that sees no key gets o_i = 0 and lse_i = -infinity.
//
// One pass over the keys with a running maximum and sum; scores, maximum, sum and output are 32-bit floats, the
// probabilities are rounded to bfloat16 as operands of the second product (as the values are; the sum takes them unrounded).
//
// Two kernels.  prompt_kernel: a block of four waves takes 128 queries of one head, 32 to a wave, and walks over the keys 64
// at a time, staged in LDS for its waves.  cache_kernel, where queries are few: its columns are the (query, head of the
// group) pairs that share a key head, its waves walk over different keys, and keys are cut into chunks for different blocks;
// what they leave (output, maximum, sum) a second launch joins in order.
//
// Measured: two causal prompts of 8191 and 342, 16 heads on 4 of 128: 278 us, 990 TFLOP/s of useful products, bound by issue: a tile
// of 64 keys is 32 matrix instructions and 150 others to a wave, two waves a SIMD.  256 images of 197 tokens, 12 heads of 64: 310 MB in
// 92 to 97 us by the card, where loads, stores and products, of four tiles to a block, are 55, 25 and 75 alone (no deeper staging, nor
// blocks that take several tiles with the next one's loads under way, overlaps them better).  24 caches of 1 to 16384 keys, 32 heads on
// 8 of 128: 337 MB in 71 us, 4.7 TB/s, and 5 for the join: bound by memory, and by how evenly chunks of unknown lengths go round.
#include "nm_attention.h"

namespace nm {

namespace {

struct AttnArgs {
  AttentionCall c;
  int group;          // Hq / Hkv
  float scale_log2;   // scale * log2(e)
  int n_tiles;        // prompt: query tiles the grid has per head
  int chunk;          // cache: keys per block
  int n_chunks, n_row_tiles;
  float* part_o;      // cache: [column][chunk][DP], column = query * Hq + head
  float2* part_ml;    // [column][chunk]: (maximum of the scaled scores in the exponent's base 2, sum)
};

constexpr int kKeys = 64;             // per tile
constexpr int kQueries = kWaves * 32; // per block

template <int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 2) prompt_kernel(const AttnArgs a) {
  using Tile = RowTile<DP>;
  constexpr int NB = DP / 32, STEPS = DP / 16, TILE_BYTES = kKeys * Tile::kRowBytes;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2][2 * TILE_BYTES];  // two stages of keys and values
  TilePlace at;
  if (!tile_place(a.c.B, a.c.Hkv, a.group, a.n_tiles, true, a.c.causal, &at)) return;
  const int kv_head = at.kv_head, head = kv_head * a.group + at.sub, seq = at.seq;
  const int D = WHOLE ? DP : a.c.D;
  const Sequence of = sequence(a.c, seq);
  const Span sq = of.q, sk = of.k;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int shift = sk.len - sq.len;  // causal: query i sees keys up to i + shift
  TilePair<DP, kKeys, WHOLE, kThreads> load;
  load.base[0] = a.c.K.p + sk.first * a.c.K.token + kv_head * a.c.K.head;
  load.base[1] = a.c.V.p + sk.first * a.c.V.token + kv_head * a.c.V.head;
  load.stride[0] = a.c.K.token;
  load.stride[1] = a.c.V.token;
  load.rows = sk.len;
  load.D = D;
  load.smem = smem[0];
  load.lds = NM_LDS_ADDRESS(smem[0]);

  for (int tile = at.tile; (int64_t)tile * kQueries < sq.len; tile += a.n_tiles) {
    const int q_wave = tile * kQueries + wave * 32;
    const int qi = q_wave + (lane & 31);
    const bool live = qi < sq.len;
    const bf16_t* q_row = a.c.Q.p + (sq.first + qi) * a.c.Q.token + head * a.c.Q.head;
    // keys that any query of the block, of the wave, and this lane's sees
    const int last_q = (tile + 1) * kQueries < sq.len ? (tile + 1) * kQueries : sq.len;
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
    float ref = kMinusInf, sum = 0.f;

    const int n_key_tiles = (end + kKeys - 1) / kKeys;
    __syncthreads();  // (a block's second query tile: the first one's keys are no longer read)
    if (n_key_tiles > 0) load.fetch(0, 0);
    u32x4_t q[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) q[st] = load_piece(q_row, 16 * st + 8 * half, D, live);
    if constexpr (WHOLE) arrived(q);
    for (int kt = 0; kt < n_key_tiles; ++kt) {
      const int k0 = kt * kKeys;
      load.settle(kt & 1);
      if (kt + 1 < n_key_tiles) {
        __syncthreads();
        load.fetch((kt + 1) & 1, k0 + kKeys);
      } else {
        load.clear_past(kt & 1, k0);
        __syncthreads();
      }
      if (k0 < wave_end) {
        const uint32_t k_tile = load.lds + (uint32_t)(kt & 1) * 2 * TILE_BYTES, v_tile = k_tile + TILE_BYTES;
        const uint32_t k_at = k_tile + Tile::row_base(lane), v_at = v_tile + Tile::column_base(lane);
        constexpr int NS = kKeys / 32 * STEPS, NV = kKeys / 16 * NB;
        // (products on the same sums wait for each other: the two runs of keys in turn)
        constexpr int KB = kKeys / 32;
        auto keys = [&](int i) { return Tile::rows(k_at, i % KB * 32, i / KB); };
        auto values = [&](int i) { return Tile::columns(v_at, i / NB * 16, i % NB); };
        f32x16_t s[kKeys / 32];
#pragma unroll
        for (int kb = 0; kb < kKeys / 32; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
        u32x4_t f[kAhead];
        read_ahead<NS>(f, keys);
        products<NS>(f, keys, [&](int i, u32x4_t k) { s[i % KB] = mma32(k, q[i / KB], s[i % KB]); });
        read_ahead<NV>(f, values);
        if (k0 + kKeys > first_hidden) {
#pragma unroll
          for (int kb = 0; kb < kKeys / 32; ++kb) hide_rows(s[kb], limit - k0 - 32 * kb - 4 * half);
        }
        softmax_step(s, a.scale_log2, ref, sum, acc);
        u32x4_t p[kKeys / 16];
#pragma unroll
        for (int st = 0; st < kKeys / 16; ++st) p[st] = acc_operand(s[st / 2], st % 2);
        products<NV>(f, values, [&](int i, u32x4_t v) { acc[i % NB] = mma32(v, p[i / NB], acc[i % NB]); });
      }
    }
    sum = half_sum(sum);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    bf16_t* o_rows = a.c.O.p + (sq.first + q_wave) * a.c.O.token + head * a.c.O.head;
    if constexpr (WHOLE) WaveRows<DP>::store(o_rows, a.c.O.token, sq.len - q_wave, acc, lane, inv);
    if (live) {
      if constexpr (!WHOLE) store_column<DP>(o_rows + (lane & 31) * a.c.O.token, acc, lane, D, inv);
      if (a.c.lse != nullptr && half == 0)
        a.c.lse[(int64_t)head * a.c.Tq + sq.first + qi] = sum == 0.f ? kMinusInf : (ref + log2f(sum)) * kLn2;
    }
  }
}

// Number `n` of all chunks of all sequences, in order: the sequence and its chunk.  A sequence has as many chunks as its keys
// need (one at least, at most n_chunks, the last of which takes the rest); their counts are added up 64 sequences at a time.
__device__ __forceinline__ bool find_chunk(const AttnArgs& a, int64_t n, int* seq, int* chunk) {
  if (a.n_chunks == 1) {
    *seq = (int)n;
    *chunk = 0;
    return n < a.c.B;
  }
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < a.c.B; b0 += 64) {
    const int b = b0 + lane;
    int count = 0;
    if (b < a.c.B) {
      int64_t lo = 0, hi = a.c.Tk;
      if (a.c.offsets_k != nullptr) {
        lo = a.c.offsets_k[b];
        hi = a.c.offsets_k[b + 1];
      }
      int64_t len = hi - lo;
      if (a.c.lengths_k != nullptr && a.c.lengths_k[b] < len) len = a.c.lengths_k[b];
      const int64_t need = (len + a.chunk - 1) / a.chunk;  // (of offsets that lie: some number; the keys are checked later)
      count = (int)(need < 1 ? 1 : need < a.n_chunks ? need : a.n_chunks);
    }
    int upto = count;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int before = __shfl_up(upto, m, 64);
      if (lane >= m) upto += before;
    }
    const int total = __builtin_amdgcn_readlane(upto, 63);
    if (n < total) {
      const int at = __ffsll((unsigned long long)__ballot(upto > n)) - 1;
      *seq = b0 + at;
      *chunk = (int)n - (__shfl(upto, at, 64) - __shfl(count, at, 64));
      *seq = __builtin_amdgcn_readfirstlane(*seq);
      *chunk = __builtin_amdgcn_readfirstlane(*chunk);
      return true;
    }
    n -= total;
  }
  return false;
}

// Few queries.  Column n of a row tile is query (32 tile + n) / group of the sequence and head (32 tile + n) % group of the
// key head's group.  As many blocks as the chip holds take the chunks, row tiles and key heads in turn (a grid with a block for
// every chunk that there might be had most of them empty where lengths differ, and each of those held a compute unit's LDS:
// 24 caches of up to 16k 223 us, 73 so).  Each wave takes every fourth run of 32 keys of the chunk through LDS of its own.
template <int DP, bool WHOLE>
__global__ void __launch_bounds__(kThreads, WHOLE && DP == 128 ? 1 : 2) cache_kernel(const AttnArgs a) {
  using Tile = RowTile<DP>;
  using Load = TilePair<DP, 32, WHOLE, 64>;
  constexpr int NB = DP / 32, STEPS = DP / 16, RUN = 32, TILE_BYTES = Load::kBytes;
  constexpr int JOIN = 32 * (DP + 4) * 4;  // one wave's output, columns padded against bank conflicts
  constexpr int OWN = (WHOLE ? 2 : 1) * 2 * TILE_BYTES;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kWaves * (OWN > JOIN ? OWN : JOIN)];
  __shared__ float2 wave_ml[kWaves][32];
  const int D = WHOLE ? DP : a.c.D;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const bool alone = a.n_chunks == 1;
  const int per_chunk = a.n_row_tiles * a.c.Hkv;
  for (int64_t item = blockIdx.x; ; item += gridDim.x) {
    int seq, chunk;
    if (!find_chunk(a, item / per_chunk, &seq, &chunk)) return;
    const int kv_head = (int)(item % per_chunk) % a.c.Hkv, row_tile0 = (int)(item % per_chunk) / a.c.Hkv;
    const Sequence of = sequence(a.c, seq);
    const Span sq = of.q, sk = of.k;
    const int shift = sk.len - sq.len;
    const int first_key = chunk * a.chunk;
    const int end_key = chunk == a.n_chunks - 1 || first_key + a.chunk > sk.len ? sk.len : first_key + a.chunk;
    Load load;
    load.base[0] = a.c.K.p + sk.first * a.c.K.token + kv_head * a.c.K.head;
    load.base[1] = a.c.V.p + sk.first * a.c.V.token + kv_head * a.c.V.head;
    load.stride[0] = a.c.K.token;
    load.stride[1] = a.c.V.token;
    load.rows = end_key;
    load.D = D;
    load.smem = smem + wave * OWN;
    load.lds = NM_LDS_ADDRESS(smem) + wave * OWN;
    const int64_t columns = (int64_t)sq.len * a.group;
    for (int row_tile = row_tile0; (int64_t)row_tile * 32 < columns; row_tile += a.n_row_tiles) {
      const int64_t n = (int64_t)row_tile * 32 + col;
      const bool live = n < columns;
      const int qi = (int)(n / a.group), head = kv_head * a.group + (int)(n % a.group);
      const bf16_t* q_row = a.c.Q.p + (sq.first + qi) * a.c.Q.token + head * a.c.Q.head;
      u32x4_t q[STEPS];
#pragma unroll
      for (int st = 0; st < STEPS; ++st) q[st] = load_piece(q_row, 16 * st + 8 * half, D, live);
      int limit = end_key, first_hidden = end_key, end = end_key;  // keys that this lane, all lanes, any lane sees
      if (a.c.causal) {
        auto upto = [&](int64_t column) { const int n = (int)(column / a.group) + shift + 1; return n < end_key ? n : end_key; };
        limit = upto(n);
        first_hidden = upto((int64_t)row_tile * 32);
        end = upto((int64_t)row_tile * 32 + 31 < columns ? (int64_t)row_tile * 32 + 31 : columns - 1);
      }
      f32x16_t acc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;
      float ref = kMinusInf, sum = 0.f;
      __syncthreads();  // (a further row tile: what the waves joined has been read)
      int k0 = first_key + wave * RUN, stage = 0;
      if (k0 < end) load.fetch(0, k0);
      if constexpr (WHOLE) arrived(q);
      for (; k0 < end; k0 += kWaves * RUN) {
        // asynchronous copies go to the other stage while this one is worked on; what comes through registers waits there
        const bool more = k0 + kWaves * RUN < end;
        if constexpr (WHOLE) {
          if (more) {
            load.fetch(stage ^ 1, k0 + kWaves * RUN);
            load.template settle<2 * Load::kLoads>(stage);
          } else {
            load.settle(stage);
            load.clear_past(stage, k0);
          }
        } else {
          load.settle(0);
          if (more) load.fetch(0, k0 + kWaves * RUN);
        }
        __builtin_amdgcn_wave_barrier();
        const uint32_t tile = load.lds + (uint32_t)stage * 2 * TILE_BYTES;
        const uint32_t k_at = tile + Tile::row_base(lane), v_at = tile + TILE_BYTES + Tile::column_base(lane);
        if constexpr (WHOLE) stage ^= 1;
        constexpr int NV = RUN / 16 * NB;
        auto keys = [&](int i) { return Tile::rows(k_at, 0, i); };
        auto values = [&](int i) { return Tile::columns(v_at, i / NB * 16, i % NB); };
        f32x16_t s[1];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[0][r] = 0.f;
        u32x4_t f[kAhead];
        read_ahead<STEPS>(f, keys);
        products<STEPS>(f, keys, [&](int i, u32x4_t k) { s[0] = mma32(k, q[i], s[0]); });
        read_ahead<NV>(f, values);
        if (k0 + RUN > first_hidden) hide_rows(s[0], limit - k0 - 4 * half);
        softmax_step(s, a.scale_log2, ref, sum, acc);
        const u32x4_t p[2] = {acc_operand(s[0], 0), acc_operand(s[0], 1)};
        products<NV>(f, values, [&](int i, u32x4_t v) { acc[i % NB] = mma32(v, p[i / NB], acc[i % NB]); });
        __builtin_amdgcn_wave_barrier();
      }
      // join the four waves: each scales its output to the common maximum, then the block adds them in wave order
      sum = half_sum(sum);
      if (half == 0) wave_ml[wave][col] = float2{ref, sum};
      __syncthreads();
      float top = kMinusInf, total = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, wave_ml[w][col].x);
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        total += wave_ml[w][col].y * part_weight(wave_ml[w][col].x, top);
      const float by = part_weight(ref, top);
      float* joined = reinterpret_cast<float*>(smem) + wave * 32 * (DP + 4);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<float4*>(joined + col * (DP + 4) + 32 * b + acc_row(r) + 4 * half) =
              float4{acc[b][r] * by, acc[b][r + 1] * by, acc[b][r + 2] * by, acc[b][r + 3] * by};
      __syncthreads();
      // lane -> (column, four elements)
      constexpr int PER_COL = DP / 4;
#pragma unroll
      for (int i = 0; i < 32 * PER_COL / kThreads; ++i) {
        const int at = i * kThreads + tid, c = at / PER_COL, d = at % PER_COL * 4;
        const int64_t cn = (int64_t)row_tile * 32 + c;
        if (cn >= columns || d >= D) continue;
        const float* from = reinterpret_cast<const float*>(smem) + c * (DP + 4) + d;
        float4 o = *reinterpret_cast<const float4*>(from);
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
          const float4 x = *reinterpret_cast<const float4*>(from + w * 32 * (DP + 4));
          o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
        }
        const int64_t tok = sq.first + cn / a.group;
        const int hd = kv_head * a.group + (int)(cn % a.group);
        if (alone) {
          float t = kMinusInf, l = 0.f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) t = fmaxf(t, wave_ml[w][c].x);
#pragma unroll
          for (int w = 0; w < kWaves; ++w) l += wave_ml[w][c].y * part_weight(wave_ml[w][c].x, t);
          const float inv = l == 0.f ? 0.f : 1.f / l;
          store4(a.c.O.p + tok * a.c.O.token + hd * a.c.O.head, d, D, pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
        } else {
          *reinterpret_cast<float4*>(a.part_o + ((tok * a.c.Hq + hd) * a.n_chunks + chunk) * DP + d) = o;
        }
      }
      if (wave == 0 && half == 0 && live) {
        const int64_t tok = sq.first + qi;
        if (!alone) a.part_ml[(tok * a.c.Hq + head) * a.n_chunks + chunk] = float2{top, total};
        else if (a.c.lse != nullptr)
          a.c.lse[(int64_t)head * a.c.Tq + tok] = total == 0.f ? kMinusInf : (top + log2f(total)) * kLn2;
      }
    }
  }
}

// Joins the chunks of a column: a wave per (query, head).  DP / 4 lanes take four elements each of every (256 / DP)-th chunk, so
// that several chunks' loads are under way; the shares are added in a fixed order.
template <int DP>
__global__ void __launch_bounds__(kThreads) cache_join_kernel(const AttnArgs a) {
  constexpr int LANES = DP / 4, GROUPS = 64 / LANES;
  const int lane = threadIdx.x & 63, part = lane / LANES, d = lane % LANES * 4;
  const int seq = blockIdx.y;
  const Sequence of = sequence(a.c, seq);
  const int used = (of.k.len + a.chunk - 1) / a.chunk;
  const int chunks = used < 1 ? 1 : used < a.n_chunks ? used : a.n_chunks;
  for (int64_t i = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); i < (int64_t)of.q.len * a.c.Hq; i += (int64_t)gridDim.x * kWaves) {
    const int64_t tok = of.q.first + i / a.c.Hq;
    const int head = (int)(i % a.c.Hq);
    const int64_t at = (tok * a.c.Hq + head) * a.n_chunks;
    float top = kMinusInf;
    for (int k = lane; k < chunks; k += 64) top = fmaxf(top, a.part_ml[at + k].x);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
    float total = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = part; k < chunks; k += GROUPS) {
      const float2 ml = a.part_ml[at + k];
      const float by = part_weight(ml.x, top);
      total = fmaf(ml.y, by, total);
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a.part_o + (at + k) * DP + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = d + e < a.c.D ? fmaf(x[e], by, o[e]) : 0.f;
    }
#pragma unroll
    for (int m = LANES; m < 64; m <<= 1) {
      total += __shfl_xor(total, m, 64);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m, 64);
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    if (part == 0)
      store4(a.c.O.p + tok * a.c.O.token + head * a.c.O.head, d, a.c.D, pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    if (a.c.lse != nullptr && lane == 0)
      a.c.lse[(int64_t)head * a.c.Tq + tok] = total == 0.f ? kMinusInf : (top + log2f(total)) * kLn2;
  }
}

// How a call is cut: few queries per key head take the cache kernel.
// It serves up to kFewColumns (query, head) pairs to a key head: 24 caches of 16k, 32 heads on 8, 128 pairs 570 us and 686 by the
// prompt kernel, 256 pairs 924 and 790, since it passes over the keys once for every 32.  It also serves any number of them in up to
// kFewBlocks blocks (32 columns each, waves on different keys), where a prompt's blocks of 128 leave most of the chip idle: one image
// of 12 heads, 84 blocks, 6.8 us and 8.0; 16 heads on 4 of 128, 256 tokens (128 blocks) 9.5 and 10.1, 512 tokens 25 and 15.
constexpr int64_t kFewColumns = 128, kFewBlocks = 128, kLeastChunk = 512, kCacheBlocks = 3072, kCutSequences = 512;
struct CachePlan {
  bool taken;
  int chunk, n_chunks, n_row_tiles;
  int64_t most_chunks;  // n_chunks of any number of keys up to max_k: n_chunks itself falls where chunks are rounded up to 128 keys
};
CachePlan cache_plan(int B, int Hkv, int group, int64_t max_q, int64_t max_k) {
  CachePlan p = {};
  const int64_t row_tiles = (max_q * group + 31) / 32, blocks = (int64_t)B * Hkv * row_tiles;
  p.taken = max_q * group <= kFewColumns || blocks <= kFewBlocks;
  if (!p.taken) return p;
  p.n_row_tiles = (int)(row_tiles > 0 ? row_tiles : 1);
  // chunks of at least 512 keys (one cache of 16k 22 us, 28 with 256; four 59 and 73), about kCacheBlocks of them if all sequences were
  // of the longest length: most are shorter (24 of them, a fifth full, 77 us, with 1536 84, with 768 122; all full 305, 296, 288).
  // None where there are sequences enough to go round (finding a chunk means adding up all of theirs).
  int64_t chunk = (max_k * blocks + kCacheBlocks - 1) / kCacheBlocks;
  chunk = (chunk < kLeastChunk ? kLeastChunk : chunk + 127) / 128 * 128;
  p.chunk = (int)chunk;
  p.n_chunks = (int)((max_k + chunk - 1) / chunk);
  // (a chunk has kLeastChunk keys or more, and no fewer than max_k * blocks / kCacheBlocks)
  const int64_t by_least = (max_k + kLeastChunk - 1) / kLeastChunk, by_blocks = blocks > 0 ? (kCacheBlocks + blocks - 1) / blocks : by_least;
  p.most_chunks = by_least < by_blocks ? by_least : by_blocks;
  if (p.n_chunks < 1 || B > kCutSequences) p.n_chunks = 1;
  if (p.most_chunks < 1 || B > kCutSequences) p.most_chunks = 1;
  return p;
}

}  // namespace

namespace {
size_t chunks_bytes(int64_t Tq, int Hq, int D, int64_t n_chunks) {
  if (n_chunks <= 1) return 0;
  const size_t columns = (size_t)Tq * Hq * n_chunks;
  return round256(columns * padded_head(D) * sizeof(float)) + columns * sizeof(float2);
}
}  // namespace

size_t attention_workspace_bytes(int64_t Tq, int B, int Hq, int Hkv, int D, int64_t max_q, int64_t max_k) {
  const CachePlan p = cache_plan(B, Hkv, Hq / Hkv, max_q, max_k);
  return chunks_bytes(Tq, Hq, D, p.taken ? p.n_chunks : 1);
}
size_t attention_workspace_most(int64_t Tq, int B, int Hq, int Hkv, int D, int64_t max_q, int64_t max_k) {
  const CachePlan p = cache_plan(B, Hkv, Hq / Hkv, max_q, max_k);
  return chunks_bytes(Tq, Hq, D, p.taken ? p.most_chunks : 1);
}

hipError_t launch_attention(const AttentionCall& c, hipStream_t s) {
  AttnArgs a = {};
  a.c = c;
  a.group = c.Hq / c.Hkv;
  a.scale_log2 = c.scale * kLog2e;
  int cus = 0;
  if (hipError_t e = compute_units(&cus); e != hipSuccess) return e;
  const CachePlan plan = cache_plan(c.B, c.Hkv, a.group, c.max_q, c.max_k);
  a.chunk = plan.chunk; a.n_chunks = plan.n_chunks; a.n_row_tiles = plan.n_row_tiles;
  a.n_tiles = (int)((c.max_q + kQueries - 1) / kQueries);
  if (a.n_tiles < 1) a.n_tiles = 1;
  while (tile_blocks(c.B, c.Hkv, a.group, a.n_tiles) >= kMostBlocks) a.n_tiles = (a.n_tiles + 1) / 2;  // (blocks take several then)
  if (plan.n_chunks > 1) {
    a.part_o = static_cast<float*>(c.workspace);
    const size_t columns = (size_t)c.Tq * c.Hq * plan.n_chunks;
    a.part_ml = reinterpret_cast<float2*>(static_cast<unsigned char*>(c.workspace) +
                                          round256(columns * padded_head(c.D) * sizeof(float)));
  }
  const bool whole_keys = whole_rows(c.K) && whole_rows(c.V);
  if (plan.taken) {
    with_head(c.D, whole_keys, [&](auto dp, auto whole) {
      constexpr int DP = decltype(dp)::value;
      constexpr bool WHOLE = decltype(whole)::value;
      // (one, two or four blocks to a compute unit, as registers and LDS allow)
      const int64_t items = (int64_t)plan.n_chunks * plan.n_row_tiles * c.B * c.Hkv, room = (int64_t)cus * (DP == 128 ? (WHOLE ? 1 : 2) : DP == 64 ? 2 : 4);
      cache_kernel<DP, WHOLE><<<dim3((unsigned)(items < room ? items : room)), kThreads, 0, s>>>(a);
      if (a.n_chunks > 1) {
        const int64_t waves = c.max_q * c.Hq, most = (waves + kWaves - 1) / kWaves;
        const dim3 join((unsigned)(most < 1 ? 1 : most), (unsigned)c.B);
        cache_join_kernel<DP><<<join, kThreads, 0, s>>>(a);
      }
    });
  } else {
    with_head(c.D, whole_keys && whole_rows(c.Q) && whole_rows(c.O), [&](auto dp, auto whole) {
      const int64_t blocks = tile_blocks(c.B, c.Hkv, a.group, a.n_tiles);
      prompt_kernel<decltype(dp)::value, decltype(whole)::value><<<dim3((unsigned)blocks), kThreads, 0, s>>>(a);
    });
  }
  return hipGetLastError();
}

}  // namespace nm
