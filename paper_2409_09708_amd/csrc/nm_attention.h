// What the attention kernels share: sequences, tiles of rows in LDS and the fragments that the 32 x 32 matrix instruction
// takes from them.
//
// Scores are computed transposed, S^T = K Q^T (or S = Q K^T where the keys stay put), so that a lane holds values of one
// column -- one query (one key) -- in the accumulator layout of v_mfma_f32_32x32x16_bf16: lane l has column l % 32, and its
// register r row 8 (r / 4) + 4 (l / 32) + r % 4.  A softmax over the rows is then a reduction over the lane's own registers
// and its partner 32 lanes away, and the probabilities are, rounded to bfloat16, already the second operand of the next
// product: of a run of 16 rows the instruction wants 8 from each half of the wave, in any order that its first operand
// shares, and registers 8 s .. 8 s + 7 are rows {0 .. 3, 8 .. 11} + 4 (l / 32) of run s.  The first operand is read in that
// order by the transposing LDS read.
#ifndef NM_ATTENTION_H
#define NM_ATTENTION_H

#include "nm_launch.h"
#include "nm_mma.h"
#include "nm_rows.h"

#include <type_traits>

namespace nm {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t* lds_i16x4_ptr;
typedef __attribute__((address_space(3))) const u32x4_t* lds_u32x4_ptr;
typedef __attribute__((address_space(3))) u32x4_t* lds_u32x4_out_ptr;

__device__ __forceinline__ f32x16_t mma32(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// row of register r in the accumulator, without the lane's 4 (lane / 32)
__host__ __device__ constexpr int acc_row(int r) { return 8 * (r / 4) + r % 4; }

// N products whose first operands come from LDS, read kAhead of them ahead of their use and in just this order: left to
// itself the compiler reads an operand right before the product that takes it, to spare registers, and waits for it.
constexpr int kAhead = 4;
template <int N, class Load>
__device__ __forceinline__ void read_ahead(u32x4_t (&f)[kAhead], Load load) {
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (i < N) f[i] = load(i);
  __builtin_amdgcn_sched_barrier(0);
}
template <int N, class Load, class Use>
__device__ __forceinline__ void products(u32x4_t (&f)[kAhead], Load load, Use use) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    use(i, f[i % kAhead]);
    if (i + kAhead < N) f[i % kAhead] = load(i + kAhead);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The value of the lane 32 away, combined.
__device__ __forceinline__ float half_max(float v) { return fmaxf(v, __shfl_xor(v, 32, 64)); }
__device__ __forceinline__ float half_sum(float v) { return v + __shfl_xor(v, 32, 64); }

// exp2 of a difference: the hardware instruction, whose results below 2^-126 are zero
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMinusInf = -__builtin_huge_valf();

// Sequence b of the packed tensors: first rows and lengths, of the keys those in use and the rows that belong to them.  Offsets
// are the caller's; whatever they hold, rows stay inside the tensors.  Five lanes read the five numbers at once, with one wait.
struct Span {
  int64_t first;
  int len;
};
struct Sequence {
  Span q, k;
  int room;
};
__device__ __forceinline__ Sequence sequence(const AttentionCall& c, int b) {
  const int lane = threadIdx.x & 63;
  const int32_t* from = lane < 2 ? c.offsets_q : lane < 4 ? c.offsets_k : c.lengths_k;
  int v = lane == 1 ? (int)c.Tq : lane == 3 ? (int)c.Tk : lane == 4 ? 0x7FFFFFFF : 0;
  if (lane < 5 && from != nullptr) v = from[b + (lane < 4 ? lane & 1 : 0)];
  auto within = [](int x, int lo, int hi) { return x < lo ? lo : x < hi ? x : hi; };
  const int q0 = within(__builtin_amdgcn_readlane(v, 0), 0, (int)c.Tq), q1 = within(__builtin_amdgcn_readlane(v, 1), q0, (int)c.Tq);
  const int k0 = within(__builtin_amdgcn_readlane(v, 2), 0, (int)c.Tk), k1 = within(__builtin_amdgcn_readlane(v, 3), k0, (int)c.Tk);
  const int used = within(__builtin_amdgcn_readlane(v, 4), 0, k1 - k0);
  return {{q0, q1 - q0}, {k0, used}, k1 - k0};
}

// A tile of rows of DP bfloat16 in LDS.  The 16-byte pieces of a row are permuted so that both ways of reading it touch every
// bank once: 16 rows at one piece (fragments of rows), and runs of four pieces from four rows (transposing reads).
template <int DP>
struct RowTile {
  static constexpr int kRowBytes = DP * 2, kPieces = DP / 8;
  static __host__ __device__ constexpr int swizzle(int row) {
    return DP == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : DP == 64 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : (row >> 2) & 3;
  }
  static __device__ __forceinline__ int place(int row, int piece) { return row * kRowBytes + ((piece ^ swizzle(row)) << 4); }

  // Operands from the tile at LDS address `tile` (a multiple of 256).  An operand's address is a lane's own constant with a few
  // bits changed, one instruction each, so that none is kept.
  //   rows     elements 16 step + 8 (lane / 32) .. + 7 of row row0 + lane % 32 (row0 a multiple of 32);  at = tile + row_base(lane)
  //   columns  columns 32 block .. + 31 of rows row0 .. row0 + 15 (row0 a multiple of 16) as the first operand, rows in the order
  //            {0 .. 3, 8 .. 11} + 4 (lane / 32);  at = tile + column_base(lane)
  static __device__ __forceinline__ uint32_t row_base(int lane) { return place(lane & 31, lane >> 5); }
  static __device__ __forceinline__ uint32_t column_base(int lane) {
    return place(4 * (lane >> 5) + ((lane >> 2) & 3), 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) + (lane & 1) * 8;
  }
  static __device__ __forceinline__ u32x4_t rows(uint32_t at, int row0, int step) {
    return *(lds_u32x4_ptr)(uintptr_t)((at ^ (step << 5)) + row0 * kRowBytes);
  }
  static __device__ __forceinline__ u32x4_t columns(uint32_t at, int row0, int block) {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    const uint32_t lo = (at ^ (block << 6)) + row0 * kRowBytes, hi = (at ^ (block << 6) ^ 32) + (row0 + 8) * kRowBytes;
    const u32x2_t l = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(uintptr_t)lo));
    const u32x2_t h = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(uintptr_t)hi));
    return u32x4_t{l[0], l[1], h[0], h[1]};
  }
};

constexpr int kWaves = 4, kThreads = kWaves * 64;

// Eight elements of a row, zeros past element D or where `there` is false.  Any alignment.
__device__ __forceinline__ u32x4_t load_piece(const bf16_t* row, int d, int D, bool there) {
  Raw8<false> r;
  r.load(row, d, there ? D - d : 0);
  return r.v[0];
}

// Two tiles of ROWS rows (of keys and values, or of queries and dO) from memory to LDS, by LANES lanes: a block of kThreads, or a
// wave.
// WHOLE (rows of exactly DP elements, all 16-byte aligned): asynchronous copies straight to LDS, one wave-load a kilobyte; rows past
// the last one repeat it, so the scores of those have to be hidden, and they must not be summed (clear_past).  Otherwise through
// registers, with zeros past the last row and the last element.
//   fetch(stage, row0)       starts the loads of a tile (rows row0 .., one of them there at least)
//   settle(stage)            the tile is in LDS, as far as this wave brought it, up to LATER copies started after it: a block's
//                            barrier follows
//   clear_past(stage, row0)  between the two, where the second tile's rows are summed: zeros for those past the last one, again as far
//                            as this wave brought them.  (Their weight is zero, and zero times an infinity in the last row is NaN.)
template <int DP, int ROWS, bool WHOLE, int LANES>
struct TilePair {
  using Tile = RowTile<DP>;
  static constexpr int kBytes = ROWS * Tile::kRowBytes, kPieces = ROWS * Tile::kPieces;
  static constexpr int kWide = LANES / 64, kLoads = (kPieces + LANES - 1) / LANES;
  const bf16_t* base[2];  // row 0 of the sequence and head
  int64_t stride[2];
  int rows, D;            // of the sequence
  unsigned char* smem;    // stages of 2 * kBytes
  uint32_t lds;           // its address
  u32x4_t in[WHOLE ? 1 : 2][WHOLE ? 1 : kLoads];

  __device__ __forceinline__ void fetch(int stage, int row0) {
    const int tid = threadIdx.x % LANES;
    if constexpr (WHOLE) {
      const int wave = kWide == 1 ? 0 : (int)__builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (uint32_t)stage * 2 * kBytes);
      const int last = rows - 1 - row0;  // >= 0
      if (kPieces % LANES == 0 || wave * 64 < kPieces) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uniform_ptr_t from = make_uniform(base[t] + (int64_t)row0 * stride[t]);
          const uint32_t bytes = (uint32_t)stride[t] * 2;
#pragma unroll
          for (int n = 0; n < kLoads; ++n) {
            const int i = (n * kWide + wave) * 64 + lane;
            int row = i / Tile::kPieces;
            const int piece = (i % Tile::kPieces) ^ Tile::swizzle(row);
            row = row < last ? row : last;
            dma16(from, (uint32_t)row * bytes + piece * 16, to + t * kBytes + (n * kWide + wave) * 1024);
          }
        }
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
          const int i = n * LANES + tid, row = row0 + i / Tile::kPieces;
          in[t][n] = load_piece(base[t] + (int64_t)row * stride[t], i % Tile::kPieces * 8, D,
                                row < rows && (kPieces % LANES == 0 || i < kPieces));
        }
    }
  }
  template <int LATER = 0>
  __device__ __forceinline__ void settle(int stage) {
    if constexpr (WHOLE) {
      wait_loads_outstanding<LATER>();
    } else {
      const int tid = threadIdx.x % LANES;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
          const int i = n * LANES + tid;
          if (kPieces % LANES == 0 || i < kPieces)
            *reinterpret_cast<u32x4_t*>(smem + (2 * stage + t) * kBytes + Tile::place(i / Tile::kPieces, i % Tile::kPieces)) = in[t][n];
        }
    }
  }
  __device__ __forceinline__ void clear_past(int stage, int row0) {
    if constexpr (WHOLE) {
      const int there = rows - row0;
      if (there >= ROWS) return;
      int tid = threadIdx.x % LANES;
      uint32_t zero = 0;
      asm volatile("" : "+v"(tid), "+v"(zero));  // (computed here, in a sequence's last tile: held over the loop it would cost registers)
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int i = n * LANES + tid;  // the piece that this lane's copy brought
        if (i / Tile::kPieces >= there && (kPieces % LANES == 0 || i < kPieces))
          *(lds_u32x4_out_ptr)(uintptr_t)(lds + (2 * stage + 1) * kBytes + i * 16) = u32x4_t{zero, zero, zero, zero};
      }
    }
  }
};
// WHOLE tiles address their rows by 32-bit offsets
constexpr int64_t kMostStride = (int64_t)1 << 24;
inline bool whole_rows(const HeadRows& r) {
  return ((uintptr_t)r.p & 15) == 0 && (r.token | r.head) % 8 == 0 && r.token <= kMostStride;
}

// Operands that a loop keeps have arrived.  The compiler, which does not see the asynchronous copies, would wait for them at their
// first use in the loop, and there for all copies that have just been started, on every round.
template <int N>
__device__ __forceinline__ void arrived(u32x4_t (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// probabilities (registers 8 s .. 8 s + 7 of an accumulator) as an operand
__device__ __forceinline__ u32x4_t acc_operand(const f32x16_t& p, int s) {
  return u32x4_t{pack_bf16x2(p[8 * s], p[8 * s + 1]), pack_bf16x2(p[8 * s + 2], p[8 * s + 3]),
                 pack_bf16x2(p[8 * s + 4], p[8 * s + 5]), pack_bf16x2(p[8 * s + 6], p[8 * s + 7])};
}

// Four elements of a row of D from element d on, of which those from D on are not stored.  Any alignment.
__device__ __forceinline__ void store4(bf16_t* row, int d, int D, uint32_t lo, uint32_t hi) {
  if (d + 4 <= D) {
    *reinterpret_cast<u32x2_any_t*>(row + d) = u32x2_any_t{lo, hi};
  } else {
    if (d < D) row[d] = (bf16_t)lo;
    if (d + 1 < D) row[d + 1] = (bf16_t)(lo >> 16);
    if (d + 2 < D) row[d + 2] = (bf16_t)hi;
  }
}

// A wave's 32 rows of DP elements, between memory and operands.  The operand form: lane l has, of row l % 32, the 16-byte pieces
// 2 m + l / 32.  Loads and stores of just those would move 32 bytes of each of 32 rows; lanes 16 apart exchange pieces, so that an
// instruction moves 64 bytes of each of 16: then v[i] is of row row(i, lane), piece piece(i, lane).  256 images of 12 heads: 90 us, 96
// with pieces of 8 bytes stored from the accumulators; gradients of 64: 83 and 92.  (A second exchange, for whole lines, gave no more.)
template <int DP>
struct WaveRows {
  static constexpr int N = DP / 16;
  static __device__ __forceinline__ int row(int i, int lane) { return 16 * (i & 1) + (lane & 15); }
  static __device__ __forceinline__ int piece(int i, int lane) { return 4 * (i >> 1) + 2 * (lane >> 4 & 1) + (lane >> 5); }
  // From one form to the other.  (Even registers' odd groups of 16 lanes change places with odd registers' even ones.)
  static __device__ __forceinline__ void exchange(u32x4_t (&v)[N]) {
#pragma unroll
    for (int n = 0; n < N; n += 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const auto s = __builtin_amdgcn_permlane16_swap(v[n][e], v[n + 1][e], false, false);
        v[n][e] = s[0];
        v[n + 1][e] = s[1];
      }
  }
  // Of the `rows` rows from `from` on, `stride` elements apart; zeros past them.  In the form of memory.
  static __device__ __forceinline__ void load(u32x4_t (&v)[N], const bf16_t* from, int64_t stride, int rows, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(i, lane);
      v[i] = u32x4_t{0, 0, 0, 0};
      if (r < rows) v[i] = *reinterpret_cast<const u32x4_t*>(from + r * stride + piece(i, lane) * 8);
    }
  }
  // A transposed product (DP / 32 accumulators: a lane's column is a row of the output) times `by`, to the first `rows` rows.
  static __device__ __forceinline__ void store(bf16_t* to, int64_t stride, int rows, const f32x16_t (&acc)[DP / 32], int lane, float by) {
    u32x4_t v[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {  // (the lane has half of each piece, its partner 32 lanes away the other)
      const f32x16_t& x = acc[n / 2];
      const int r = n % 2 * 8;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto s = __builtin_amdgcn_permlane32_swap(pack_bf16x2(x[r + 2 * e] * by, x[r + 2 * e + 1] * by),
                                                        pack_bf16x2(x[r + 4 + 2 * e] * by, x[r + 5 + 2 * e] * by), false, false);
        v[n][e] = s[0];
        v[n][2 + e] = s[1];
      }
    }
    exchange(v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(i, lane);
      if (r < rows) *reinterpret_cast<u32x4_t*>(to + r * stride + piece(i, lane) * 8) = v[i];
    }
  }
};

// One column of a transposed product (DP / 32 accumulators: the elements of one row of the output) to memory, times `by`.
template <int DP>
__device__ __forceinline__ void store_column(bf16_t* row, const f32x16_t (&acc)[DP / 32], int lane, int D, float by) {
  const int h = lane >> 5;
#pragma unroll
  for (int b = 0; b < DP / 32; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d = 32 * b + 8 * q + 4 * h;
      store4(row, d, D, pack_bf16x2(acc[b][4 * q] * by, acc[b][4 * q + 1] * by), pack_bf16x2(acc[b][4 * q + 2] * by, acc[b][4 * q + 3] * by));
    }
}


// Scores of the rows from `limit` on (relative to the lane's first row, 4 (lane / 32)) are not seen.
__device__ __forceinline__ void hide_rows(f32x16_t& s, int limit) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = acc_row(r) < limit ? s[r] : kMinusInf;
}

// Block -> (sequence, key head, head of its group, tile).  Consecutive blocks go to consecutive XCDs, each with an L2 of its
// own.  Where a head has few tiles, XCD x takes all tiles of every eighth key head.  Where it has many, each XCD takes one of
// every eight: of one key head after another, so that at any time an L2 holds the keys of about one head, or, where tiles
// differ in length (`longest_first`: causal), the longest of all heads first, since a kernel ends when its last tile does;
// which of the eight alternates in direction, or the first XCDs would get the longer ones every time.  The last tiles come first
// where `last_first` (under a causal mask the last queries see the most keys, and the first keys the most queries).
constexpr int kManyTiles = 16;
struct TilePlace {
  int seq, kv_head, sub, tile;
};
__device__ __forceinline__ bool tile_place(int sequences, int kv_heads, int group, int n_tiles, bool last_first,
                                           bool longest_first, TilePlace* p) {
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  int unit, t;
  if (n_tiles >= kManyTiles) {
    const int units = sequences * kv_heads, rounds = (n_tiles + 7) / 8;
    int round;
    if (longest_first) {
      round = slot / (units * group);
      unit = slot % (units * group) / group;
    } else {
      unit = slot / (rounds * group);
      round = slot % (rounds * group) / group;
    }
    p->sub = slot % group;
    t = round * 8 + (round % 2 ? 7 - xcd : xcd);
    if (t >= n_tiles) return false;
  } else {
    const int per_unit = n_tiles * group;
    unit = slot / per_unit * 8 + xcd;
    t = slot % per_unit / group;
    p->sub = slot % per_unit % group;
  }
  if (unit >= sequences * kv_heads) return false;
  p->seq = unit / kv_heads;
  p->kv_head = unit % kv_heads;
  p->tile = last_first ? n_tiles - 1 - t : t;
  return true;
}
inline int64_t tile_blocks(int sequences, int kv_heads, int group, int n_tiles) {
  const int64_t units = (int64_t)sequences * kv_heads;
  if (n_tiles >= kManyTiles) return units * ((n_tiles + 7) / 8) * group * 8;
  return (units + 7) / 8 * n_tiles * group * 8;
}

// A launch holds fewer than 2^32 lanes, 2^24 blocks of 256.
constexpr int64_t kMostBlocks = (int64_t)1 << 24;

inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }
constexpr int padded_head(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

// calls f(padded head size, WHOLE) as integral constants; whole: what is loaded by tiles has aligned rows of short strides
template <class F>
void with_head(int D, bool whole, F&& f) {
  auto sized = [&](auto dp) {
    if (whole && D == decltype(dp)::value) f(dp, std::true_type{});
    else f(dp, std::false_type{});
  };
  if (D <= 32) sized(std::integral_constant<int, 32>{});
  else if (D <= 64) sized(std::integral_constant<int, 64>{});
  else sized(std::integral_constant<int, 128>{});
}

#define NM_LDS_ADDRESS(p) ((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)(p))


}  // namespace nm

#endif  // NM_ATTENTION_H
