// Softmax attention of new tokens over a cache in pages, one token or a chunk of them per sequence, grouped heads.  Query i of the Lq
// new tokens of a sequence of n tokens stands at p = n - Lq + i and sees the keys
//
//   j <= p  with  j > p - window (where there is one)  or  j < sinks,   whose pages are there;
//   s_j = scale q_i . k_j,  o_i = sum_j exp(s_j - lse_i) v_j,  lse_i = log sum_j exp(s_j);   none: o_i = 0, lse_i = -infinity.
//
// Scores are computed transposed, as nm_attention.h has it; the columns are the (query, head of the group) pairs that share a key head, so
// that all of them share the keys that are read.  The keys that any query of a run can see are numbered without the gap between sinks and
// window ("views"), so tiles hold no keys that nobody sees but at their edges.  What is hidden from all, past the end or on a page that is not
// there has no effect: its value is a zero and its score minus infinity.  (Copies straight to LDS bring such rows all the same, for a page that
// is not there rows of page 0; loads through registers leave them out.)  A lane looks up the page of one row of a tile, two tiles ahead of its
// use, and 8-bit rows become bfloat16 on the way, exactly.
//
// Two kernels.  paged_few_kernel: 16 columns, waves on different keys; all keys of all sequences and heads are one list that is dealt to
// the blocks in equal runs, and what a block leaves of a unit that others share (output, maximum, sum) a second launch joins in order.
// paged_chunk_kernel: 128 columns to a block, 64 keys at a time for its four waves, or for each of two such teams; keys cut where there are
// few blocks.
//
// The first is bound by memory: 24 caches of up to 16384 tokens in 8 bits, 32 heads on 8 of 128, 49.5 us with the join's 5 (3.5 TB/s; caches of one
// length 169 us, 4.8 TB/s): what is left is the latency of a block's first look-ups and of its last unit's end.  The second by the matrix cores and the
// vector work beside them: chunks of 2047 and 1080 tokens on caches of 16384, 16 heads on 4 of 128: 304 us, 900 TFLOP/s (8 bits 368); under windows of
// 1024, five chunks in 8 bits, 36.6 us: ten steps of 2.6 us for each of two teams, and eleven to begin and end (windows of 512 to 2048: 29 to 59 us).
#include "nm_attention.h"
#include "nm_pages.h"

namespace nm {

namespace {

// What a block of the first launch leaves for the second: the unit that begins in it and goes on in the blocks after it.
struct FewShared {
  int parts;  // blocks that share it; 0: there is none
  int q0, columns, tile, kv_head;
  int unused[3];
};
// Where part k of the unit that begins in a block lies: a block has at most two parts of units that others share, one that it goes on with and
// one that it leaves for others.
__device__ __forceinline__ int few_slot(int block, int k) { return 2 * (block + k) + (k == 0 ? 1 : 0); }

struct PagedArgs {
  PagedCall c;
  PageDivide divide;
  int group;         // heads that share a key head
  float scale_log2;  // scale * log2(e)
  int n_tiles;       // column tiles of a sequence, as far as is known
  bool listed;       // chunk: whether blocks count the sequences' tiles
  int cuts;          // few: whether units are dealt to blocks; chunk: pieces of a unit's keys, at most
  int piece;         // chunk: tiles of keys above which a unit is cut
  float* part_o;     // few: [slot][16][DP]; chunk: [query][head][cut][DP]
  float2* part_ml;   // likewise: (maximum of the scaled scores in the exponent's base 2, sum)
  FewShared* shared; // few: [block]
  int lead;          // few: steps that a unit counts for before those of its keys, 0 or 1
  bool whole_o;      // chunk: rows of the output are stored 16 bytes at a time
};

// Sequence b: its first packed query, how many there are, and its tokens (also those behind the table's room: queries stand where their
// tokens do).  Whatever the caller's numbers are, rows stay inside the tensors.
struct PagedSequence {
  int q0, len, n;
};
__device__ __forceinline__ PagedSequence paged_sequence(const PagedCall& c, int b) {
  const int lane = threadIdx.x & 63;
  const int each = (int)(c.Tq / c.p.B);
  int v = lane == 0 ? b * each : (b + 1) * each;
  if (lane == 2) v = c.p.lengths[b];
  else if (lane < 2 && c.offsets_q != nullptr) v = c.offsets_q[b + lane];
  const int n = __builtin_amdgcn_readlane(v, 2);
  int q0 = __builtin_amdgcn_readlane(v, 0), q1 = __builtin_amdgcn_readlane(v, 1);
  q0 = q0 < 0 ? 0 : q0 < c.Tq ? q0 : (int)c.Tq;
  q1 = q1 < q0 ? q0 : q1 < c.Tq ? q1 : (int)c.Tq;
  return {q0, q1 - q0, n < 0 ? 0 : n};
}

// ... of a lane's own sequence
__device__ __forceinline__ PagedSequence lane_sequence(const PagedCall& c, int b) {
  const int each = (int)(c.Tq / c.p.B), Tq = (int)c.Tq;
  int q0 = b * each, q1 = q0 + each;
  if (c.offsets_q != nullptr) {
    q0 = c.offsets_q[b];
    q1 = c.offsets_q[b + 1];
  }
  q0 = q0 < 0 ? 0 : q0 < Tq ? q0 : Tq;
  q1 = q1 < q0 ? q0 : q1 < Tq ? q1 : Tq;
  const int n = c.p.lengths[b];
  return {q0, q1 - q0, n < 0 ? 0 : n};
}

// The keys that queries at positions first .. last may see, as far as the table has room for them (2^30 at most), numbered without the gap:
// view v is key v below `sinks`, else v + gap.
// ALIGN: both parts begin at multiples of it, which adds views that nobody sees.
struct Views {
  int sinks, gap, count;
  int hidden_from, hidden_to;  // keys in between are seen by none of the queries
  __device__ __forceinline__ int key(int v) const { return v < sinks ? v : v + gap; }
};
template <int ALIGN>
__device__ __forceinline__ Views paged_views(const PagedCall& c, int first, int last) {
  const int room = c.p.width * c.p.page_size, end = last < 0 ? 0 : last < room ? last + 1 : room;
  int64_t lo = 0;
  if (c.window > 0) lo = (int64_t)first - c.window + 1;
  const int from = lo > 0 ? (int)(lo < end ? lo : end) : 0, sinks = c.sinks < from ? c.sinks : from;
  const int from_a = from / ALIGN * ALIGN, sinks_a = (sinks + ALIGN - 1) / ALIGN * ALIGN;
  if (from_a <= sinks_a) return {0, 0, end, sinks, from};
  return {sinks_a, from_a - sinks_a, sinks_a + end - from_a, sinks, from};
}

// How a block's tiles come: asynchronous copies straight to LDS (bfloat16 rows of exactly DP elements, 16-byte aligned, in pages that
// hold whole runs of the rows that a wave's copy brings), or through registers, bfloat16 or codes, whole rows or any.
enum { kPagedDirect, kPagedBf16, kPagedCodes, kPagedAnyBf16, kPagedAnyCodes };
constexpr int copy_rows(int DP) { return 512 / DP; }  // that a wave's copy of a kilobyte brings

// A tile of 64 keys and values in LDS, as bfloat16, for a team of four waves.
//   look_up(v0)    starts the look-up of the pages of views v0 .. (every wave for itself)
//   fetch(stage)   starts the loads of the tile looked up last
//   settle(stage)  the rows that this wave brings are in LDS, zeros for those that are not there (of the values, where copies are
//                  direct: scores of such keys have to be hidden anyway); a block's barrier follows
//   seen           the rows of the tile fetched last that are there, a bit each
constexpr int kChunkKeys = 64, kChunkColumns = kWaves * 32;
template <int DP, int HOW>
struct ChunkTile {
  using Tile = RowTile<DP>;
  static constexpr bool CODES = HOW == kPagedCodes || HOW == kPagedAnyCodes, DIRECT = HOW == kPagedDirect;
  static constexpr int kBytes = kChunkKeys * Tile::kRowBytes;
  static constexpr int kPer = CODES ? DP / 16 : DP / 8, kPieces = kChunkKeys * kPer;  // 16-byte pieces as they come
  static constexpr int kLoads = (kPieces + kThreads - 1) / kThreads;
  const int32_t* table;
  Views w;
  const unsigned char* base[2];  // of the key head
  const uint8_t* scales[2];
  unsigned char* smem;           // stages of 2 * kBytes
  uint32_t lds;                  // its address
  int entry, slot;               // lane r: row r of the next tile, its table's entry and the slot in its page (-1: not there)
  bool shown;                    // ... and whether any query sees it
  u32x4_t in[DIRECT ? 1 : 2][DIRECT ? 1 : kLoads];
  uint32_t exponents;            // lane r: those of row r's keys and values
  uint64_t seen;

  __device__ __forceinline__ void begin(const PagedCall& c, int seq, int head, const Views& views) {
    w = views;
    table = c.p.table + (int64_t)seq * c.p.width;
    const int64_t at = (int64_t)head * c.p.head * (CODES ? 1 : 2);
    base[0] = static_cast<const unsigned char*>(c.p.K) + at;
    base[1] = static_cast<const unsigned char*>(c.p.V) + at;
    if constexpr (CODES) {
      scales[0] = c.p.K_scales + head * c.p.scale_head;
      scales[1] = c.p.V_scales + head * c.p.scale_head;
    }
  }
  __device__ __forceinline__ void look_up(const PagedArgs& a, int v0) {
    const int v = v0 + (threadIdx.x & 63), key = w.key(v);
    slot = entry = -1;
    shown = key < w.hidden_from || key >= w.hidden_to;
    if (v < w.count && (DIRECT || shown)) {  // (a copy's rows lie on one page, whose place the first of them gives)
      const int page = page_of(a.divide, key);
      slot = key - page * a.c.p.page_size;
      entry = table[page];
    }
  }
  __device__ __forceinline__ void fetch(const PagedArgs& a, int stage) {
    const PagesCall& p = a.c.p;
    const int tid = threadIdx.x % kThreads, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool there = slot >= 0 && (uint32_t)entry < (uint64_t)p.pages;
    seen = __ballot(there && shown);
    if constexpr (DIRECT) {
      // (rows that are not there: others of the same page, or of the first)
      const int known = there ? entry : -1;
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (uint32_t)stage * 2 * kBytes);
      constexpr int ROWS = copy_rows(DP), PIECES = Tile::kPieces;
      const int row = lane / PIECES;
      const uint32_t from_lane = (uint32_t)row * (uint32_t)p.token * 2 + ((lane % PIECES) ^ Tile::swizzle(wave * ROWS + row)) * 16;
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        if (kPieces % kThreads != 0 && wave * 64 >= kPieces) break;
        const int row0 = (n * kWaves + wave) * ROWS;
        int page = __builtin_amdgcn_readlane(known, row0), in_page = __builtin_amdgcn_readlane(slot, row0);
        if (page < 0) page = in_page = 0;
        const int64_t at = ((int64_t)page * p.page + (int64_t)in_page * p.token) * 2;
#pragma unroll
        for (int t = 0; t < 2; ++t)
          dma16(make_uniform(base[t] + at), from_lane, to + t * kBytes + (n * kWaves + wave) * 1024);
      }
    } else {
      const int64_t at = there ? (int64_t)entry * p.page + (int64_t)slot * p.token : 0;
      const int lo = (int)(uint32_t)at, hi = (int)(at >> 32);
      if constexpr (CODES) {
        exponents = 0;
        if (there) {
          const int64_t s = (int64_t)entry * p.scale_page + (int64_t)slot * p.scale_token;
          exponents = scales[0][s] | (uint32_t)scales[1][s] << 8;
        }
      }
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int i = n * kThreads + tid, piece = i % kPer, row = kPieces % kThreads == 0 ? i / kPer : i / kPer & 63;
        const int64_t from = ((int64_t)__shfl(hi, row, 64) << 32 | (uint32_t)__shfl(lo, row, 64)) * (CODES ? 1 : 2) + piece * 16;
        const bool live = (kPieces % kThreads == 0 || i < kPieces) && (seen >> row & 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          in[t][n] = u32x4_t{0, 0, 0, 0};
          if (!live) continue;
          if constexpr (HOW == kPagedAnyCodes) in[t][n] = load_codes(base[t] + from, 0, p.D - piece * 16);
          else if constexpr (HOW == kPagedAnyBf16) in[t][n] = load_piece(reinterpret_cast<const bf16_t*>(base[t] + from), 0, p.D - piece * 8, true);
          else in[t][n] = *reinterpret_cast<const u32x4_t*>(base[t] + from);
        }
      }
    }
  }
  __device__ __forceinline__ void settle(int stage) {
    if constexpr (DIRECT) {
      wait_loads_outstanding<0>();
      if (seen == ~0ull) return;
      int tid = threadIdx.x % kThreads;
      uint32_t zero = 0;
      asm volatile("" : "+v"(tid), "+v"(zero));  // (computed here, in a few tiles: held over the loop it would cost registers)
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int i = n * kThreads + tid;  // the piece that this lane's copy brought
        if ((kPieces % kThreads == 0 || i < kPieces) && !(seen >> (i / Tile::kPieces) & 1))
          *(lds_u32x4_out_ptr)(uintptr_t)(lds + (2 * stage + 1) * kBytes + i * 16) = u32x4_t{zero, zero, zero, zero};
      }
    } else {
      const int tid = threadIdx.x % kThreads;
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int i = n * kThreads + tid, piece = i % kPer, row = kPieces % kThreads == 0 ? i / kPer : i / kPer & 63;
        const uint32_t e = CODES ? (uint32_t)__shfl((int)exponents, row, 64) : 0;
        if (kPieces % kThreads == 0 || i < kPieces) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            unsigned char* to = smem + (2 * stage + t) * kBytes;
            if constexpr (CODES) {
              u32x4_t v[2];
              decode16(in[t][n], t ? e >> 8 : e & 255, v);
              *reinterpret_cast<u32x4_t*>(to + Tile::place(row, 2 * piece)) = v[0];
              *reinterpret_cast<u32x4_t*>(to + Tile::place(row, 2 * piece + 1)) = v[1];
            } else {
              *reinterpret_cast<u32x4_t*>(to + Tile::place(row, piece)) = in[t][n];
            }
          }
        }
      }
    }
  }
};

// Whether a tile of views v0 .. v0 + ROWS - 1 whose rows are all there is seen whole by queries at positions first .. last.
template <int ROWS>
__device__ __forceinline__ bool seen_whole(const PagedCall& c, const Views& w, int v0, int first, int last) {
  const int from = w.key(v0), to = w.key(v0 + ROWS - 1);
  return to <= first && (c.window <= 0 || from > last - c.window || to < c.sinks);
}

// Which keys the query at position p sees, in two comparisons: key - from < count (unsigned), or key < sinks.
struct Sight {
  int from, count, sinks;
  __device__ __forceinline__ Sight(const PagedCall& c, int p) {
    from = c.window > 0 && p - c.window + 1 > 0 ? p - c.window + 1 : 0;
    count = p + 1 - from > 0 ? p + 1 - from : 0;
    sinks = c.sinks < p + 1 ? c.sinks : p + 1;
  }
  __device__ __forceinline__ bool sees(int key) const { return (uint32_t)(key - from) < (uint32_t)count || key < sinks; }
};

// ------------------------------------------------------------------------------------------------------
// few queries
// ------------------------------------------------------------------------------------------------------
// 16 columns on the 16 x 16 x 32 instruction: lane l has, as an operand, eight elements of row (column) l % 16, and in an accumulator
// rows 4 (l / 16) .. + 3 of column l % 16.  A wave takes 32 keys at a time, each lane the rows l % 16 and l % 16 + 16: it looks up their
// pages, loads 16-byte pieces l / 16, l / 16 + 4, .. of their keys and values, and brings them to bfloat16 with their own powers of two,
// with no exchange between lanes.  Pieces of keys are operands as they are: the elements of a product may come in any order that the
// queries share.  Values go through LDS, to be read transposed.
constexpr int kRun = 32, kStep = kWaves * kRun;  // keys of a wave, of a block, at a time
constexpr int kCols = 16;

__device__ __forceinline__ f32x4_t mma16(u32x4_t a, u32x4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Values in LDS: rows of DP bfloat16, their 16-byte pieces permuted so that 16 rows at one piece (as they are written) and two pieces of
// eight rows (as half a wave reads them) touch every bank once.
template <int DP>
struct ValueRun {
  static constexpr int kRowBytes = DP * 2, kBytes = kRun * kRowBytes;
  static __device__ __forceinline__ int swizzle(int row) {
    return DP == 128 ? ((row & 7) << 1) | (row >> 3 & 1) : DP == 64 ? ((row >> 1 & 3) << 1) | (row >> 3 & 1) : ((row >> 2 & 1) << 1) | (row >> 3 & 1);
  }
  static __device__ __forceinline__ int place(int row, int piece) { return row * kRowBytes + ((piece ^ swizzle(row)) << 4); }
  // columns 16 block .. + 15 as the first operand, rows in the order {0 .. 3, 16 .. 19} + 4 (lane / 16);  at = address + base(lane)
  static __device__ __forceinline__ uint32_t base(int lane) { return place(lane >> 2 & 15, lane >> 1 & 1) + (lane & 1) * 8; }
  static __device__ __forceinline__ u32x4_t columns(uint32_t at, int block) {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    const uint32_t from = at ^ (block << 5);
    const u32x2_t l = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(uintptr_t)from));
    const u32x2_t h = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_ptr)(uintptr_t)(from + 16 * kRowBytes)));
    return u32x4_t{l[0], l[1], h[0], h[1]};
  }
};

// A wave's run of 32 keys and values, from the pages to operands.
template <int DP, bool CODES, bool WHOLE>
struct FewRun {
  // elements of a load, and loads of a lane's row (codes of a row of 32: eight each)
  static constexpr int kWide = CODES && DP >= 64 ? 16 : 8, kLoads = DP / (4 * kWide);
  const int32_t* table;
  Views w;
  const unsigned char* base[2];  // of the key head
  const uint8_t* scales[2];
  int entry[2], slot[2];         // of the next run: the tables' entries and the slots of the lane's two rows (-1: not there)
  u32x4_t in[2][2][kLoads];      // [keys, values][row]
  uint32_t exponents[2];         // keys' and values', of each row
  uint32_t seen;                 // rows of the run loaded last that are there

  __device__ __forceinline__ void begin(const PagedCall& c, int seq, int head, const Views& views) {
    w = views;
    table = c.p.table + (int64_t)seq * c.p.width;
    const int64_t at = (int64_t)head * c.p.head * (CODES ? 1 : 2);
    base[0] = static_cast<const unsigned char*>(c.p.K) + at;
    base[1] = static_cast<const unsigned char*>(c.p.V) + at;
    if constexpr (CODES) {
      scales[0] = c.p.K_scales + head * c.p.scale_head;
      scales[1] = c.p.V_scales + head * c.p.scale_head;
    }
  }
  __device__ __forceinline__ void look_up(const PagedArgs& a, int v0, int lane) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int v = v0 + 16 * r + (lane & 15);
      slot[r] = entry[r] = -1;
      if (v < w.count) {
        const int key = w.key(v), page = page_of(a.divide, key);
        slot[r] = key - page * a.c.p.page_size;
        entry[r] = table[page];
      }
    }
  }
  __device__ __forceinline__ void fetch(const PagedArgs& a, int lane) {
    const PagesCall& p = a.c.p;
    const int group = lane >> 4;
    seen = 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const bool there = slot[r] >= 0 && (uint32_t)entry[r] < (uint64_t)p.pages;
      seen |= ((uint32_t)__ballot(there) & 0xFFFFu) << (16 * r);
      exponents[r] = 0;
#pragma unroll
      for (int n = 0; n < kLoads; ++n) in[0][r][n] = in[1][r][n] = u32x4_t{0, 0, 0, 0};
      if (!there) continue;
      const int64_t at = ((int64_t)entry[r] * p.page + (int64_t)slot[r] * p.token) * (CODES ? 1 : 2);
      if constexpr (CODES) {
        const int64_t s = (int64_t)entry[r] * p.scale_page + (int64_t)slot[r] * p.scale_token;
        exponents[r] = scales[0][s] | (uint32_t)scales[1][s] << 8;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
          const int d = (4 * n + group) * kWide;
          const unsigned char* row = base[t] + at;
          if constexpr (CODES && kWide == 8) {
            typedef uint32_t u32x2_byte_t __attribute__((ext_vector_type(2), aligned(1)));
            if constexpr (WHOLE) {
              const u32x2_byte_t v = *reinterpret_cast<const u32x2_byte_t*>(row + d);
              in[t][r][n][0] = v[0];
              in[t][r][n][1] = v[1];
            } else {
              const int there_d = p.D - d;
              in[t][r][n] = load_codes(row, d, there_d < 8 ? there_d : 8);
            }
          } else if constexpr (CODES) {
            if constexpr (WHOLE) in[t][r][n] = *reinterpret_cast<const u32x4_t*>(row + d);
            else in[t][r][n] = load_codes(row, d, p.D - d);
          } else {
            if constexpr (WHOLE) in[t][r][n] = *reinterpret_cast<const u32x4_t*>(row + 2 * d);
            else in[t][r][n] = load_piece(reinterpret_cast<const bf16_t*>(row), d, p.D, true);
          }
        }
    }
  }
  // Eight elements of the keys (t 0) or values (t 1) of row r; i counts them: element(i, lane) is the first.
  static constexpr int kPieces = DP / 32;
  static __device__ __forceinline__ int element(int i, int lane) {
    return kWide == 16 ? (4 * (i / 2) + (lane >> 4)) * 16 + i % 2 * 8 : (4 * i + (lane >> 4)) * 8;
  }
  __device__ __forceinline__ u32x4_t piece(int t, int r, int i) const {
    if constexpr (!CODES) {
      return in[t][r][i];
    } else {
      const float scale = __uint_as_float((t ? exponents[r] >> 8 : exponents[r] & 255) << 23);
      const u32x4_t& v = in[t][r][kWide == 16 ? i / 2 : i];
      u32x4_t out;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t codes = v[(kWide == 16 ? i % 2 * 2 : 0) + h];
        out[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
        out[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true));
      }
      return out;
    }
  }
};

// A column's running maximum and sum, as softmax_step has them, for 32 scores of four lanes (eight each).
template <int NB>
__device__ __forceinline__ void few_softmax(f32x4_t (&s)[2], float c, float& ref, float& sum, f32x4_t (&acc)[NB]) {
  float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
  for (int r = 1; r < 4; ++r) top = fmaxf(top, fmaxf(s[0][r], s[1][r]));
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64)) * c;
  if (__any(top > ref + kSlack)) {
    const float next = fmaxf(top, ref);
    const float by = ref == kMinusInf ? 0.f : fast_exp2(ref - next);
    ref = next;
    sum *= by;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[b][r] *= by;
  }
  const float base = ref == kMinusInf ? 0.f : ref;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[k][r] = fast_exp2(fmaf(s[k][r], c, -base));
      sum += s[k][r];
    }
}

// The list of all units' steps, key heads outermost, then sequences, then their column tiles; every tile of a sequence has as many steps.
// 64 sequences at a time: a lane has one's queries and tokens, its steps and tiles, and their running sums.
struct Units {
  int b0;             // first sequence of those at hand
  PagedSequence of;
  int steps, tiles;
  int64_t upto;       // steps of all tiles, up to the lane's sequence and with it
};
__device__ __forceinline__ Views few_views(const PagedCall& c, const PagedSequence& of) {
  return paged_views<1>(c, of.n - of.len, of.n - 1);
}
__device__ __forceinline__ void few_units(const PagedArgs& a, int b0, Units* u) {
  const int lane = threadIdx.x & 63, b = b0 + lane;
  u->b0 = b0;
  u->steps = u->tiles = 0;
  if (b < a.c.p.B) {
    u->of = lane_sequence(a.c, b);
    const int steps = (few_views(a.c, u->of).count + kStep - 1) / kStep;
    u->steps = (steps > 0 ? steps : 1) + a.lead;
    u->tiles = (u->of.len * a.group + kCols - 1) / kCols;
  }
  u->upto = (int64_t)u->steps * u->tiles;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int lo = __shfl_up((int)(uint32_t)u->upto, m, 64), hi = __shfl_up((int)(u->upto >> 32), m, 64);
    if (lane >= m) u->upto += (int64_t)hi << 32 | (uint32_t)lo;
  }
}
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
  return (int64_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

// Steps of all sequences, for one key head; `u` is left at the first 64.
__device__ __forceinline__ int64_t few_total(const PagedArgs& a, Units* u) {
  int64_t steps = 0;
  for (int b0 = (a.c.p.B - 1) / 64 * 64; b0 >= 0; b0 -= 64) {
    few_units(a, b0, u);
    steps += lane_value(u->upto, 63);
  }
  return steps;
}

// Where step `at` of a key head's list lies.
struct UnitPlace {
  int seq, tile, step, steps;  // a tile of `steps` steps, `step` of which are before this one
  PagedSequence of;
};
__device__ __forceinline__ UnitPlace few_place(const PagedArgs& a, Units* u, int64_t at) {
  int64_t steps_before = 0;
  for (int b0 = 0;; b0 += 64) {
    if (u->b0 != b0) few_units(a, b0, u);
    const int64_t all = lane_value(u->upto, 63);
    if (at < steps_before + all || b0 + 64 >= a.c.p.B) {
      const uint64_t above = __ballot(steps_before + u->upto > at);
      const int l = above ? __ffsll((unsigned long long)above) - 1 : 0;
      UnitPlace p;
      p.seq = b0 + l;
      p.of = {__builtin_amdgcn_readlane(u->of.q0, l), __builtin_amdgcn_readlane(u->of.len, l), __builtin_amdgcn_readlane(u->of.n, l)};
      p.steps = __builtin_amdgcn_readlane(u->steps, l);
      const int tiles = __builtin_amdgcn_readlane(u->tiles, l);
      const int64_t first = steps_before + lane_value(u->upto, l) - (int64_t)p.steps * tiles;
      p.tile = tiles == 1 ? 0 : (int)((at - first) / p.steps);
      p.step = (int)(at - first - (int64_t)p.tile * p.steps);
      return p;
    }
    steps_before += all;
  }
}
// Steps that a block takes.
__device__ __forceinline__ int64_t few_share(int64_t all, int blocks) {
  const int64_t even = (all + blocks - 1) / blocks;
  return even > 0 ? even : 1;
}

template <int DP, bool CODES, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 2) paged_few_kernel(const PagedArgs a) {
  using Load = FewRun<DP, CODES, WHOLE>;
  using Value = ValueRun<DP>;
  constexpr int NB = DP / 16, STEPS = DP / 32;
  constexpr int JOIN = kCols * (DP + 4) * 4;  // one wave's output, columns padded against bank conflicts
  constexpr int OWN = Value::kBytes > JOIN ? Value::kBytes : JOIN;
  static_assert(OWN % 256 == 0, "operand addresses change bits below 256");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kWaves * OWN];
  __shared__ float2 wave_ml[kWaves][kCols];
  const PagedCall& c = a.c;
  const int D = WHOLE ? DP : c.p.D;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int quarter = lane >> 4, col = lane & 15;
  unsigned char* own = smem + wave * OWN;
  const uint32_t v_at = NM_LDS_ADDRESS(smem) + wave * OWN + Value::base(lane);
  // this block's run of the list of steps -- or, uncut, every (gridDim.x)-th of the units that the grid was made for
  Units units;
  units.b0 = -1;
  int64_t at, end = 0, per_head = 0, share = 0;
  FewShared left = {};
  if (a.cuts) {
    per_head = few_total(a, &units);
    share = few_share(per_head * c.p.H, (int)gridDim.x);
    at = blockIdx.x * share;
    end = at + share < per_head * c.p.H ? at + share : per_head * c.p.H;
  } else {
    at = blockIdx.x;
    end = (int64_t)c.p.B * c.p.H * a.n_tiles;
  }
  while (at < end) {
    int seq, kv_head, tile, step = 0, steps = 0, slot = 0;
    bool alone = true;  // the whole unit is this block's
    PagedSequence of;
    if (a.cuts) {
      kv_head = (int)((uint64_t)at / (uint64_t)per_head);
      const UnitPlace p = few_place(a, &units, at - kv_head * per_head);
      seq = p.seq; tile = p.tile; step = p.step; of = p.of;
      steps = (int)(end - at < p.steps - step ? end - at : p.steps - step);
      alone = steps == p.steps;
      slot = step == 0 ? few_slot(blockIdx.x, 0) : 2 * (int)blockIdx.x;  // (the latter: few_slot of an earlier block)
      if (!alone && step == 0) {
        const int to = (int)((uint64_t)(at + p.steps - 1) / (uint64_t)share);
        left = {to - (int)blockIdx.x + 1, of.q0, of.len * a.group, tile, kv_head, {}};
      }
      at += steps;
    } else {
      seq = (int)(at / (c.p.H * a.n_tiles));
      kv_head = (int)(at / a.n_tiles % c.p.H);
      tile = (int)(at % a.n_tiles);
      at += gridDim.x;
      of = paged_sequence(c, seq);
    }
    const Views views = few_views(c, of);
    const int first_step = step > a.lead ? step - a.lead : 0, end_step = step + steps > a.lead ? step + steps - a.lead : 0;
    const int last_view = a.cuts && end_step * kStep < views.count ? end_step * kStep : views.count;
    Load load;
    load.begin(c, seq, kv_head, views);
    const int columns = of.len * a.group;
    // (a sequence of more queries than the grid was made for has further tiles)
    for (; tile * kCols < columns; tile += a.n_tiles) {
      int v0 = first_step * kStep + wave * kRun;
      load.look_up(a, v0, lane);
      const int n = tile * kCols + col;
      const bool live = n < columns;
      const int qi = n / a.group, head = kv_head * a.group + n % a.group;
      const int first = of.n - of.len, p = first + (live ? qi : 0);  // positions
      const int last_column = tile * kCols + kCols - 1 < columns ? tile * kCols + kCols - 1 : columns - 1;
      const int least_p = first + tile * kCols / a.group, most_p = first + last_column / a.group;
      const bf16_t* q_row = c.Q.p + (int64_t)(of.q0 + qi) * c.Q.token + head * c.Q.head;
      u32x4_t q[STEPS];
#pragma unroll
      for (int i = 0; i < STEPS; ++i) q[i] = load_piece(q_row, Load::element(i, lane), D, live);
      if (v0 < last_view) {
        load.fetch(a, lane);
        load.look_up(a, v0 + kStep, lane);
      }
      f32x4_t acc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      float ref = kMinusInf, sum = 0.f;
      __syncthreads();  // (what the waves joined last has been read)
      for (; v0 < last_view; v0 += kStep) {
        const uint32_t seen = load.seen;
        f32x4_t s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
          for (int r = 0; r < 2; ++r) s[r] = mma16(load.piece(0, r, i), q[i], s[r]);
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int i = 0; i < Load::kPieces; ++i)
            *reinterpret_cast<u32x4_t*>(own + Value::place(16 * r + col, Load::element(i, lane) / 8)) = load.piece(1, r, i);
        if (v0 + kStep < last_view) {
          load.fetch(a, lane);
          load.look_up(a, v0 + 2 * kStep, lane);
        }
        __builtin_amdgcn_wave_barrier();
        if (seen != 0xFFFFFFFFu || !seen_whole<kRun>(c, views, v0, least_p, most_p)) {
          const Sight sight(c, p);
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int row = 16 * k + 4 * quarter + r;
              s[k][r] = sight.sees(views.key(v0 + row)) && (seen >> row & 1) ? s[k][r] : kMinusInf;
            }
        }
        few_softmax(s, a.scale_log2, ref, sum, acc);
        // Probabilities go in as two bfloat16 each, the second what the first leaves: the matrix instructions have time for it here, and the
        // result is as exact as its rounding (200 keys: relative error 0.0016, 0.0025 with one).
        u32x4_t pr, rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lo = s[i / 2][i % 2 * 2], hi = s[i / 2][i % 2 * 2 + 1];
          pr[i] = pack_bf16x2(lo, hi);
          rest[i] = pack_bf16x2(lo - __uint_as_float(pr[i] << 16), hi - __uint_as_float(pr[i] & 0xFFFF0000u));
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const u32x4_t v = Value::columns(v_at, b);
          acc[b] = mma16(v, pr, acc[b]);
          acc[b] = mma16(v, rest, acc[b]);
        }
        __builtin_amdgcn_wave_barrier();
      }
      // join the four waves: each scales its output to the common maximum, then the block adds them in wave order
      sum += __shfl_xor(sum, 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      if (quarter == 0) wave_ml[wave][col] = float2{ref, sum};
      __syncthreads();
      float top = kMinusInf, total = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, wave_ml[w][col].x);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) total += wave_ml[w][col].y * part_weight(wave_ml[w][col].x, top);
      const float by = part_weight(ref, top);
      float* joined = reinterpret_cast<float*>(own);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *reinterpret_cast<float4*>(joined + col * (DP + 4) + 16 * b + 4 * quarter) = float4{acc[b][0] * by, acc[b][1] * by, acc[b][2] * by, acc[b][3] * by};
      __syncthreads();
      // lane -> (column, four elements)
      constexpr int PER_COL = DP / 4;
#pragma unroll
      for (int i = 0; i < (kCols * PER_COL + kThreads - 1) / kThreads; ++i) {
        const int to = i * kThreads + tid, cc = to / PER_COL, d = to % PER_COL * 4;
        const int cn = tile * kCols + cc;
        if (cc >= kCols || cn >= columns || d >= D) continue;
        const float* from = reinterpret_cast<const float*>(smem) + cc * (DP + 4) + d;
        float4 o = *reinterpret_cast<const float4*>(from);
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
          const float4 x = *reinterpret_cast<const float4*>(from + w * (OWN / 4));
          o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
        }
        if (alone) {
          const int64_t tok = of.q0 + cn / a.group;
          const int hd = kv_head * a.group + cn % a.group;
          float t = kMinusInf, l = 0.f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) t = fmaxf(t, wave_ml[w][cc].x);
#pragma unroll
          for (int w = 0; w < kWaves; ++w) l += wave_ml[w][cc].y * part_weight(wave_ml[w][cc].x, t);
          const float inv = l == 0.f ? 0.f : 1.f / l;
          store4(c.O.p + tok * c.O.token + hd * c.O.head, d, D, pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
        } else {
          *reinterpret_cast<float4*>(a.part_o + ((int64_t)slot * kCols + cc) * DP + d) = o;
        }
      }
      if (wave == 0 && quarter == 0 && live) {
        if (!alone) {
          a.part_ml[(int64_t)slot * kCols + col] = float2{top, total};
        } else if (c.lse != nullptr) {
          c.lse[(int64_t)head * c.Tq + of.q0 + qi] = total == 0.f ? kMinusInf : (top + log2f(total)) * kLn2;
        }
      }
      if (a.cuts) break;
    }
  }
  if (a.cuts && tid == 0) a.shared[blockIdx.x] = left;
}

// A column's parts of the unit that began in a block, joined in order by a wave: DP / 4 lanes take four elements each of every
// (256 / DP)-th part, so that several parts' loads are under way.
template <int DP>
__device__ __forceinline__ void join_parts(const PagedArgs& a, int block, int parts, int col, int64_t tok, int head) {
  const PagedCall& c = a.c;
  auto at = [&](int k) { return (int64_t)few_slot(block, k) * kCols + col; };
  constexpr int LANES = DP / 4, GROUPS = 64 / LANES;
  const int lane = threadIdx.x & 63, part = lane / LANES, d = lane % LANES * 4;
  float top = kMinusInf;
  for (int k = lane; k < parts; k += 64) top = fmaxf(top, a.part_ml[at(k)].x);
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
  float total = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int k = part; k < parts; k += GROUPS) {
    const float2 ml = a.part_ml[at(k)];
    const float by = part_weight(ml.x, top);
    total = fmaf(ml.y, by, total);
    const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a.part_o + at(k) * DP + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = d + e < c.p.D ? fmaf(x[e], by, o[e]) : 0.f;
  }
#pragma unroll
  for (int m = LANES; m < 64; m <<= 1) {
    total += __shfl_xor(total, m, 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m, 64);
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  if (part == 0)
    store4(c.O.p + tok * c.O.token + head * c.O.head, d, c.p.D, pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
  if (c.lse != nullptr && lane == 0) c.lse[(int64_t)head * c.Tq + tok] = total == 0.f ? kMinusInf : (top + log2f(total)) * kLn2;
}

// A block to each of the first launch, for the unit that began there; a wave takes a column at a time.
template <int DP>
__global__ void __launch_bounds__(kThreads) paged_few_join_kernel(const PagedArgs a) {
  const FewShared u = a.shared[blockIdx.x];
  if (u.parts <= 0 || u.parts > (int)(gridDim.x - blockIdx.x)) return;
  for (int col = blockIdx.y * kWaves + (threadIdx.x >> 6); col < kCols && u.tile * kCols + col < u.columns; col += gridDim.y * kWaves) {
    const int n = u.tile * kCols + col;
    join_parts<DP>(a, blockIdx.x, u.parts, col, u.q0 + n / a.group, u.kv_head * a.group + n % a.group);
  }
}

// ------------------------------------------------------------------------------------------------------
// chunks of queries
// ------------------------------------------------------------------------------------------------------
// The keys that a tile's columns see, and how many blocks share them.
__device__ __forceinline__ int chunk_position(const PagedSequence& of, int group, int column) {
  const int columns = of.len * group;
  return of.n - of.len + (column < columns ? column : columns - 1) / group;
}
__device__ __forceinline__ Views chunk_views(const PagedArgs& a, const PagedSequence& of, int tile) {
  return paged_views<kChunkKeys>(a.c, chunk_position(of, a.group, tile * kChunkColumns), chunk_position(of, a.group, (tile + 1) * kChunkColumns - 1));
}
__device__ __forceinline__ int chunk_pieces(const PagedArgs& a, int all) {
  const int pieces = (all + a.piece - 1) / a.piece;
  return pieces < 1 ? 1 : pieces < a.cuts ? pieces : a.cuts;
}

// Tile `at` of all sequences' tiles, one sequence after another, a sequence's last tile first, since it sees the most keys.  False: there are
// not so many.  (The last tiles of all sequences first, which left shorter and longer units in turn: the two chunks of 2047 and 1080 tokens 545 us
// for 360.  Every second block went to the same compute units.)
__device__ __forceinline__ bool chunk_place(const PagedArgs& a, int64_t at, int* seq, int* tile, PagedSequence* of) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < a.c.p.B; b0 += 64) {
    PagedSequence its = {0, 0, 0};
    if (b0 + lane < a.c.p.B) its = lane_sequence(a.c, b0 + lane);
    const int tiles = (its.len * a.group + kChunkColumns - 1) / kChunkColumns;
    int upto = tiles;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int before = __shfl_up(upto, m, 64);
      if (lane >= m) upto += before;
    }
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (at < all) {
      const int l = __ffsll((unsigned long long)__ballot(upto > (int)at)) - 1;
      *seq = b0 + l;
      *tile = __builtin_amdgcn_readlane(upto, l) - 1 - (int)at;
      *of = {__builtin_amdgcn_readlane(its.q0, l), __builtin_amdgcn_readlane(its.len, l), __builtin_amdgcn_readlane(its.n, l)};
      return true;
    }
    at -= all;
  }
  return false;
}

constexpr int kNoTiles = 1 << 24;  // more than a sequence has (2^30 columns at most)
// A block has one or two teams of four waves, 32 columns to a wave; two teams have the same columns and take the tiles of keys in turn.
template <int DP, int HOW, int TEAMS>
__global__ void __launch_bounds__(kThreads* TEAMS, 2) paged_chunk_kernel(const PagedArgs a) {
  using Tile = RowTile<DP>;
  using Load = ChunkTile<DP, HOW>;
  constexpr bool WHOLE = HOW <= kPagedCodes;
  constexpr int NB = DP / 32, STEPS = DP / 16;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[TEAMS][2][2 * Load::kBytes];
  const PagedCall& c = a.c;
  const int D = WHOLE ? DP : c.p.D;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x % kThreads >> 6);
  const int team = TEAMS == 1 ? 0 : (int)__builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  // Consecutive blocks go to consecutive XCDs, each with an L2 of its own: key heads change fastest, so that an XCD has few of them.  Where
  // sequences are as long as each other, or too many to count their tiles, the last tiles of all of them come first, then those before them.
  const int64_t items = (int64_t)a.n_tiles * c.p.B * c.p.H * a.cuts;
  for (int64_t item = blockIdx.x; a.listed || item < items; item += gridDim.x) {
    const int kv_head = (int)(item % c.p.H), cut = (int)(item / c.p.H % a.cuts);
    const int64_t at = item / c.p.H / a.cuts;
    int seq, tile;
    PagedSequence of;
    if (a.listed) {
      if (!chunk_place(a, at, &seq, &tile, &of)) return;
    } else {
      seq = (int)(at % c.p.B);
      tile = a.n_tiles - 1 - (int)(at / c.p.B);
      of = paged_sequence(c, seq);
    }
    const int columns = of.len * a.group, first = of.n - of.len;  // (the first query's position)
    // (Without a list, a sequence of more queries than the grid was made for has further tiles, for the blocks of its first ones.  Where each
    // block went through the tiles of all sequences' queries for them, 600 chunks of 64, 8 heads on 2 of 64, caches of 200 took 2470 us for 56.)
    for (const int step = a.listed ? kNoTiles : a.n_tiles; (int64_t)tile * kChunkColumns < columns; tile += step) {
      const int c_wave = tile * kChunkColumns + wave * 32, n = c_wave + (lane & 31);
      const bool live = n < columns;
      const int qi = n / a.group, head = kv_head * a.group + n % a.group, p = first + (live ? qi : 0);
      const int least_p = chunk_position(of, a.group, c_wave), most_p = chunk_position(of, a.group, c_wave + 31);
      const Views views = chunk_views(a, of, tile);
      const int all = (views.count + kChunkKeys - 1) / kChunkKeys, pieces = chunk_pieces(a, all);
      if (cut >= pieces) continue;
      const int from = (int)((int64_t)all * cut / pieces), to = (int)((int64_t)all * (cut + 1) / pieces);
      Load load;
      load.begin(c, seq, kv_head, views);
      load.smem = smem[team][0];
      load.lds = NM_LDS_ADDRESS(smem[team][0]);
      __syncthreads();  // (a block's second tile: what the first one had in LDS is no longer read)
      load.look_up(a, (from + team) * kChunkKeys);
      u32x4_t q[STEPS];
      const bf16_t* q_row = c.Q.p + (int64_t)(of.q0 + qi) * c.Q.token + head * c.Q.head;
#pragma unroll
      for (int st = 0; st < STEPS; ++st) q[st] = load_piece(q_row, 16 * st + 8 * half, D, live);
      if (from + team < to) load.fetch(a, 0);
      load.look_up(a, (from + team + TEAMS) * kChunkKeys);
      if constexpr (Load::DIRECT) arrived(q);
      f32x16_t acc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;
      float ref = kMinusInf, sum = 0.f;
      int stage = 0;
      for (int k0 = from; k0 < to; k0 += TEAMS, stage ^= 1) {
        const int kt = k0 + team, v0 = kt * kChunkKeys;
        if (TEAMS == 1 || kt < to) load.settle(stage);
        const uint64_t seen = load.seen;
        __syncthreads();
        if (kt + TEAMS < to) {
          load.fetch(a, stage ^ 1);
          load.look_up(a, v0 + 2 * TEAMS * kChunkKeys);
        }
        // (a wave whose queries are all before the tile, or past what their window holds of it, has nothing to do)
        const int k_first = views.key(v0), k_last = views.key(v0 + kChunkKeys - 1);
        if ((TEAMS > 1 && kt >= to) || c_wave >= columns || k_first > most_p || (c.window > 0 && k_last <= least_p - c.window && k_first >= c.sinks))
          continue;
        const uint32_t k_tile = load.lds + (uint32_t)stage * 2 * Load::kBytes, v_tile = k_tile + Load::kBytes;
        const uint32_t k_at = k_tile + Tile::row_base(lane), v_at = v_tile + Tile::column_base(lane);
        constexpr int KB = kChunkKeys / 32, NS = KB * STEPS, NV = kChunkKeys / 16 * NB;
        // (products on the same sums wait for each other: the two runs of keys in turn)
        auto keys = [&](int i) { return Tile::rows(k_at, i % KB * 32, i / KB); };
        auto values = [&](int i) { return Tile::columns(v_at, i / NB * 16, i % NB); };
        f32x16_t s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
        u32x4_t f[kAhead];
        read_ahead<NS>(f, keys);
        products<NS>(f, keys, [&](int i, u32x4_t k) { s[i % KB] = mma32(k, q[i / KB], s[i % KB]); });
        read_ahead<NV>(f, values);
        if (seen != ~0ull || !seen_whole<kChunkKeys>(c, views, v0, least_p, most_p)) {
          const Sight sight(c, p);
          int key = k_first + 4 * half;  // (a tile lies on one side of the gap)
          uint64_t there = seen >> (4 * half);
          asm volatile("" : "+v"(key), "+v"(there));  // (or the sums with rows' constants would be held over the loop)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int row = 32 * kb + acc_row(r);
              s[kb][r] = sight.sees(key + row) && (there >> row & 1) ? s[kb][r] : kMinusInf;
            }
        }
        softmax_step(s, a.scale_log2, ref, sum, acc);
        // Probabilities go in as one bfloat16 each, unlike the few queries' above: the matrix instructions have no time to spare here.  (Relative
        // error of the two chunks 0.0023, of which the output's own rounding is 0.0017; with two 0.0017 and 423 us for 327; windows 47 for 41.)
        u32x4_t pr[kChunkKeys / 16];
#pragma unroll
        for (int st = 0; st < kChunkKeys / 16; ++st) pr[st] = acc_operand(s[st / 2], st % 2);
        products<NV>(f, values, [&](int i, u32x4_t v) { acc[i % NB] = mma32(v, pr[i / NB], acc[i % NB]); });
      }
      sum = half_sum(sum);
      if constexpr (TEAMS == 2) {  // the second team's sums to the first, which has the same columns in the same lanes
        static_assert(kWaves * (NB * 16 + 2) * 64 * 4 <= (int)sizeof(smem), "in LDS that tiles have left");
        f32x4_t* box = reinterpret_cast<f32x4_t*>(smem) + wave * NB * 4 * 64 + lane;
        float2* ml = reinterpret_cast<float2*>(reinterpret_cast<f32x4_t*>(smem) + kWaves * NB * 4 * 64) + wave * 64 + lane;
        __syncthreads();
        if (team == 1) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) box[(b * 4 + r) * 64] = f32x4_t{acc[b][4 * r], acc[b][4 * r + 1], acc[b][4 * r + 2], acc[b][4 * r + 3]};
          *ml = float2{ref, sum};
        }
        __syncthreads();
        if (team == 1) continue;
        const float2 other = *ml;
        const float top = fmaxf(ref, other.x), mine = part_weight(ref, top), its = part_weight(other.x, top);
        ref = top;
        sum = sum * mine + other.y * its;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[b][r] = acc[b][r] * mine + box[(b * 4 + r / 4) * 64][r % 4] * its;
      }
      if (pieces > 1) {
        if (live) {
          const int64_t part = ((int64_t)(of.q0 + qi) * c.Hq + head) * a.cuts + cut;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
              *reinterpret_cast<float4*>(a.part_o + part * DP + 32 * b + acc_row(r) + 4 * half) =
                  float4{acc[b][r], acc[b][r + 1], acc[b][r + 2], acc[b][r + 3]};
          if (half == 0) a.part_ml[part] = float2{ref, sum};
        }
        continue;
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      auto o_row = [&](int column) {
        return c.O.p + (int64_t)(of.q0 + column / a.group) * c.O.token + (kv_head * a.group + column % a.group) * c.O.head;
      };
      if (WHOLE && a.whole_o) {
        WaveRows<DP>::store([&](int r) { return o_row(c_wave + r); }, columns - c_wave, acc, lane, inv);
      } else if (live) {
        store_column<DP>(o_row(n), acc, lane, D, inv);
      }
      if (live && c.lse != nullptr && half == 0)
        c.lse[(int64_t)head * c.Tq + of.q0 + qi] = sum == 0.f ? kMinusInf : (ref + log2f(sum)) * kLn2;
    }
  }
}

// The pieces of a column joined in order: DP / 4 lanes to a (query, head), four elements each.
template <int DP>
__global__ void __launch_bounds__(kThreads) paged_chunk_join_kernel(const PagedArgs a) {
  constexpr int LANES = DP / 4, GROUPS = kThreads / LANES;
  const PagedCall& c = a.c;
  const PagedSequence of = paged_sequence(c, (int)blockIdx.y);
  const int d = threadIdx.x % LANES * 4, rows = of.len * c.Hq;
  for (int i = blockIdx.x * GROUPS + threadIdx.x / LANES; i < rows; i += gridDim.x * GROUPS) {
    const int query = i / c.Hq, head = i - query * c.Hq, tile = (query * a.group + head % a.group) / kChunkColumns;
    const int pieces = chunk_pieces(a, (chunk_views(a, of, tile).count + kChunkKeys - 1) / kChunkKeys);
    if (pieces == 1) continue;
    const int64_t tok = of.q0 + query, at = (tok * c.Hq + head) * a.cuts;
    const float2* ml = a.part_ml + at;
    const float* part = a.part_o + at * DP + d;
    float top = kMinusInf, total = 0.f;
    for (int k = 0; k < pieces; ++k) top = fmaxf(top, ml[k].x);
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < pieces; ++k) {
      const float by = part_weight(ml[k].x, top);
      total = fmaf(ml[k].y, by, total);
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(part + (int64_t)k * DP);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(x[e], by, o[e]);
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    if (d < c.p.D)
      store4(c.O.p + tok * c.O.token + head * c.O.head, d, c.p.D, pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    if (c.lse != nullptr && d == 0) c.lse[(int64_t)head * c.Tq + tok] = total == 0.f ? kMinusInf : (top + log2f(total)) * kLn2;
  }
}

// ------------------------------------------------------------------------------------------------------
// How a call is cut
// ------------------------------------------------------------------------------------------------------
// (query, head) pairs of a key head up to which the first kernel serves, of bfloat16 and of codes: it reads keys once per 16 of them, the second
// once per 128 (16 heads on 4 of 128, two caches of 16384, first and second kernel, bfloat16: 16 columns 31.7 and 35.3 us, 32 36.0 and 35.3,
// 48 44.4 and 36.6; codes, which come to LDS through registers in the second: 32 30.3 and 38.5, 64 37.2 and 40.3, 96 50.0 and 41.8;
// 24 ragged caches: bfloat16 32 85 and 99, 64 100 and 102, codes 64 62 and 118).
constexpr int64_t kFewColumns = 32, kFewColumnsCodes = 64;
constexpr int64_t kFewSequences = 512;         // up to which lists are made
constexpr int64_t kFewTiles = 4096;            // column tiles of all sequences, likewise
// Blocks that the list is dealt to: two of each compute unit (24 ragged caches of up to 16384: 55.6 us; 71.4 with 256, 64.2 with 768, which come
// in two rounds).
constexpr int64_t kFewBlocks = 512;
// Most keys of a call whose units are left whole, and for every four units of the call: dealing costs a launch, and each unit that a block goes
// on to a look-up and a join of waves that nothing hides; whole units leave blocks idle (whole and dealt; one sequence, 12 heads of 64, 400 keys:
// 9.4 and 12.4 us, 1000: 14.2 and 10.8; ragged ones, 32 heads on 8 of 128, 8 bits, 192 units up to 500: 12.9 and 14.3, 1000: 20.9 and 14.4;
// 512 units, 1000: 22.9 and 22.1; 800, 1000: 29.6 and 32.3, 2000: 53 and 42; 1600, 2000: 82 and 81, 4000: 143 and 119; 3200, 2000: 142 and
// 172, 4000: 246 and 260).
constexpr int64_t kUncutKeys = 4 * kStep, kUncutKeysOfUnits = 5;
// Steps to each block, if all units were as long as the longest, from which on a unit's begin and end count for a step: a block that goes on to
// another unit takes fewer then, and ends with the others (24 ragged caches of up to 16384: 55.8 and 51.5 us, 64 of 4000 44 and 37, 100 of 2000 51 and 42;
// with two 53, 40 and 42; where blocks have a step or two it costs one: 24 of 1000 15.7 and 16.5).
constexpr int64_t kLeadSteps = 4;
struct PagedPlan {
  bool few, listed;
  int cuts, piece, teams, lead;
  int64_t n_tiles, blocks;
  size_t columns, most_columns;  // of DP sums, in the workspace; of any max_k, window and sinks
};
// Chunks: teams of a block and pieces of the longest unit's keys, by what the call takes if all units are as long; shorter ones get fewer
// of the same size.  A step of 64 keys takes a team 1.9 us alone on its compute unit and 2.2 beside another one, of the same block or not (two
// causal prompts of 8191 and 342: 2.17; chunks of 2047 and 1080 on caches of 16k, one team to most units: 1.92); a block takes three steps
// to begin and end, a block of two teams four, and where blocks are many the last ones end alone.  The pieces' sums are written and read at
// 5 TB/s, and a launch joins them; where that wins less than a tenth, sequences are hardly ever all as long as the longest (the two chunks
// with teams of two and one, two and three pieces: 352, 389 and 393 us; one team 439, 379 and 359).
constexpr int64_t kUnits = 256, kMostCuts = 16;
struct ChunkPlan {
  int teams, cuts;
};
int chunk_most_cuts(int64_t units) {
  const int64_t cuts = 8 * kUnits / units;
  return (int)(cuts < 1 ? 1 : cuts < kMostCuts ? cuts : kMostCuts);
}
ChunkPlan chunk_plan(int64_t units, int64_t key_tiles, int64_t columns, int DP) {
  ChunkPlan best = {1, 1};
  double least = 0;
  for (int teams = 1; teams <= 2; ++teams)
    for (int cuts = 1; cuts <= chunk_most_cuts(units); ++cuts) {
      const double steps = (double)((key_tiles + cuts * teams - 1) / (cuts * teams) + 2 + teams), blocks = (double)units * cuts;
      const double rounds = blocks * teams / (2 * kUnits);
      double us = teams == 1 && blocks <= kUnits ? 1.9 * steps : 2.2 * steps * (rounds <= 1 ? 1 : rounds + 0.3);
      if (cuts > 1) us += 6 + (double)columns * cuts * DP * 8 / 5e6;
      if (cuts > 1) us *= 1.1;
      if ((teams == 1 && cuts == 1) || us < least) {
        best = {teams, cuts};
        least = us;
      }
    }
  return best;
}
// keys that some queries in a row may see
int64_t paged_most_views(int64_t queries, int64_t max_k, int window, int sinks) {
  if (window <= 0) return max_k;
  const int64_t some = (int64_t)window + sinks + queries;
  return some < max_k ? some : max_k;
}
PagedPlan paged_plan(bool codes, int64_t Tq, int B, int Hq, int Hkv, int D, int64_t max_q, int64_t max_k, int window, int sinks) {
  PagedPlan p = {};
  const int64_t group = Hq / Hkv, units = (int64_t)B * Hkv;
  p.few = max_q * group <= (codes ? kFewColumnsCodes : kFewColumns);
  const int64_t per_tile = p.few ? kCols : kChunkColumns;
  p.n_tiles = (max_q * group + per_tile - 1) / per_tile;
  if (p.n_tiles < 1) p.n_tiles = 1;
  if (p.few) {
    const int64_t tiles = B + Tq * group / kCols;  // at most
    p.cuts = B <= kFewSequences && tiles <= kFewTiles;
    p.most_columns = p.cuts ? (size_t)(2 * kFewBlocks * kCols) : 0;  // (few_slot)
    const int64_t views = paged_most_views(max_q, max_k, window, sinks);
    if (views <= kUncutKeys || 4 * views <= kUncutKeysOfUnits * units * p.n_tiles) p.cuts = 0;
    p.lead = p.cuts && (views + kStep - 1) / kStep * units * p.n_tiles >= kLeadSteps * kFewBlocks;
    p.blocks = p.cuts ? kFewBlocks : units * p.n_tiles < kMostBlocks ? units * p.n_tiles : kMostBlocks - 1;
    p.columns = p.cuts ? p.most_columns : 0;
  } else {
    const int64_t tiles = B + Tq * group / kChunkColumns, some = tiles < B * p.n_tiles ? tiles : B * p.n_tiles;  // with queries, at most
    const int64_t views = paged_most_views(max_q < kChunkColumns / group ? max_q : kChunkColumns / group + 1, max_k, window, sinks);
    const int64_t key_tiles = (views + kChunkKeys - 1) / kChunkKeys;
    const ChunkPlan chunk = chunk_plan(some * Hkv, key_tiles, Tq * Hq, padded_head(D));
    p.cuts = chunk.cuts;
    p.teams = chunk.teams;
    p.listed = B <= kFewSequences && Tq != B * max_q;
    p.blocks = (p.listed ? some : B * p.n_tiles) * Hkv * p.cuts;
    if (p.blocks >= kMostBlocks) p.blocks = kMostBlocks - 1;  // (blocks take several then)
    p.piece = (int)((key_tiles + p.cuts - 1) / p.cuts > 0 ? (key_tiles + p.cuts - 1) / p.cuts : 1);
    const int most = chunk_most_cuts(some * Hkv);
    p.columns = p.cuts > 1 ? (size_t)Tq * Hq * p.cuts : 0;
    p.most_columns = most > 1 ? (size_t)Tq * Hq * most : 0;
  }
  return p;
}
size_t paged_bytes(size_t columns, int D) {
  return columns ? round256(columns * padded_head(D) * sizeof(float)) + round256(columns * sizeof(float2)) + kFewBlocks * sizeof(FewShared) : 0;
}

}  // namespace

size_t paged_workspace_bytes(const PagedCall& c) {
  return paged_bytes(paged_plan(c.p.e4m3, c.Tq, c.p.B, c.Hq, c.p.H, c.p.D, c.max_q, c.max_k, c.window, c.sinks).columns, c.p.D);
}
size_t paged_workspace_most(int64_t Tq, int B, int Hq, int Hkv, int D, int64_t max_q) {
  size_t most = 0;
  for (const bool codes : {false, true}) {
    const size_t columns = paged_plan(codes, Tq, B, Hq, Hkv, D, max_q, 0, 0, 0).most_columns;
    most = columns > most ? columns : most;
  }
  return paged_bytes(most, D);
}

hipError_t launch_paged(const PagedCall& c, hipStream_t s) {
  PagedArgs a = {};
  a.c = c;
  a.divide = page_divide(c.p.page_size);
  a.group = c.Hq / c.p.H;
  a.scale_log2 = c.scale * kLog2e;
  const PagedPlan plan = paged_plan(c.p.e4m3, c.Tq, c.p.B, c.Hq, c.p.H, c.p.D, c.max_q, c.max_k, c.window, c.sinks);
  a.n_tiles = (int)plan.n_tiles;
  a.cuts = plan.cuts;
  a.piece = plan.piece;
  a.listed = plan.listed;
  a.lead = plan.lead;
  a.whole_o = whole_rows(c.O);
  if (plan.columns) {
    a.part_o = static_cast<float*>(c.workspace);
    unsigned char* behind = static_cast<unsigned char*>(c.workspace) + round256(plan.columns * padded_head(c.p.D) * sizeof(float));
    a.part_ml = reinterpret_cast<float2*>(behind);
    a.shared = reinterpret_cast<FewShared*>(behind + round256(plan.columns * sizeof(float2)));
  }
  const int64_t unit = c.p.e4m3 ? 16 : 8;  // elements of 16 bytes
  const bool whole = (((uintptr_t)c.p.K | (uintptr_t)c.p.V) & 15) == 0 && (c.p.page | c.p.token | c.p.head) % unit == 0;
  const bool direct = whole && !c.p.e4m3 && c.p.page_size % copy_rows(padded_head(c.p.D)) == 0 && c.p.token <= kMostStride;
  with_head(c.p.D, whole, [&](auto dp, auto is_whole) {
    constexpr int DP = decltype(dp)::value;
    constexpr bool WHOLE = decltype(is_whole)::value;
    auto go = [&](auto codes) {
      constexpr bool CODES = decltype(codes)::value;
      if (plan.few) {
        paged_few_kernel<DP, CODES, WHOLE><<<dim3((unsigned)plan.blocks), kThreads, 0, s>>>(a);
        if (a.cuts) {
          const int64_t columns = c.max_q * a.group < kCols ? c.max_q * a.group : kCols;
          const dim3 join((unsigned)plan.blocks, (unsigned)(columns > kWaves ? (columns + kWaves - 1) / kWaves : 1));
          paged_few_join_kernel<DP><<<join, kThreads, 0, s>>>(a);
        }
      } else {
        const dim3 grid((unsigned)plan.blocks);
        auto launch = [&](auto how) {
          if (plan.teams == 1) paged_chunk_kernel<DP, decltype(how)::value, 1><<<grid, kThreads, 0, s>>>(a);
          else paged_chunk_kernel<DP, decltype(how)::value, 2><<<grid, 2 * kThreads, 0, s>>>(a);
        };
        if constexpr (CODES) launch(std::integral_constant<int, WHOLE ? kPagedCodes : kPagedAnyCodes>{});
        else if (WHOLE && direct) launch(std::integral_constant<int, kPagedDirect>{});
        else launch(std::integral_constant<int, WHOLE ? kPagedBf16 : kPagedAnyBf16>{});
        if (a.cuts > 1) {
          // (two rows to a group of lanes)
          const int64_t blocks = (c.max_q * c.Hq * (DP / 4) + 2 * kThreads - 1) / (2 * kThreads);
          const dim3 join((unsigned)(blocks < 1 ? 1 : blocks < kMostBlocks ? blocks : kMostBlocks - 1), (unsigned)c.p.B);
          paged_chunk_join_kernel<DP><<<join, kThreads, 0, s>>>(a);
        }
      }
    };
    if (c.p.e4m3) go(std::true_type{});
    else go(std::false_type{});
  });
  return hipGetLastError();
}

}  // namespace nm
