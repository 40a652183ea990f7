// New keys and values to the pages of their sequences, and tokens read back from there.
//
//   e4m3: per head of a token e = the smallest with max |x| <= 448 2^e, code = x 2^-e to four significant bits (multiples of 2^-9
//   near zero), nearest even;  read back: code 2^e.   bfloat16: as they are.
//
// Bound by memory: a row is read and written once.  Sixteen elements to a lane, so that a row in 8 bits is one 16-byte access a lane,
// and its maximum a few exchanges.  A block takes a run of tokens; which sequence each belongs to, and which page and slot, a wave finds
// for one token at a time: 64 sequences' ends are compared at once.
#include "nm_pages.h"

#include <type_traits>

namespace nm {

namespace {

constexpr int kPageThreads = 256;  // (flat_grid_256)
constexpr int kPageTokens = 32;    // of a block

struct PagesArgs {
  PagesCall p;
  HeadRows K, V;
  const int32_t* offsets;
  const int32_t* first;
  int64_t T;
  int tokens;       // per block
  PageDivide divide;
};

// Where a token's rows lie: its page's number and the slot, -1 where there is none.
struct Place {
  int page, slot;
};

// The sequence that packed token t belongs to: the number of ends at or before it.  By a whole wave.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int B, int64_t t) {
  const int lane = threadIdx.x & 63;
  int from = 0, count = B;  // ends from .. from + count - 1 are in question
  while (count > 0) {
    const int step = (count + 63) / 64, at = from + (lane + 1) * step - 1;  // each lane looks at the last end of its share
    const bool before = (lane + 1) * step <= count && offsets[at + 1] <= t;
    const int full = __popcll(__ballot(before)) * step;
    from += full;
    count -= full;
    if (step == 1) break;
    count = count < step ? count : step;
  }
  return from;
}

// Position of packed token t in its sequence, by a whole wave; -1: no sequence holds it.
template <bool WRITE>
__device__ __forceinline__ Place place_of(const PagesArgs& a, int64_t t) {
  int b;
  int64_t start, end;
  if (a.offsets != nullptr) {
    b = sequence_of(a.offsets, a.p.B, t);
    if (b >= a.p.B) return {-1, 0};
    start = a.offsets[b];
    end = a.offsets[b + 1];
  } else {
    const int64_t each = a.T / a.p.B;
    b = (int)(t / each);
    if (b >= a.p.B) return {-1, 0};
    start = b * each;
    end = start + each;
  }
  if (t < start) return {-1, 0};
  const int64_t length = a.p.lengths[b];
  // (new tokens are a sequence's last ones)
  const int64_t at = t - start + (WRITE ? length - (end - start) : a.first != nullptr ? (int64_t)a.first[b] : 0);
  if (at < 0 || at >= length || at >= a.p.width * a.p.page_size) return {-1, 0};
  const int in_table = page_of(a.divide, (int)at);
  const int page = a.p.table[(int64_t)b * a.p.width + in_table];
  return {page >= 0 && page < a.p.pages ? page : WRITE ? -1 : -2, (int)at - in_table * a.p.page_size};
}

// The first n of sixteen elements.  Any alignment.
__device__ __forceinline__ void store16(bf16_t* to, const u32x4_t (&v)[2], int n) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (n >= 8 * h + 8) {
      *reinterpret_cast<u32x4_any_t*>(to + 8 * h) = v[h];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * h + e < n) to[8 * h + e] = (bf16_t)(v[h][e / 2] >> (16 * (e & 1)));
    }
}

// LANES lanes to a row, sixteen elements each.
template <bool WRITE, bool E4M3, int LANES>
__global__ void __launch_bounds__(kPageThreads) pages_kernel(const PagesArgs a) {
  __shared__ Place places[kPageTokens];
  constexpr int ROWS = kPageThreads / LANES;
  const int64_t t0 = flat_lane_256() / kPageThreads * a.tokens;
  if (t0 >= a.T) return;
  const int n_tokens = (int)(a.T - t0 < a.tokens ? a.T - t0 : a.tokens);
  for (int i = threadIdx.x >> 6; i < n_tokens; i += kPageThreads / 64) {
    const Place at = place_of<WRITE>(a, t0 + i);
    if ((threadIdx.x & 63) == 0) places[i] = at;
  }
  __syncthreads();
  const int d = threadIdx.x % LANES * 16, n = a.p.D - d, per_token = 2 * a.p.H;
  for (int i = threadIdx.x / LANES; i < n_tokens * per_token; i += ROWS) {
    const int tok = i / per_token, which = i % per_token / a.p.H, head = i % per_token % a.p.H;
    const Place at = places[tok];
    if (at.page == -1) continue;
    const HeadRows& out = which ? a.V : a.K;
    bf16_t* row = out.p + (t0 + tok) * out.token + head * out.head + d;
    const int64_t in_page = at.page * a.p.page + at.slot * a.p.token + head * a.p.head + d;
    const int64_t in_scales = at.page * a.p.scale_page + at.slot * a.p.scale_token + head * a.p.scale_head;
    void* pages = which ? a.p.V : a.p.K;
    uint8_t* scales = which ? a.p.V_scales : a.p.K_scales;
    if constexpr (WRITE) {
      Raw8<false> x[2];
      x[0].load(row, 0, n);
      x[1].load(row, 8, n - 8);
      if constexpr (E4M3) {
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          const uint32_t v = x[w / 4].v[0][w % 4], lo = v & 0x7FFFu, hi = v >> 16 & 0x7FFFu;
          top = lo < 0x7F80u && lo > top ? lo : top;
          top = hi < 0x7F80u && hi > top ? hi : top;
        }
#pragma unroll
        for (int m = 1; m < LANES; m <<= 1) {
          const uint32_t other = (uint32_t)__shfl_xor((int)top, m, 64);
          top = other > top ? other : top;
        }
        const uint32_t exponent = row_exponent(top);
        const float scale = __uint_as_float(exponent << 23);
        u32x4_t codes;
#pragma unroll
        for (int w = 0; w < 4; ++w)
          codes[w] = encode2(x[w / 2].v[0][w % 2 * 2], scale) | encode2(x[w / 2].v[0][w % 2 * 2 + 1], scale) << 16;
        uint8_t* to = static_cast<uint8_t*>(pages) + in_page;
        if (n >= 16) {
          *reinterpret_cast<u32x4_byte_t*>(to) = codes;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (e < n) to[e] = (uint8_t)(codes[e / 4] >> (8 * (e % 4)));
        }
        if (d == 0) scales[in_scales] = (uint8_t)exponent;
      } else {
        const u32x4_t v[2] = {x[0].v[0], x[1].v[0]};
        store16(static_cast<bf16_t*>(pages) + in_page, v, n);
      }
    } else {
      u32x4_t v[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      if (at.page >= 0) {  // (a page that is not there: zeros)
        if constexpr (E4M3) {
          decode16(load_codes(static_cast<const uint8_t*>(pages) + in_page, 0, n), scales[in_scales], v);
        } else {
          Raw8<false> x[2];
          x[0].load(static_cast<const bf16_t*>(pages) + in_page, 0, n);
          x[1].load(static_cast<const bf16_t*>(pages) + in_page, 8, n - 8);
          v[0] = x[0].v[0];
          v[1] = x[1].v[0];
        }
      }
      store16(row, v, n);
    }
  }
}

template <bool WRITE>
hipError_t launch_pages(PagesArgs a, hipStream_t s) {
  const int lanes = a.p.D <= 16 ? 1 : a.p.D <= 32 ? 2 : a.p.D <= 64 ? 4 : 8;
  a.divide = page_divide(a.p.page_size);
  // tokens of a block: four rows for each of its groups of lanes, and blocks enough for the chip
  const int64_t rows = 4 * kPageThreads / lanes, per_token = 2 * a.p.H;
  int64_t tokens = (rows + per_token - 1) / per_token;
  const int64_t spread = (a.T + 1023) / 1024;
  tokens = tokens < spread ? tokens : spread;
  a.tokens = (int)(tokens < kPageTokens ? tokens : kPageTokens);
  const dim3 grid = flat_grid_256((a.T + a.tokens - 1) / a.tokens * kPageThreads);
  auto go = [&](auto l) {
    constexpr int LANES = decltype(l)::value;
    if (a.p.e4m3) pages_kernel<WRITE, true, LANES><<<grid, kPageThreads, 0, s>>>(a);
    else pages_kernel<WRITE, false, LANES><<<grid, kPageThreads, 0, s>>>(a);
  };
  if (lanes == 1) go(std::integral_constant<int, 1>{});
  else if (lanes == 2) go(std::integral_constant<int, 2>{});
  else if (lanes == 4) go(std::integral_constant<int, 4>{});
  else go(std::integral_constant<int, 8>{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheWriteCall& c, hipStream_t s) {
  PagesArgs a = {};
  a.p = c.p; a.K = c.K; a.V = c.V; a.offsets = c.offsets; a.T = c.T;
  return launch_pages<true>(a, s);
}

hipError_t launch_cache_read(const CacheReadCall& c, hipStream_t s) {
  PagesArgs a = {};
  a.p = c.p; a.K = c.K; a.V = c.V; a.offsets = c.offsets; a.first = c.first; a.T = c.T;
  return launch_pages<false>(a, s);
}

}  // namespace nm
