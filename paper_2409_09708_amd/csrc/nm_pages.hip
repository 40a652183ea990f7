// New keys and values to the pages of their sequences, and tokens read back from there.
//
//   e4m3: per head of a token e = the smallest with max |x| <= 448 2^e, code = x 2^-e to four significant bits (multiples of 2^-9
//   near zero), nearest even;  read back: code 2^e.   bfloat16: as they are.
//
// Bound by memory: a row is read and written once (24 caches in 8 bits read back, 172 MB and 344: 107.8 us, 4.8 TB/s, in bfloat16 140; prompts of 21
// thousand tokens written and read back: 36 + 25, in bfloat16 45 + 31: a token's heads are written one after another, which are rows of as many
// places where pages keep the heads apart, with a byte of its own for each).  Eight elements to a lane, so that accesses in either type run along
// whole rows, and four rows' loads under way (119 us with sixteen elements to a lane and a row at a time).  A block takes the keys or the values
// of a run of tokens; which sequence each belongs to, and which page and slot, its first wave finds for all of them at once.
#include "nm_pages.h"

#include <type_traits>

namespace nm {

namespace {

constexpr int kPageThreads = 256;  // (flat_grid_256)
constexpr int kPageTokens = 64;    // of a block at most

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

// The sequences that packed tokens t0 .. t0 + n - 1 belong to, a token to each lane of a wave: the number of ends at or before it.  Up to 64
// sequences a lane has each one's end, and they are counted without memory; more are halved.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int B, int64_t t0, int n) {
  const int lane = threadIdx.x & 63;
  if (B <= 64) {
    const int64_t end = lane < B ? (int64_t)offsets[lane + 1] : (int64_t)1 << 40;
    int before = 0;
    for (int k = 0; k < n; ++k) {
      const int count = __popcll(__ballot(end <= t0 + k));
      if (lane == k) before = count;
    }
    return before;
  }
  const int64_t t = t0 + lane;
  int from = 0, to = B;
  while (from < to) {
    const int mid = (from + to) / 2;
    if (offsets[mid + 1] <= t) from = mid + 1;
    else to = mid;
  }
  return from;
}

// Where those tokens go, or come from; by a whole wave, a token to each lane.
template <bool WRITE>
__device__ __forceinline__ Place place_of(const PagesArgs& a, int64_t t0, int n) {
  const int64_t t = t0 + (threadIdx.x & 63);
  int b;
  int64_t start, end;
  if (a.offsets != nullptr) {
    b = sequence_of(a.offsets, a.p.B, t0, n);
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
  const int64_t length = a.p.lengths[b];
  // (new tokens are a sequence's last ones)
  const int64_t at = t - start + (WRITE ? length - (end - start) : a.first != nullptr ? (int64_t)a.first[b] : 0);
  if (t < start || at < 0 || at >= length || at >= a.p.width * a.p.page_size) return {-1, 0};
  const int in_table = page_of(a.divide, (int)at);
  const int page = a.p.table[(int64_t)b * a.p.width + in_table];
  return {page >= 0 && page < a.p.pages ? page : WRITE ? -1 : -2, (int)at - in_table * a.p.page_size};
}

// i / d for 0 <= i < 2^21, from 1 / d: the quotient is at least 0.5 / d away from the next integer, the product off by less
__device__ __forceinline__ int page_quotient(int i, float inverse) { return (int)(((float)i + 0.5f) * inverse); }

// The first n of eight elements, of eight codes.  Any alignment.
typedef uint32_t u32x2_byte_t __attribute__((ext_vector_type(2), aligned(1)));
__device__ __forceinline__ void store_elements(bf16_t* to, u32x4_t v, int n) {
  if (n >= 8) {
    *reinterpret_cast<u32x4_any_t*>(to) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) to[e] = (bf16_t)(v[e / 2] >> (16 * (e & 1)));
  }
}
__device__ __forceinline__ void store_codes(uint8_t* to, uint32_t lo, uint32_t hi, int n) {
  if (n >= 8) {
    *reinterpret_cast<u32x2_byte_t*>(to) = u32x2_byte_t{lo, hi};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) to[e] = (uint8_t)((e < 4 ? lo : hi) >> (8 * (e % 4)));
  }
}

// LANES lanes to a row, eight elements each.
constexpr int kPageRows = 4;  // of a lane group, under way at once
template <bool WRITE, bool E4M3, int LANES>
__global__ void __launch_bounds__(kPageThreads) pages_kernel(const PagesArgs a) {
  __shared__ Place places[kPageTokens];
  constexpr int GROUPS = kPageThreads / LANES;
  const int64_t block = flat_lane_256() / kPageThreads, t0 = block / 2 * a.tokens;
  if (t0 >= a.T) return;
  const bool values = block & 1;
  const int n_tokens = (int)(a.T - t0 < a.tokens ? a.T - t0 : a.tokens);
  if (threadIdx.x < 64) {
    static_assert(kPageTokens <= 64, "a lane to each");
    const Place at = place_of<WRITE>(a, t0, n_tokens);
    if (threadIdx.x < n_tokens) places[threadIdx.x] = at;
  }
  __syncthreads();
  const HeadRows& rows = values ? a.V : a.K;
  unsigned char* pages = static_cast<unsigned char*>(values ? a.p.V : a.p.K);
  uint8_t* scales = values ? a.p.V_scales : a.p.K_scales;
  const int d = threadIdx.x % LANES * 8, n = a.p.D - d, units = n_tokens * a.p.H;
  const float by_heads = 1.f / (float)a.p.H;
  for (int i0 = threadIdx.x / LANES; i0 < units; i0 += kPageRows * GROUPS) {
    Place at[kPageRows];
    bf16_t* row[kPageRows];
    int64_t in_page[kPageRows], in_scales[kPageRows];
    u32x4_t in[kPageRows];
    uint32_t exponent[kPageRows];
#pragma unroll
    for (int k = 0; k < kPageRows; ++k) {
      const int i = i0 + k * GROUPS, tok = page_quotient(i, by_heads), head = i - tok * a.p.H;
      at[k] = Place{-1, 0};
      in[k] = u32x4_t{0, 0, 0, 0};
      exponent[k] = 0;
      if (i < units) at[k] = places[tok];
      if (at[k].page == -1) continue;
      row[k] = rows.p + (t0 + tok) * rows.token + head * rows.head + d;
      in_page[k] = at[k].page * a.p.page + at[k].slot * a.p.token + head * a.p.head + d;
      in_scales[k] = at[k].page * a.p.scale_page + at[k].slot * a.p.scale_token + head * a.p.scale_head;
      if constexpr (WRITE) {
        Raw8<false> x;
        x.load(row[k], 0, n);
        in[k] = x.v[0];
      } else if (at[k].page >= 0) {  // (a page that is not there: zeros)
        if constexpr (E4M3) {
          if (n >= 8) {
            const u32x2_byte_t c = *reinterpret_cast<const u32x2_byte_t*>(pages + in_page[k]);
            in[k][0] = c[0];
            in[k][1] = c[1];
          } else {
            in[k] = load_codes(pages + in_page[k], 0, n);
          }
          exponent[k] = scales[in_scales[k]];
        } else {
          Raw8<false> x;
          x.load(reinterpret_cast<const bf16_t*>(pages) + in_page[k], 0, n);
          in[k] = x.v[0];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kPageRows; ++k) {
      if constexpr (WRITE && E4M3) {
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t v = in[k][w], lo = v & 0x7FFFu, hi = v >> 16 & 0x7FFFu;
          top = lo < 0x7F80u && lo > top ? lo : top;
          top = hi < 0x7F80u && hi > top ? hi : top;
        }
#pragma unroll
        for (int m = 1; m < LANES; m <<= 1) {
          const uint32_t other = (uint32_t)__shfl_xor((int)top, m, 64);
          top = other > top ? other : top;
        }
        if (at[k].page == -1) continue;
        const uint32_t e = row_exponent(top);
        const float scale = __uint_as_float(e << 23);
        store_codes(pages + in_page[k], encode2(in[k][0], scale) | encode2(in[k][1], scale) << 16,
                    encode2(in[k][2], scale) | encode2(in[k][3], scale) << 16, n);
        if (d == 0) scales[in_scales[k]] = (uint8_t)e;
      } else {
        if (at[k].page == -1) continue;
        if constexpr (WRITE) store_elements(reinterpret_cast<bf16_t*>(pages) + in_page[k], in[k], n);
        else if constexpr (E4M3) store_elements(row[k], at[k].page >= 0 ? decode8(in[k][0], in[k][1], exponent[k]) : in[k], n);
        else store_elements(row[k], in[k], n);
      }
    }
  }
}

template <bool WRITE>
hipError_t launch_pages(PagesArgs a, hipStream_t s) {
  const int lanes = a.p.D <= 8 ? 1 : a.p.D <= 16 ? 2 : a.p.D <= 32 ? 4 : a.p.D <= 64 ? 8 : 16;
  a.divide = page_divide(a.p.page_size);
  // tokens of a block: kPageRows rows for each of its groups of lanes, twice, and blocks enough for the chip
  const int64_t rows = 2 * kPageRows * kPageThreads / lanes;
  int64_t tokens = (rows + a.p.H - 1) / a.p.H;
  const int64_t spread = (a.T + 1023) / 1024;
  tokens = tokens < spread ? tokens : spread;
  a.tokens = (int)(tokens < kPageTokens ? tokens : kPageTokens);
  const dim3 grid = flat_grid_256((a.T + a.tokens - 1) / a.tokens * 2 * kPageThreads);
  auto go = [&](auto l) {
    constexpr int LANES = decltype(l)::value;
    if (a.p.e4m3) pages_kernel<WRITE, true, LANES><<<grid, kPageThreads, 0, s>>>(a);
    else pages_kernel<WRITE, false, LANES><<<grid, kPageThreads, 0, s>>>(a);
  };
  if (lanes == 1) go(std::integral_constant<int, 1>{});
  else if (lanes == 2) go(std::integral_constant<int, 2>{});
  else if (lanes == 4) go(std::integral_constant<int, 4>{});
  else if (lanes == 8) go(std::integral_constant<int, 8>{});
  else go(std::integral_constant<int, 16>{});
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
