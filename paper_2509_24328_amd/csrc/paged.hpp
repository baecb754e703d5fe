// New tokens of the sequences of a batch and the pages that hold them: what the calls on a cache share.
// Sequence b has new tokens i = 0 .. n_b - 1 at positions start[b] + i; position p lies in physical page
// pages[b, p / page], place p % page.
#pragma once

#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

// n / d of 0 <= n < 2^31 by one multiplication: with l = ceil(log2 d) and m = floor(2^(31 + l) / d) + 1 <= 2^32 - 1 (d >= 2; m d lies
// in (2^(31 + l), 2^(31 + l) + 2^l]), n m / 2^(31 + l) exceeds n / d by less than 1 / d.  d = 1: m = 2^31 + 1.
struct FastDiv {
  uint32_t d, m;
  int shift;
};
inline FastDiv fast_div(int d) {
  int l = 0;
  while ((1ll << l) < d) ++l;
  return FastDiv{(uint32_t)d, (uint32_t)((1ull << (31 + l)) / (uint64_t)d + 1), 31 + l};
}
__device__ __forceinline__ int divide(int n, const FastDiv& f) { return (int)(((uint64_t)(uint32_t)n * f.m) >> f.shift); }

// The packed or dense rows of a batch's new tokens.
struct Rows {
  const int32_t* offsets;    // [B + 1], or null: sequence b has the rows b P .. b P + P - 1
  const int32_t* start;      // [B]
  int n_rows, B, P;
};

struct Place {
  int b, position;           // b < 0: the row belongs to no sequence
};

// The sequence and position of row r (the same in all lanes of the wavefront, all of them active): the sequences that end at or before
// r are counted, a lane for each, and its beginning and start come from the lane that holds them: one load's time, not a chain of
// them.
__device__ __forceinline__ Place place_of_row(const Rows& rows, int r) {
  int b, i, s;
  if (rows.offsets) {
    const int lane = threadIdx.x & (kWave - 1);
    int k0 = 0, begin = 0, start = 0, n = 0;
    for (; k0 < rows.B; k0 += kWave) {
      const int k = k0 + lane;
      const bool in = k < rows.B;
      begin = in ? rows.offsets[k] : 0;
      start = in ? rows.start[k] : 0;
      n = __popcll(__ballot(in && rows.offsets[k + 1] <= r));
      if (n < kWave) break;
    }
    b = k0 + n;
    if (b >= rows.B) return {-1, 0};
    i = r - __builtin_amdgcn_readlane(begin, n);
    s = __builtin_amdgcn_readlane(start, n);
  } else {
    b = r / rows.P;
    i = r - b * rows.P;
    s = rows.start[b];
  }
  if (i < 0 || i >= rows.P) return {-1, 0};
  // (a start below 0, or one so large that the position leaves 32 bits, is in no page)
  return {b, s < 0 || s > 0x7fffffff - i ? -1 : s + i};
}

struct Pages {
  const int32_t* table;      // [B, max_pages]
  int max_pages, n_pages, heads;
  FastDiv page;
};

// Row of the cache, in units of D elements, of position p of sequence b and head 0; -1: in no page.  Heads lie page.d rows apart.
__device__ __forceinline__ int64_t cache_row(const Pages& pg, int b, int position) {
  if (position < 0) return -1;
  const int k = divide(position, pg.page);
  if (k >= pg.max_pages) return -1;
  const int at = pg.table[(int64_t)b * pg.max_pages + k];
  if (at < 0 || at >= pg.n_pages) return -1;
  return (int64_t)at * pg.heads * (int)pg.page.d + (position - k * (int)pg.page.d);
}

inline int check_rows(const int32_t* t_offsets, int n_rows, int B, int P, int max_pages, int n_pages, int heads, int page, int D) {
  SV_REQUIRE(B >= 0 && P >= 1 && n_rows >= 0 && max_pages >= 1 && n_pages >= 0 && heads >= 1 && page >= 1 && D >= 1,
             SV_ERR_INVALID_ARG);
  SV_REQUIRE((t_offsets ? (long long)n_rows : (long long)B * P) <= SV_TOKENS_MAX, SV_ERR_TOO_LARGE);   // (64 threads to a row, 2^32 to a launch)
  SV_REQUIRE(D <= SV_HEAD_MAX && heads <= SV_HEADS_MAX && page <= SV_PAGE_MAX, SV_ERR_TOO_LARGE);
  return SV_OK;
}

}  // namespace sv
