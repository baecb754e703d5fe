// sv_chunk_attention: attention of the new tokens of every sequence over the pages of its cache.
//
// For a head of the cache, the rows are the new tokens times the query heads that share it (group G): row rho is token rho / G, head
// h G + rho % G.  Both products run transposed on the matrix cores, so that nothing of a tile is rearranged between lanes:
//   S^T[key][row] = K Q^T      operand A: sixteen keys, a lane holds sixteen bytes of one key's row
//   O^T[col][row] = V^T P^T    operand A: sixteen groups of W columns, a lane holds W columns of eight keys
// The result of the first product has, in lane (g, m), keys 4 g .. 4 g + 3 of row m, which is operand B of the second one if its sum
// over 32 keys takes them in the order (tile, key 4 g + r): the order of a sum is free as long as both operands follow it.
// Likewise the columns of the first product: a lane's sixteen bytes are at 64 s + 16 g of the row, for keys and queries alike.
// So keys and values go from the cache's pages into registers and from there into the matrix cores, without LDS (up to 64 rows).
// The softmax is one pass: a running maximum (in units of log2, raised only when it is exceeded by more than 8: a weight is at most 2^8
// then) and, in every lane, the sum of the weights of its keys.  Scores, weights, sums and outputs are float32; weights are rounded to
// bfloat16 for the second product where the queries are bfloat16 (half a step: at most 2^-8 of a weight).
//
// A workgroup has four wavefronts: one, two or four blocks of rows, and as many interleaved parts of the keys as that leaves, joined in
// LDS at the end.  Where there are few rows, the keys of a row block are divided among up to `splits` workgroups, whose results a second kernel
// joins; each has at least kMinSteps x 32 keys, and about as many as the average of kTargetGroups of them, from the lengths that the device
// knows.
// What bounds it: reading the cache once (64 x 1 over 16384 tokens, 8 heads of 128 bf16 columns: 708 us, 6.1 TB/s); 8-bit keys and values are also
// converted, four instructions to eight columns, and sequences of 2048 to 8192 tokens do not divide evenly (64 x 9: 199 us, 3.5 TB/s).  In one sequence of
// 1500 tokens nothing but a chain of loads is left: 7 us and 5 for the join.
// Rows are laid out over wavefronts, and keys over workgroups, by the largest number of new tokens that a sequence may have: one chunk of 512 tokens and
// 63 single ones of other sequences, all over 8192, take 973 us in one call, and 376 and 150 in two.
#pragma once

#include "paged.hpp"

namespace sv {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = 32;              // keys of a step
constexpr int kMinSteps = 4;           // steps of a workgroup that divides a row block's keys with others, at least
// Workgroups that the keys of a call are divided among: two to a compute unit, which is what the registers hold.  Calls with 512, 1024 and 2048 of
// them, on one card: 64 x 1 over 16384 bf16 714, 722 and 726 us; 64 x 9 over 2048 to 8192 in 8 bits 217, 225 and 230; 2048 over 6144 389, 474 and 504.
constexpr int kTargetGroups = 512;
constexpr int kMaxSplits = 64;
constexpr int kAttnWaves = 4;
constexpr float kFar = 16777216.f;     // 2^24
constexpr long long kMaxRows = 1 << 28;   // B * P * Hq: positions and rows stay within 32 bits

struct AttnArgs {
  const char* q;
  char* out;
  float* lse;                          // [n_rows, Hq], or null
  int64_t q_stride, out_stride;        // bytes from row to row
  Rows rows;
  Pages pages;
  const int32_t* first;                // [B], or null
  int Hq, group, D, window;
  FastDiv by_group;
  float scale2;                        // scale * log2 e
  bool zero;                           // the scale is 0, scale2 1: queries are multiplied by 0 instead, since 0 times the -inf of an unseen key is
                                       // a NaN (not over 8-bit caches, where keys are masked behind the product with the scale)
  const char *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  int tiles, splits, tile_rows;        // row blocks of a head of a sequence; most workgroups to one; rows of one
  int* n_split;                        // [items]            scratch, null without it
  float* part_ml;                      // [items, splits, tile_rows, 2]
  float* part_o;                       // [items, splits, tile_rows, D]
};

// A sequence as all calls see it.
struct Sequence {
  int row0, n, start, first;           // its first row, new tokens, tokens before them, first token that may be seen
  int cap;                             // positions from here on are in no page
};

__device__ __forceinline__ Sequence sequence_of(const AttnArgs& a, int b) {
  Sequence s;
  if (a.rows.offsets) {
    s.row0 = a.rows.offsets[b];
    s.n = min(a.rows.offsets[b + 1] - s.row0, a.rows.P);
    if (s.row0 < 0 || s.row0 > a.rows.n_rows - s.n) s.n = 0;        // (rows outside the tensor are not touched)
  } else {
    s.row0 = b * a.rows.P;
    s.n = a.rows.P;
  }
  s.start = a.rows.start[b];
  s.first = a.first ? max(a.first[b], 0) : 0;
  const int64_t cap = (int64_t)a.pages.max_pages * (int)a.pages.page.d;
  const int most = 0x7fffff00 - a.rows.P;      // (positions of the last new tokens, and of the steps around them, stay within 32 bits)
  s.cap = (int)(cap < most ? cap : most);
  if (s.start < 0 || s.start > s.cap) s.start = s.cap;              // every row is behind the last page
  return s;
}

// Keys [lo, hi) that the rows of tokens i0 .. i1 see between them.
__device__ __forceinline__ void keys_of(const AttnArgs& a, const Sequence& s, int i0, int i1, int* lo, int* hi) {
  *lo = s.first;
  if (a.window > 0) *lo = max(*lo, s.start + i0 - a.window + 1);
  *hi = min(s.start + i1 + 1, s.cap);
}

// Steps of a workgroup that divides keys with others, from the lengths of all sequences (all lanes of the wavefront active).
__device__ __forceinline__ int steps_per_group(const AttnArgs& a) {
  int64_t sum = 0;
  const int lane = threadIdx.x & (kWave - 1);
  for (int k = lane; k < a.rows.B; k += kWave) {
    const Sequence s = sequence_of(a, k);
    if (s.n <= 0) continue;
    int lo, hi;
    keys_of(a, s, 0, s.n - 1, &lo, &hi);
    const int rows = (s.n * a.group + a.tile_rows - 1) / a.tile_rows;
    if (hi > lo) sum += (int64_t)((hi - lo + kStep - 1) / kStep) * rows;
  }
  const double total = wave_sum_f64((double)sum) * a.pages.heads;
  const double steps = total * (1.0 / kTargetGroups);
  return max(kMinSteps, (int)fmin(steps + 1.0, 1e9));
}

template <int ET, int CT, int DPAD>
struct Shape {
  static constexpr bool f8 = CT == SV_F8;
  static constexpr bool f32 = ET == SV_F32;
  static constexpr int cb = f8 ? 1 : (f32 ? 4 : 2);     // bytes of a column in the cache
  static constexpr int eb = f32 ? 4 : 2;
  static constexpr int NK = DPAD * cb / 64;             // sixteen-byte loads of a key
  static constexpr int EK = 16 / cb;                    // columns of one
  static constexpr int W = f32 || DPAD == 64 ? 4 : 8;   // columns of a value that a lane holds in one block
  static constexpr int NB = DPAD / (16 * W);            // blocks of 16 W columns
  static constexpr int WV = (W * cb + 3) / 4;           // words of one
};

template <int N>
struct Words {
  uint32_t w[N];
};

template <int N>
__device__ __forceinline__ void load_words(const char* p, uint32_t (&w)[N]) {
  typedef uint32_t vec __attribute__((ext_vector_type(N == 1 ? 2 : N), aligned(1)));
  if constexpr (N == 1) {
    typedef uint32_t one __attribute__((aligned(1)));
    w[0] = *reinterpret_cast<const one*>(p);
  } else {
    const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = v[i];
  }
}

// From LDS, aligned to its size.
template <int N>
__device__ __forceinline__ void load_lds(const char* p, uint32_t (&w)[N]) {
  typedef uint32_t vec __attribute__((ext_vector_type(N)));
  const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = v[i];
}

__device__ __forceinline__ uint32_t f8_pair_bf16(uint32_t w, bool high) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d});
}

// 0 times the number whose exponent has the bits E: 0, or a NaN (in those bits and the one below) for what is not finite.
template <uint32_t E>
__device__ __forceinline__ uint32_t zero_or_nan(uint32_t w) { return (w & E) == E ? E | (E >> 1) : 0u; }

// max / sum over the four lanes that hold the same row (lanes m, m + 16, m + 32, m + 48)
__device__ __forceinline__ float across_max(float v) {
  Halves h = swap32(__float_as_uint(v), __float_as_uint(v));
  v = fmaxf(__uint_as_float(h.a), __uint_as_float(h.b));
  h = swap16(__float_as_uint(v), __float_as_uint(v));
  return fmaxf(__uint_as_float(h.a), __uint_as_float(h.b));
}
__device__ __forceinline__ float across_sum(float v) {
  Halves h = swap32(__float_as_uint(v), __float_as_uint(v));
  v = __uint_as_float(h.a) + __uint_as_float(h.b);
  h = swap16(__float_as_uint(v), __float_as_uint(v));
  return __uint_as_float(h.a) + __uint_as_float(h.b);
}

// The part of a row block's keys that a wavefront goes through, and its rows.
template <int ET, int CT, int DPAD, int NT, bool WHOLE, bool STAGED = false>
struct Wavefront {
  // STAGED: keys and values come from LDS in the type of the queries, whatever the cache holds
  using Sh = Shape<ET, STAGED ? ET : CT, DPAD>;
  static constexpr bool kScaled = CT == SV_F8;          // rows have scales
  static constexpr int kCacheBytes1 = CT == SV_F8 ? 1 : (CT == SV_F32 ? 4 : 2);
  static constexpr int NO = DPAD / 16;                  // output tiles of a block of sixteen rows

  const AttnArgs& a;
  const int g, m;                                       // lane = 16 g + m
  const int32_t* table;                                 // the sequence's pages
  int64_t head_off;                                     // rows of D from a page's first to this head's first
  int pos[NT], low[NT];                                 // the row's position, and the first key that it sees
  uint32_t qw[NT][Sh::NK * Sh::EK * Sh::eb / 4];        // queries, by the columns of the keys' loads
  f32x4 o[NT][NO];
  float mx[NT], l[NT];
  bool far;                                             // some row's maximum is beyond 2^24 (the same in all lanes; not with kScaled)

  __device__ __forceinline__ Wavefront(const AttnArgs& args) : a(args), g((threadIdx.x & 63) >> 4), m(threadIdx.x & 15) {}

  // Row of the cache, in units of D columns, of a position and this head; -1: in no page.
  __device__ __forceinline__ int64_t page_row(int key) const {
    const int k = divide(key, a.pages.page);
    const int at = k < a.pages.max_pages ? table[k] : -1;
    if (at < 0 || at >= a.pages.n_pages) return -1;
    return (int64_t)at * a.pages.heads * (int)a.pages.page.d + head_off + (key - k * (int)a.pages.page.d);
  }

  __device__ __forceinline__ float scale() const { return fabsf(a.scale2); }
  __device__ __forceinline__ int row_bytes() const { return (WHOLE ? DPAD : a.D) * kCacheBytes1; }

  __device__ __forceinline__ void start(const Sequence& s, int rho0, int h) {
    far = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int rho = rho0 + 16 * n + m, i = divide(rho, a.by_group), hq = h * a.group + rho - i * a.group;
      const bool there = i < s.n;
      // rows that are not there see everything: they never make a step a partial one, and are not written
      pos[n] = there ? s.start + i : 0x7fffffff;
      low[n] = there ? s.first : 0;
      if (there && a.window > 0) low[n] = max(low[n], pos[n] - a.window + 1);
      const char* row = a.q + (int64_t)(s.row0 + (there ? i : 0)) * a.q_stride + (int64_t)hq * a.D * Sh::eb;
#pragma unroll
      for (int k = 0; k < Sh::NK; ++k) {
        constexpr int words = Sh::EK * Sh::eb / 4, per = Sh::eb == 4 ? 4 : 8;    // (columns in whole vectors of `per`)
        const int col = (64 * k + 16 * g) / Sh::cb;
#pragma unroll
        for (int e = 0; e < Sh::EK; e += per) {
          uint32_t w[4] = {};
          if (there && (WHOLE || col + e < a.D)) load_words<4>(row + (int64_t)(col + e) * Sh::eb, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) qw[n][k * words + e * Sh::eb / 4 + j] = w[j];
        }
      }
      if (!kScaled && a.zero) {
#pragma unroll
        for (int j = 0; j < Sh::NK * Sh::EK * Sh::eb / 4; ++j) qw[n][j] = Sh::f32 ? zero_or_nan<0x7f800000u>(qw[n][j])
                                                                                 : zero_or_nan<0x7f800000u>(qw[n][j]) | zero_or_nan<0x00007f80u>(qw[n][j]);
      }
      if (a.scale2 < 0.f) {                              // (the scale is taken positive)
#pragma unroll
        for (int j = 0; j < Sh::NK * Sh::EK * Sh::eb / 4; ++j) qw[n][j] ^= Sh::f32 ? 0x80000000u : 0x80008000u;
      }
      mx[n] = -INFINITY;
      l[n] = 0.f;
#pragma unroll
      for (int t = 0; t < NO; ++t) o[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  struct Keys {
    Words<4> k[2][Sh::NK];
    float scale[2][4];
  };
  struct Values {
    Words<Sh::WV> v[8][Sh::NB];
    float scale[8];
  };
  // Where the keys of a step are.  WHOLE: rows of the first keys of its two tiles, the same in all lanes (a tile lies in one page);
  // otherwise the row of key `lane % 32`, which the lanes that need it take from there.  -1: in no page.
  struct Where {
    int64_t row[WHOLE ? 2 : 1];
  };

  // Keys outside [lo, hi) stand for one inside: they are read, and have no weight.
  __device__ __forceinline__ void find(int key0, int lo, int hi, Where& w) const {
    if constexpr (WHOLE) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int first = min(max(key0 + 16 * t, lo & ~15), (hi - 1) & ~15);
        w.row[t] = page_row(__builtin_amdgcn_readfirstlane(first));
      }
    } else {
      w.row[0] = page_row(min(max(key0 + (int)(threadIdx.x & 31), lo), hi - 1));
    }
  }
  // (after a wait for the table's entries)
  __device__ __forceinline__ void settle(Where& w) const {
    if constexpr (WHOLE) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t r0 = __builtin_amdgcn_readfirstlane((uint32_t)w.row[t]), r1 = __builtin_amdgcn_readfirstlane((uint32_t)(w.row[t] >> 32));
        w.row[t] = (int64_t)(((uint64_t)r1 << 32) | r0);
      }
    }
  }
  __device__ __forceinline__ int64_t found(const Where& w, int t, int k) const {         // (unclamped: -1 where there is none)
    if constexpr (WHOLE) return w.row[t] < 0 ? -1 : w.row[t] + k;
    const int from = 16 * t + k;
    const uint32_t r0 = __shfl((int)(uint32_t)w.row[0], from, kWave), r1 = __shfl((int)(w.row[0] >> 32), from, kWave);
    return (int64_t)(((uint64_t)r1 << 32) | r0);
  }

  __device__ __forceinline__ void load_keys(const Where& w, Keys& kk) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const char* row;
      if constexpr (WHOLE) row = a.k_cache + (w.row[t] < 0 ? 0 : w.row[t]) * row_bytes() + (uint32_t)(m * row_bytes() + 16 * g);
      else row = a.k_cache + max(found(w, t, m), (int64_t)0) * row_bytes() + 16 * g;
#pragma unroll
      for (int k = 0; k < Sh::NK; ++k) {
        const int at = 64 * k + 16 * g, bytes = row_bytes();
        if constexpr (WHOLE) {
          load_words<4>(row + 64 * k, kk.k[t][k].w);
        } else {
          kk.k[t][k] = Words<4>{{0u, 0u, 0u, 0u}};
          if (at + 16 <= bytes) load_words<4>(row + 64 * k, kk.k[t][k].w);
          else if (at + 8 <= bytes) {
            uint32_t w2[2];
            load_words<2>(row + 64 * k, w2);
            kk.k[t][k].w[0] = w2[0];
            kk.k[t][k].w[1] = w2[1];
          }
        }
      }
      if constexpr (Sh::f8) {
        if constexpr (WHOLE) {
          uint32_t x[4];
          load_words<4>(reinterpret_cast<const char*>(a.k_scale + (w.row[t] < 0 ? 0 : w.row[t]) + 4 * g), x);
#pragma unroll
          for (int r = 0; r < 4; ++r) kk.scale[t][r] = __uint_as_float(x[r]);
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) kk.scale[t][r] = a.k_scale[max(found(w, t, 4 * g + r), (int64_t)0)];
        }
      }
    }
  }

  __device__ __forceinline__ void load_values(const Where& w, Values& vv) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = i / 4, r = i % 4;
      const char* row;
      int64_t at = 0;
      if constexpr (WHOLE) {
        row = a.v_cache + (w.row[t] < 0 ? 0 : w.row[t]) * row_bytes() + (uint32_t)(4 * g * row_bytes() + m * Sh::W * Sh::cb) + r * row_bytes();
      } else {
        at = max(found(w, t, 4 * g + r), (int64_t)0);
        row = a.v_cache + at * row_bytes() + m * Sh::W * Sh::cb;
      }
#pragma unroll
      for (int n = 0; n < Sh::NB; ++n) {
        const int col = (16 * n + m) * Sh::W;
        if (WHOLE || col < a.D) load_words<Sh::WV>(row + 16 * n * Sh::W * Sh::cb, vv.v[i][n].w);
        else {
#pragma unroll
          for (int j = 0; j < Sh::WV; ++j) vv.v[i][n].w[j] = 0u;
        }
      }
      if constexpr (Sh::f8 && !WHOLE) vv.scale[i] = a.v_scale[at];
    }
    if constexpr (Sh::f8 && WHOLE) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint32_t x[4];
        load_words<4>(reinterpret_cast<const char*>(a.v_scale + (w.row[t] < 0 ? 0 : w.row[t]) + 4 * g), x);
#pragma unroll
        for (int r = 0; r < 4; ++r) vv.scale[4 * t + r] = __uint_as_float(x[r]);
      }
    }
  }

  __device__ __forceinline__ void scores(const Keys& kk, f32x4 (&s)[NT][2]) const {
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int k = 0; k < Sh::NK; ++k) {
        const uint32_t(&w)[4] = kk.k[t][k].w;
        if constexpr (!Sh::f32 && !Sh::f8) {
          const bf16x8 ka = as_bf16x8(w[0], w[1], w[2], w[3]);
#pragma unroll
          for (int n = 0; n < NT; ++n)
            s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                ka, as_bf16x8(qw[n][4 * k], qw[n][4 * k + 1], qw[n][4 * k + 2], qw[n][4 * k + 3]), s[n][t], 0, 0, 0);
        } else if constexpr (!Sh::f32) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const bf16x8 ka = as_bf16x8(f8_pair_bf16(w[2 * u], false), f8_pair_bf16(w[2 * u], true),
                                        f8_pair_bf16(w[2 * u + 1], false), f8_pair_bf16(w[2 * u + 1], true));
#pragma unroll
            for (int n = 0; n < NT; ++n)
              s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  ka, as_bf16x8(qw[n][8 * k + 4 * u], qw[n][8 * k + 4 * u + 1], qw[n][8 * k + 4 * u + 2], qw[n][8 * k + 4 * u + 3]),
                  s[n][t], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int e = 0; e < Sh::EK; ++e) {
            float ka;
            if constexpr (Sh::f8) {
              const auto p = (e & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8(w[e / 4], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[e / 4], false);
              ka = p[e & 1];
            } else {
              ka = __uint_as_float(w[e]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
              s[n][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka, __uint_as_float(qw[n][Sh::EK * k + e]), s[n][t], 0, 0, 0);
          }
        }
      }
    }
  }

  // Scores to weights, in place (what multiplies the values), with the running maximum and sum, in three parts.  PART: some key of the step is
  // not seen by some row, or in no page.  ks: scales of the keys (8 bits).
  template <bool PART>
  __device__ __forceinline__ void mask(int key0, const float (&ks)[2][4], const Where& w, f32x4 (&s)[NT][2]) const {
    if constexpr (!PART && !kScaled) return;
    bool none[2][4];
    if (PART) {
      asm volatile("");                                  // (a branch)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) none[t][r] = !STAGED && found(w, t, 4 * g + r) < 0;   // (staged keys in no page are NaN)
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = kScaled ? s[n][t][r] * ks[t][r] : s[n][t][r];
          if (PART) {
            const int key = key0 + 16 * t + 4 * g + r;
            x = none[t][r] ? NAN : x;
            x = key >= low[n] && key <= pos[n] ? x : -INFINITY;
          }
          s[n][t][r] = x;
        }
      }
    }
  }

  __device__ __forceinline__ void raise(const f32x4 (&s)[NT][2]) {
    bool any = false;
    float top[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float t8 = fmaxf(s[n][0][0], s[n][0][1]);
      t8 = fmaxf(fmaxf(t8, s[n][0][2]), s[n][0][3]);
      t8 = fmaxf(fmaxf(t8, s[n][1][0]), s[n][1][1]);
      t8 = fmaxf(fmaxf(t8, s[n][1][2]), s[n][1][3]);
      top[n] = across_max(kScaled ? t8 : t8 * scale());
      any |= top[n] > mx[n] + 8.f;
    }
    if (__builtin_expect(__ballot(any) != 0, 0)) {
      asm volatile("");                                  // (a branch: done without one and selected, this is a third of a step's operations)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const bool up = top[n] > mx[n] + 8.f;
        const float f = up ? exp2_fast(mx[n] - top[n]) : 1.f;      // (from -inf: 0)
        mx[n] = up ? top[n] : mx[n];
        l[n] *= f;
#pragma unroll
        for (int t = 0; t < NO; ++t) o[n][t] *= f;
      }
      if constexpr (!kScaled) {
        bool beyond = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) beyond |= fabsf(mx[n]) >= kFar && mx[n] > -INFINITY;
        far = __ballot(beyond) != 0;
      }
    }
  }

  // The maximum is that of rounded products with the scale, and an exponent an exact product less the maximum: at the largest key it is the
  // maximum's rounding, up to half a unit of it.  Below 2^24 that is 1/2 at most; from there on products are rounded first (2^-24 of a score, as
  // a score's own sum is), so that it is 0.
  template <bool PART>
  __device__ __forceinline__ void weigh(int key0, const Values& vv, f32x4 (&s)[NT][2]) {
    float by = scale();
    if constexpr (!kScaled) {
      if (__builtin_expect(far, 0)) {
        asm volatile("");                                  // (a branch)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int t = 0; t < 2; ++t) s[n][t] *= by;
        }
        by = 1.f;
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float base = mx[n] == -INFINITY ? 0.f : mx[n];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p = exp2_fast(kScaled ? s[n][t][r] - base : __builtin_fmaf(s[n][t][r], by, -base));
          l[n] += p;
          if constexpr (kScaled) {
            p *= vv.scale[4 * t + r];
            if (PART) {
              const int key = key0 + 16 * t + 4 * g + r;
              p = key >= low[n] && key <= pos[n] ? p : 0.f;        // (whatever the scale of an unseen key is)
            }
          }
          s[n][t][r] = p;
        }
      }
    }
  }

  // Operand A of output tile (block n, column c of W): the eight keys of a lane.
  __device__ __forceinline__ void value_words(const Values& vv, int nb, uint32_t (&w)[Sh::W][4]) const {
    static_assert(!Sh::f32, "pairs of bfloat16");
    uint32_t x[8][Sh::W / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int j = 0; j < Sh::W / 2; ++j) {
        if constexpr (Sh::f8) x[i][j] = f8_pair_bf16(vv.v[i][nb].w[j / 2], j & 1);
        else x[i][j] = vv.v[i][nb].w[j];
      }
    }
#pragma unroll
    for (int j = 0; j < Sh::W / 2; ++j) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[2 * j][k] = __builtin_amdgcn_perm(x[2 * k + 1][j], x[2 * k][j], 0x05040100u);
        w[2 * j + 1][k] = __builtin_amdgcn_perm(x[2 * k + 1][j], x[2 * k][j], 0x07060302u);
      }
    }
  }
  __device__ __forceinline__ float value_f32(const Values& vv, int i, int nb, int c) const {
    if constexpr (Sh::f8) {
      const auto p = (c & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8(vv.v[i][nb].w[c / 4], true)
                             : __builtin_amdgcn_cvt_pk_f32_fp8(vv.v[i][nb].w[c / 4], false);
      return p[c & 1];
    } else {
      return __uint_as_float(vv.v[i][nb].w[c]);
    }
  }

  __device__ __forceinline__ bf16x8 weights(const f32x4 (&s)[2]) const {
    return as_bf16x8(pack_bf16(s[0][0], s[0][1]), pack_bf16(s[0][2], s[0][3]), pack_bf16(s[1][0], s[1][1]), pack_bf16(s[1][2], s[1][3]));
  }

  __device__ __forceinline__ void add_values(const Values& vv, const f32x4 (&s)[NT][2]) {
    if constexpr (!Sh::f32) {
      bf16x8 p[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) p[n] = weights(s[n]);
#pragma unroll
      for (int nb = 0; nb < Sh::NB; ++nb) {
        uint32_t w[Sh::W][4];
        value_words(vv, nb, w);
#pragma unroll
        for (int c = 0; c < Sh::W; ++c) {
          const bf16x8 va = as_bf16x8(w[c][0], w[c][1], w[c][2], w[c][3]);
#pragma unroll
          for (int n = 0; n < NT; ++n)
            o[n][nb * Sh::W + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, p[n], o[n][nb * Sh::W + c], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int nb = 0; nb < Sh::NB; ++nb) {
#pragma unroll
          for (int c = 0; c < Sh::W; ++c) {
            const float va = value_f32(vv, i, nb, c);
#pragma unroll
            for (int n = 0; n < NT; ++n)
              o[n][nb * Sh::W + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(va, s[n][i / 4][i % 4], o[n][nb * Sh::W + c], 0, 0, 0);
          }
        }
      }
    }
  }

  // Values of a step some of whose keys are not seen by some row: 0 where no row of the block sees the key, and where one is not finite, which
  // the matrix cores would spread to every row (0 times it is NaN); returns whether there is one.
  __device__ __forceinline__ bool clean_values(int key0, int lo, int hi, Values& vv) const {
    auto odd_in = [](uint32_t w) -> uint32_t {             // bits of w that belong to numbers that are not finite
      if constexpr (Sh::f8) {
        // a byte 0x7f or 0xff is a NaN: adding 1 to the seven bits carries into the eighth
        const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
        return (top >> 7) * 0xffu;
      } else if constexpr (Sh::f32) {
        return (w & 0x7f800000u) == 0x7f800000u ? 0xffffffffu : 0u;
      } else {
        return ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u) | ((w & 0x00007f80u) == 0x00007f80u ? 0x0000ffffu : 0u);
      }
    };
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int key = key0 + 16 * (i / 4) + 4 * g + i % 4;
      const bool in = key >= lo && key < hi;
#pragma unroll
      for (int nb = 0; nb < Sh::NB; ++nb) {
#pragma unroll
        for (int j = 0; j < Sh::WV; ++j) {
          uint32_t& w = vv.v[i][nb].w[j];
          w = in ? w : 0u;
          const uint32_t bits = odd_in(w);
          odd |= bits;
          w &= ~bits;
        }
      }
    }
    return __ballot(odd != 0) != 0;
  }

  // What clean_values took out, added to the rows that see it: weights are positive, so a sum with such a term is that of the values
  // themselves.  Read again from the cache, key by key.
  __device__ __forceinline__ void add_odd_values(int key0, int lo, int hi) {
#pragma unroll 1
    for (int key = max(key0, lo); key < min(key0 + kStep, hi); ++key) {
      const int64_t row = page_row(key);
      if (row < 0) continue;
      const char* from = a.v_cache + row * row_bytes();
#pragma unroll
      for (int t = 0; t < NO; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = (16 * (t / Sh::W) + 4 * g + r) * Sh::W + t % Sh::W;
          float v = 0.f;
          if (WHOLE || col < a.D) {
            if constexpr (CT == SV_F8) {
              const uint8_t c = static_cast<uint8_t>(from[col]);
              v = (c & 0x7f) == 0x7f ? NAN : 0.f;
            } else if constexpr (CT == SV_F32) {
              v = reinterpret_cast<const float*>(from)[col];
            } else {
              v = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(from)[col] << 16);
            }
          }
          const bool odd = !(fabsf(v) < INFINITY);
#pragma unroll
          for (int n = 0; n < NT; ++n)
            if (odd && key >= low[n] && key <= pos[n]) o[n][t][r] += v;
        }
      }
    }
  }

  __device__ __forceinline__ void scaled(const Keys& kk, float (&ks)[2][4]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < 4; ++r) ks[t][r] = kScaled ? kk.scale[t][r] * scale() : 0.f;
    }
  }

  // Steps whose keys some row does not see, or are in no page.
  __device__ __forceinline__ void sweep_part(int s0, int s1, int stride, int lo, int hi) {
#pragma unroll 1
    for (int s = s0; s < s1; s += stride) {
      const int key0 = kStep * s;
      Where at;
      find(key0, lo, hi, at);
      settle(at);
      Keys kk;
      Values vv;
      load_keys(at, kk);
      load_values(at, vv);
      f32x4 sc[NT][2];
      scores(kk, sc);
      float ks[2][4];
      scaled(kk, ks);
      mask<true>(key0, ks, at, sc);
      raise(sc);
      weigh<true>(key0, vv, sc);
      const bool odd = clean_values(key0, lo, hi, vv);
      add_values(vv, sc);
      if (odd) add_odd_values(key0, lo, hi);
    }
  }

  // Steps whose keys all rows see.  The keys of the next step are asked for before the weights of this one are formed, its values
  // before the scores are.
  // With more than one block of rows a wavefront's products go before the other wavefronts' exponentials and conversions: 64 x 9 over 8192 in 8
  // bits, all nine there, 323 us without that and 303 with it, 64 x 8 233 and 225; one block only loses by it (64 x 1 over 16384 bf16 713 and 729).
  __device__ __forceinline__ void sweep_all(int s0, int s1, int stride, int lo, int hi) {
    if (s0 >= s1) return;
    Where at;
    Keys kk;
    find(kStep * s0, lo, hi, at);
    settle(at);
    load_keys(at, kk);
#pragma unroll 1
    for (int s = s0; s < s1; s += stride) {
      Where next;
      find(kStep * min(s + stride, s1 - 1), lo, hi, next);
      Values vv;
      load_values(at, vv);
      f32x4 sc[NT][2];
      if constexpr (NT > 1) __builtin_amdgcn_s_setprio(1);
      scores(kk, sc);
      if constexpr (NT > 1) __builtin_amdgcn_s_setprio(0);
      float ks[2][4];
      scaled(kk, ks);
      settle(next);
      if (s + stride < s1) load_keys(next, kk);
      mask<false>(kStep * s, ks, at, sc);
      raise(sc);
      weigh<false>(kStep * s, vv, sc);
      if constexpr (NT > 1) __builtin_amdgcn_s_setprio(1);
      add_values(vv, sc);
      if constexpr (NT > 1) __builtin_amdgcn_s_setprio(0);
      at = next;
    }
  }

  // Keys of [lo, hi) that every row of the wavefront sees: all_lo .. all_hi.
  __device__ __forceinline__ void seen_by_all(int lo, int hi, int* all_lo, int* all_hi) const {
    int l0 = lo, h0 = hi - 1;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      l0 = max(l0, low[n]);
      h0 = min(h0, pos[n]);
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
      l0 = max(l0, __shfl_xor(l0, d, kWave));
      h0 = min(h0, __shfl_xor(h0, d, kWave));
    }
    *all_lo = __builtin_amdgcn_readfirstlane(l0);
    *all_hi = __builtin_amdgcn_readfirstlane(h0);
  }

  // Steps s0, s0 + stride, ... below s1 of the keys [lo, hi); step s begins at key 32 s.
  __device__ __forceinline__ void sweep(int s0, int s1, int stride, int lo, int hi) {
    if (s0 >= s1) return;
    int all_lo, all_hi;
    seen_by_all(lo, hi, &all_lo, &all_hi);
    // whether a page is missing
    bool gone = false;
    const int last = divide(min(kStep * s1, hi) - 1, a.pages.page);
    for (int k = divide(max(kStep * s0, lo), a.pages.page) + (int)(threadIdx.x & (kWave - 1)); k <= last; k += kWave) {
      const int p = table[k];
      gone |= p < 0 || p >= a.pages.n_pages;
    }
    // steps [f0, f1) are seen whole
    int f0 = (all_lo + kStep - 1) / kStep, f1 = (all_hi + 1) / kStep;
    if (__ballot(gone)) f1 = f0;
    f0 = min(max(f0, s0), s1);
    f0 = s0 + (f0 - s0 + stride - 1) / stride * stride;
    f1 = min(max(f1, f0), s1);
    sweep_part(s0, min(f0, s1), stride, lo, hi);
    sweep_all(f0, f1, stride, lo, hi);
    const int from = f1 > f0 ? f0 + (f1 - f0 + stride - 1) / stride * stride : f0;
    sweep_part(from, s1, stride, lo, hi);
  }
};

// What a workgroup works on: rows rho0 .. of head h of sequence b, steps [mine0, mine1) of the keys [lo, hi) from step step_lo on.
struct Work {
  Sequence s;
  int b, h, item, split, parts, rho0, lo, hi, step0, step1;
};

// The wavefront's rows, from row rho on: outputs, or its part of them.
template <class Wf, class Sh, int NT, bool WHOLE>
__device__ __forceinline__ void write_out(const AttnArgs& a, const Work& k, const Wf& w, const float (&l)[NT], int rho_first) {
  const Sequence& s = k.s;
  const int h = k.h, rho0 = k.rho0, parts = k.parts, item = k.item, split = k.split;
  // lane (g, m): row m of the block, columns ((16 nb) + 4 g + r) W + c of output tile nb W + c
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int rho = rho_first + 16 * n + w.m, i = divide(rho, a.by_group), hq = h * a.group + rho - i * a.group;
    if (i >= s.n) continue;
    const bool out_of_pages = w.pos[n] >= s.cap;
    const bool any = w.mx[n] != -INFINITY || !(l[n] == 0.f);
    if (parts == 1) {
      const float inv = out_of_pages ? NAN : (any ? 1.f / l[n] : 0.f);
      if (a.lse && w.g == 0)
        a.lse[(int64_t)(s.row0 + i) * a.Hq + hq] = out_of_pages ? NAN : (any ? (float)((w.mx[n] + log2((double)l[n])) * kLn2) : -INFINITY);
      char* to = a.out + (int64_t)(s.row0 + i) * a.out_stride + (int64_t)hq * a.D * Sh::eb;
#pragma unroll
      for (int nb = 0; nb < Sh::NB; ++nb) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = (16 * nb + 4 * w.g + r) * Sh::W;
          if (!WHOLE && col >= a.D) continue;
          if constexpr (Sh::f32) {
            typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
            *reinterpret_cast<vec*>(to + col * 4) = vec{w.o[n][nb * 4][r] * inv, w.o[n][nb * 4 + 1][r] * inv,
                                                        w.o[n][nb * 4 + 2][r] * inv, w.o[n][nb * 4 + 3][r] * inv};
          } else {
            typedef uint32_t vec __attribute__((ext_vector_type(Sh::W / 2), aligned(2)));
            vec v;
#pragma unroll
            for (int c = 0; c < Sh::W / 2; ++c)
              v[c] = pack_bf16(w.o[n][nb * Sh::W + 2 * c][r] * inv, w.o[n][nb * Sh::W + 2 * c + 1][r] * inv);
            *reinterpret_cast<vec*>(to + col * 2) = v;
          }
        }
      }
    } else {
      const int64_t at = ((int64_t)item * a.splits + split) * a.tile_rows + (rho - rho0);
      if (w.g == 0) {
        a.part_ml[2 * at] = w.mx[n];
        a.part_ml[2 * at + 1] = l[n];
      }
#pragma unroll
      for (int nb = 0; nb < Sh::NB; ++nb) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = (16 * nb + 4 * w.g + r) * Sh::W;
          if (!WHOLE && col >= a.D) continue;
#pragma unroll
          for (int c = 0; c < Sh::W; c += 4) {
            typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
            *reinterpret_cast<vec*>(a.part_o + at * a.D + col + c) =
                vec{w.o[n][nb * Sh::W + c][r], w.o[n][nb * Sh::W + c + 1][r], w.o[n][nb * Sh::W + c + 2][r], w.o[n][nb * Sh::W + c + 3][r]};
          }
        }
      }
    }
  }
}

// The rows of a workgroup with N blocks of sixteen to a wavefront: as many wavefronts share the keys among them as the rows leave.
template <int ET, int CT, int DPAD, int N, bool WHOLE>
__device__ __forceinline__ void attend(const AttnArgs& a, const Work& k, float* shared) {
  using Wf = Wavefront<ET, CT, DPAD, N, WHOLE>;
  using Sh = Shape<ET, CT, DPAD>;
  constexpr int kRows = 16 * N, NT = N;
  const Sequence& s = k.s;
  const int rows = min(s.n * a.group - k.rho0, a.tile_rows), blocks = (rows + kRows - 1) / kRows;
  const int wr_all = blocks <= 1 ? 1 : (blocks <= 2 ? 2 : 4), wk_all = kAttnWaves / wr_all;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wr = wave & (wr_all - 1), wk = wave / wr_all;
  const int h = k.h, rho0 = k.rho0;
  Wf w(a);
  w.table = a.pages.table + (int64_t)k.b * a.pages.max_pages;
  w.head_off = (int64_t)h * (int)a.pages.page.d;
  w.start(s, rho0 + wr * kRows, h);
  w.sweep(k.step0 + wk, k.step1, wk_all, k.lo, k.hi);
  float l[N];
#pragma unroll
  for (int n = 0; n < N; ++n) l[n] = across_sum(w.l[n]);
  const int lane = threadIdx.x & (kWave - 1);
  if (wk_all > 1) {
    // joined in LDS, by halves: the upper wavefronts hand over, the lower ones add.  Two slots of [2 + 4 NO][N][64].
    constexpr int kSlot = (2 + 4 * Wf::NO) * N * kWave;
#pragma unroll 1
    for (int half = wk_all / 2; half >= 1; half /= 2) {
      if (wk >= half && wk < 2 * half) {
        float* to = shared + ((wk - half) * wr_all + wr) * kSlot + lane;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          to[(2 * n) * kWave] = w.mx[n];
          to[(2 * n + 1) * kWave] = l[n];
#pragma unroll
          for (int t = 0; t < Wf::NO; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) to[(2 * N + (n * Wf::NO + t) * 4 + r) * kWave] = w.o[n][t][r];
          }
        }
      }
      __syncthreads();
      if (wk < half) {
        const float* from = shared + (wk * wr_all + wr) * kSlot + lane;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const float m2 = from[(2 * n) * kWave], top = fmaxf(w.mx[n], m2);
          const float f1 = w.mx[n] == top ? 1.f : exp2_fast(w.mx[n] - top), f2 = m2 == top ? 1.f : exp2_fast(m2 - top);
          w.mx[n] = top;
          l[n] = l[n] * f1 + from[(2 * n + 1) * kWave] * f2;
#pragma unroll
          for (int t = 0; t < Wf::NO; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) w.o[n][t][r] = w.o[n][t][r] * f1 + from[(2 * N + (n * Wf::NO + t) * 4 + r) * kWave] * f2;
          }
        }
      }
      __syncthreads();
    }
    if (wk > 0) return;
  }
  write_out<Wf, Sh, N, WHOLE>(a, k, w, l, rho0 + wr * kRows);
}

// The part of the call that falls to this workgroup; the number of its rows, 0: nothing.
__device__ __forceinline__ int work_of(const AttnArgs& a, Work& k) {
  // workgroups go round the eight XCDs by their number: the row blocks of one head land on one (its keys and values are in that cache), and
  // so do not the parts of a row block, most of which need not exist
  const int heads = a.rows.B * a.pages.heads, bh = blockIdx.x % heads, rest = blockIdx.x / heads, tile = rest % a.tiles;
  k.split = rest / a.tiles;
  k.item = bh * a.tiles + tile;
  k.h = bh % a.pages.heads;
  k.b = bh / a.pages.heads;
  k.s = sequence_of(a, k.b);
  k.rho0 = tile * a.tile_rows;
  const int rows = min(k.s.n * a.group - k.rho0, a.tile_rows);
  if (rows <= 0) return 0;
  const int i0 = divide(k.rho0, a.by_group), i1 = divide(k.rho0 + rows - 1, a.by_group);
  keys_of(a, k.s, i0, i1, &k.lo, &k.hi);
  const int step_lo = k.lo / kStep, steps = k.hi > k.lo ? (k.hi + kStep - 1) / kStep - step_lo : 0;
  k.parts = 1;
  k.step0 = step_lo;
  k.step1 = step_lo + steps;
  if (a.splits > 1) {
    // (up to a quarter more than the average stays whole, where a part is long: 64 x 1 over 2048 to 8192 tokens 280 us so 267, in 8 bits 181
    // and 165.  Parts of a few steps do not: 5 x 7 float32 rows over 900 tokens 17.4 us, so 20.5)
    const int unit = steps_per_group(a), more = unit >= 16 ? unit / 4 : 0;
    k.parts = max(1, min((steps - more + unit - 1) / unit, a.splits));
    if (k.split >= k.parts) return 0;
    const int each = (steps + k.parts - 1) / k.parts;
    k.step0 = step_lo + min(k.split * each, steps);
    k.step1 = min(k.step0 + each, step_lo + steps);
    if (k.split == 0 && threadIdx.x == 0) a.n_split[k.item] = k.parts;
  }
  return rows;
}

// One workgroup: a row block of a head of a sequence, a part of its keys.
template <int ET, int CT, int DPAD, int NT, bool WHOLE>
__global__ void __launch_bounds__(kAttnWaves* kWave, (DPAD == 256 || (ET == SV_F32 && DPAD == 128) ? 1 : 2)) attention_kernel(AttnArgs a) {
  __shared__ float shared[2 * (2 + DPAD / 4) * NT * kWave];
  Work k;
  const int rows = work_of(a, k);
  if (rows <= 0) return;
  if (NT > 1 && rows <= 16) attend<ET, CT, DPAD, 1, WHOLE>(a, k, shared);
  else if (NT > 2 && rows <= 32) attend<ET, CT, DPAD, 2, WHOLE>(a, k, shared);
  else attend<ET, CT, DPAD, NT, WHOLE>(a, k, shared);
}

// Many rows: 128 to a workgroup, 32 to a wavefront, which all need the same keys and values.  A step of them at a time is staged in LDS as bfloat16
// (8-bit ones are converted once, not by every wavefront), the next step under way in registers meanwhile.  The sixteen-byte chunks of a row are
// permuted by its number, so that the sixteen rows of a key operand lie in different banks.  Of a wavefront's step 32 cycles of bank conflicts are
// counted, as many as its eight value reads have passes of sixteen lanes, whose groups read four rows, each permuted its own way.
// What bounds it is the vector ALU beside the matrix cores: per 32 keys and 32 rows, 32 matrix instructions of 16 cycles and about 206 of the vector
// ALU, some 900 cycles: exponentials (16, four slots each), maxima, sums, conversions, and 32 permutations that transpose the values.  A wavefront at its
// products goes before the one that shares its SIMD and is at its exponentials: 2048 over 6144 with 32 heads on 8, 450 us without that and 418
// with it, on one card, the median of the first twelve launches (of a hundred it is 375 us, of their first twelve 421).  (The scores of the next step
// formed beside the weights of this one, in one wavefront: 485 and not 418.)
constexpr int kTileKeys = kStep;

template <int CT, int DPAD, bool WHOLE>
__global__ void __launch_bounds__(kAttnWaves* kWave, 2) attention_tile_kernel(AttnArgs a) {
  constexpr int NT = 2, kChunks = DPAD / 8, kRowsAtOnce = kAttnWaves * kWave / kChunks, kLoads = kTileKeys / kRowsAtOnce;
  constexpr bool kF8 = CT == SV_F8;
  using Wf = Wavefront<SV_BF16, CT, DPAD, NT, WHOLE, true>;
  using Sh = typename Wf::Sh;
  __shared__ u32x4 tile[2][2][kTileKeys][kChunks];       // buffer, keys / values
  __shared__ float scales[kF8 ? 2 : 1][2][kTileKeys];
  auto place = [](int key, int chunk) { return chunk ^ (kChunks >= 16 ? key & 15 : (key >> 1) & (kChunks - 1)); };
  Work k;
  if (work_of(a, k) <= 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Wf w(a);
  w.table = a.pages.table + (int64_t)k.b * a.pages.max_pages;
  w.head_off = (int64_t)k.h * (int)a.pages.page.d;
  const int rho = k.rho0 + wave * 16 * NT;
  w.start(k.s, rho, k.h);
  int all_lo, all_hi;
  w.seen_by_all(k.lo, k.hi, &all_lo, &all_hi);
  // keys that some row of the wavefront sees
  const int i0 = divide(rho, a.by_group), i1 = divide(rho + 16 * NT - 1, a.by_group);
  int any_lo = k.hi, any_hi = k.hi;
  if (i0 < k.s.n) keys_of(a, k.s, i0, min(i1, k.s.n - 1), &any_lo, &any_hi);

  // a thread's chunk of rows row0, row0 + kRowsAtOnce, ... of a step.  Its rows of the cache; WHOLE: that of the first of the sixteen keys that
  // its wavefront's rows belong to, the same in all lanes.
  const int chunk = threadIdx.x % kChunks, row0 = threadIdx.x / kChunks;
  const bool there = WHOLE || 8 * chunk < a.D;
  int64_t rows[kLoads];
  Words<kF8 ? 2 : 4> kw[kLoads], vw[kLoads];
  float sc[2];
  auto find = [&](int key0) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = row0 + j * kRowsAtOnce;
      if constexpr (WHOLE) rows[j] = w.page_row(__builtin_amdgcn_readfirstlane(min(max(key0 + (r & ~15), k.lo & ~15), (k.hi - 1) & ~15)));
      else rows[j] = w.page_row(min(max(key0 + r, k.lo), k.hi - 1));
    }
  };
  const uint32_t within = (WHOLE ? (uint32_t)((row0 & 15) * w.row_bytes()) : 0u) + (uint32_t)(chunk * 8 * Wf::kCacheBytes1);
  auto load = [&]() {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      int64_t row = rows[j];
      if constexpr (WHOLE) {
        const uint32_t r0 = __builtin_amdgcn_readfirstlane((uint32_t)row), r1 = __builtin_amdgcn_readfirstlane((uint32_t)(row >> 32));
        row = (int64_t)(((uint64_t)r1 << 32) | r0);
      }
      const int64_t at = (row < 0 ? 0 : row) * w.row_bytes();
      constexpr int n = kF8 ? 2 : 4;
      if (there) {
        load_words<n>(a.k_cache + at + within, kw[j].w);
        load_words<n>(a.v_cache + at + within, vw[j].w);
      } else {
#pragma unroll
        for (int e = 0; e < n; ++e) kw[j].w[e] = vw[j].w[e] = 0u;
      }
      if (row < 0) {                                     // in no page: scores are NaN
#pragma unroll
        for (int e = 0; e < n; ++e) { kw[j].w[e] = kF8 ? 0x7f7f7f7fu : 0x7fff7fffu; vw[j].w[e] = 0u; }
      }
      // (a thread of a row for the scales of each of its rows)
      if (kF8 && chunk == j) {
        const int64_t in = row < 0 ? 0 : row + (WHOLE ? row0 & 15 : 0);
        sc[0] = row < 0 ? 1.f : a.k_scale[in];
        sc[1] = row < 0 ? 1.f : a.v_scale[in];
      }
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = row0 + j * kRowsAtOnce, at = place(r, chunk);
      if constexpr (kF8) {
        tile[buf][0][r][at] = u32x4{f8_pair_bf16(kw[j].w[0], false), f8_pair_bf16(kw[j].w[0], true), f8_pair_bf16(kw[j].w[1], false),
                                    f8_pair_bf16(kw[j].w[1], true)};
        tile[buf][1][r][at] = u32x4{f8_pair_bf16(vw[j].w[0], false), f8_pair_bf16(vw[j].w[0], true), f8_pair_bf16(vw[j].w[1], false),
                                    f8_pair_bf16(vw[j].w[1], true)};
        if (chunk == j) { scales[buf][0][r] = sc[0]; scales[buf][1][r] = sc[1]; }
      } else {
        tile[buf][0][r][at] = u32x4{kw[j].w[0], kw[j].w[1], kw[j].w[2], kw[j].w[3]};
        tile[buf][1][r][at] = u32x4{vw[j].w[0], vw[j].w[1], vw[j].w[2], vw[j].w[3]};
      }
    }
  };
  static_assert(kLoads <= kChunks, "a thread of a row for each of its scales");
  static_assert(kWave / kChunks <= 16, "the rows of a wavefront belong to sixteen keys that begin at a multiple of 16");

  typename Wf::Where nowhere;
  if (k.step0 < k.step1) {
    find(kStep * k.step0);
    load();
    store(0);
    find(kStep * (k.step0 + 1));
  }
  int buf = 0;
#pragma unroll 1
  for (int s = k.step0; s < k.step1; ++s, buf ^= 1) {
    __syncthreads();                                     // this step is written, and the one before it is done with
    const bool more = s + 1 < k.step1;
    if (more) {
      load();
      find(kStep * (s + 2));
    }
    const int key0 = kStep * s;
    if (key0 < any_hi && key0 + kStep > any_lo) {
      f32x4 sc2[NT][2];
      typename Wf::Values vv;
      float ks[2][4];
      {
        typename Wf::Keys kk;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int n = 0; n < Sh::NK; ++n) {
            const int r = 16 * t + w.m;
            const u32x4 x = tile[buf][0][r][place(r, 4 * n + w.g)];
#pragma unroll
            for (int e = 0; e < 4; ++e) kk.k[t][n].w[e] = x[e];
          }
        }
        __builtin_amdgcn_s_setprio(1);
        w.scores(kk, sc2);
        __builtin_amdgcn_s_setprio(0);
        if constexpr (kF8) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 16 * (i / 4) + 4 * w.g + i % 4;
            kk.scale[i / 4][i % 4] = scales[buf][0][r];
            vv.scale[i] = scales[buf][1][r];
          }
        }
        w.scaled(kk, ks);
      }
      __builtin_amdgcn_sched_barrier(0);                 // (values read ahead of the weights would take registers that are not there)
      const bool part = key0 < all_lo || key0 + kStep - 1 > all_hi;
      if (part) w.template mask<true>(key0, ks, nowhere, sc2);
      else w.template mask<false>(key0, ks, nowhere, sc2);
      w.raise(sc2);
      if (kF8 && part) w.template weigh<true>(key0, vv, sc2);
      else w.template weigh<false>(key0, vv, sc2);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 16 * (i / 4) + 4 * w.g + i % 4;
#pragma unroll
        for (int n = 0; n < Sh::NB; ++n) {
          const int byte = (16 * n + w.m) * Sh::W * 2;
          const char* from = reinterpret_cast<const char*>(&tile[buf][1][r][place(r, byte / 16)]) + byte % 16;
          load_lds<Sh::WV>(from, vv.v[i][n].w);
        }
      }
      bool odd = false;
      if (part) odd = w.clean_values(key0, k.lo, k.hi, vv);
      __builtin_amdgcn_s_setprio(1);
      w.add_values(vv, sc2);
      __builtin_amdgcn_s_setprio(0);
      if (odd) w.add_odd_values(key0, k.lo, k.hi);
    }
    if (more) store(buf ^ 1);
  }
  float l[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) l[n] = across_sum(w.l[n]);
  write_out<Wf, Sh, NT, WHOLE>(a, k, w, l, rho);
}

// Launches the kernel of a shape; what the rows decide is chosen in sv_chunk_attention.
struct AttnLaunch {
  int nt;              // row blocks of a wavefront, at most
  bool tile;           // more than 64 rows to a head and sequence
  bool whole;          // D is 64, 128 or 256 and no page ends inside a tile of sixteen keys
  unsigned grid;
  hipStream_t stream;
};
void launch_attention_f32(const AttnArgs&, const AttnLaunch&);
void launch_attention_f32_f8(const AttnArgs&, const AttnLaunch&);
void launch_attention_bf16(const AttnArgs&, const AttnLaunch&);
void launch_attention_bf16_f8(const AttnArgs&, const AttnLaunch&);

template <int ET, int CT, int DPAD>
void launch_attention_of(const AttnArgs& a, const AttnLaunch& t) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(t.grid), dim3(kAttnWaves * kWave), 0, t.stream, a); };
  constexpr int NT = ET == SV_F32 || DPAD == 256 ? 1 : 2;
  if constexpr (NT == 2) {
    if (t.tile) {
      if (t.whole) go(attention_tile_kernel<CT, DPAD, true>); else go(attention_tile_kernel<CT, DPAD, false>);
      return;
    }
  }
  if constexpr (NT == 2 && CT == SV_F8) {
    if (t.nt == 3) {
      if (t.whole) go(attention_kernel<ET, CT, DPAD, 3, true>); else go(attention_kernel<ET, CT, DPAD, 3, false>);
      return;
    }
  }
  if (t.nt == 1 || NT == 1) {
    if (t.whole) go(attention_kernel<ET, CT, DPAD, 1, true>); else go(attention_kernel<ET, CT, DPAD, 1, false>);
  } else {
    if (t.whole) go(attention_kernel<ET, CT, DPAD, NT, true>); else go(attention_kernel<ET, CT, DPAD, NT, false>);
  }
}
template <int ET, int CT>
void launch_attention(const AttnArgs& a, const AttnLaunch& t) {
  if (a.D <= 64) launch_attention_of<ET, CT, 64>(a, t);
  else if (a.D <= 128) launch_attention_of<ET, CT, 128>(a, t);
  else launch_attention_of<ET, CT, 256>(a, t);
}

}  // namespace sv
