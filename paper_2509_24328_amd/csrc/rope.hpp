// Rotary positions: pairs (a, b) of a head's leading `rot` columns turn by the angle  position * freq[pair],
//   a' = amplitude (a cos - b sin),   b' = amplitude (b cos + a sin),
// column j with column j + rot / 2 (halves) or column 2 j with column 2 j + 1 (pairs); the other columns stay.
// Angles, their sines and the products are float64: at position 131072 a float32 angle is off by 4e-3, and a
// turned key that is rounded to 8 bits falls on the same code whoever computed it.  Per column this is six fp64 operations
// against two to four bytes in and out: 16384 tokens x 32 heads of 128 columns keep the memory as busy without them.
#pragma once

#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kRopeLanes = 8;        // lanes that share a head
constexpr int kRopeThreads = 256;
constexpr int kRopeGroups = kRopeThreads / kRopeLanes;

// What of a head is turned, by vectors of EPV elements: `turns` chunks of EPV pairs, `copies` chunks of EPV columns.
struct RopeShape {
  int D, half, turns, copies;
  int pitch;                         // angles of a token in LDS, with a gap after every vector's: lanes read vectors' angles side by side,
};                                   // and without gaps all from the same banks (64 x 9 tokens of 48 heads into 8 bits 9.5 us and 8.1; 16384 x 32 60 and 58)
template <int EPV>
__device__ __forceinline__ int angle_at(int j) { return j + j / EPV; }
inline RopeShape rope_shape(int D, int rot, int dtype) {
  const int epv = 16 / elem_bytes(dtype), half = rot / 2;
  return RopeShape{D, half, (half + epv - 1) / epv, (D - rot + epv - 1) / epv, half + (half - 1) / epv};
}

struct CosSin {
  double c, s;
};

// cos and sin of an angle, times the amplitude: n quarters of a turn and a rest within an eighth of one, formed with the product's own
// rounding added back; the series of sine and cosine up to x^15 / 15! and x^16 / 16! (0.786^17 / 17! = 5e-17).  Good to 1e-15 and
// the angle's own rounding, in 30 operations: the library's sincos, made for any angle, takes several hundred.
__device__ __forceinline__ CosSin cos_sin(double angle, double amplitude) {
  constexpr double kTurns = 0.15915494309189533576888376337251, kTurnsLo = -9.8393383375591e-18;   // 1 / (2 pi), and what that leaves
  const double t = angle * kTurns, lo = __builtin_fma(angle, kTurns, -t) + angle * kTurnsLo;
  const double n = __builtin_rint(4.0 * t);
  const double x = (__builtin_fma(-0.25, n, t) + lo) * 6.283185307179586476925286766559, x2 = x * x;
  double s = -1.0 / 1307674368000.0;
  s = __builtin_fma(s, x2, 1.0 / 6227020800.0);
  s = __builtin_fma(s, x2, -1.0 / 39916800.0);
  s = __builtin_fma(s, x2, 1.0 / 362880.0);
  s = __builtin_fma(s, x2, -1.0 / 5040.0);
  s = __builtin_fma(s, x2, 1.0 / 120.0);
  s = __builtin_fma(s, x2, -1.0 / 6.0);
  s = __builtin_fma(s * x2, x, x);
  double c = 1.0 / 20922789888000.0;
  c = __builtin_fma(c, x2, -1.0 / 87178291200.0);
  c = __builtin_fma(c, x2, 1.0 / 479001600.0);
  c = __builtin_fma(c, x2, -1.0 / 3628800.0);
  c = __builtin_fma(c, x2, 1.0 / 40320.0);
  c = __builtin_fma(c, x2, -1.0 / 720.0);
  c = __builtin_fma(c, x2, 1.0 / 24.0);
  c = __builtin_fma(c, x2, -0.5);
  c = __builtin_fma(c, x2, 1.0);
  const int q = (int)((long long)n & 3);
  const double a = q & 1 ? s : c, b = q & 1 ? c : s;     // magnitudes of cos and sin in the quarter
  CosSin r;
  r.c = (q == 1 || q == 2 ? -a : a) * amplitude;
  r.s = (q >= 2 ? -b : b) * amplitude;
  return r;
}

typedef u32x4 u32x4_any __attribute__((aligned(1)));

// Elements [at, at + n) of a row, 0 < n <= EPV, as floats (the others 0); whole vectors by one load.
template <int DT>
__device__ __forceinline__ void load_some(const void* row, int at, int n, float (&f)[Elem<DT>::per_vec]) {
  constexpr int EPV = Elem<DT>::per_vec;
  if (n >= EPV) {
    const char* p = static_cast<const char*>(row) + (int64_t)at * Elem<DT>::bytes;
    unpack<DT>(*reinterpret_cast<const u32x4_any*>(p), f);
    return;
  }
#pragma unroll
  for (int e = 0; e < EPV; ++e) f[e] = e < n ? load_elem<DT>(row, at + e) : 0.f;
}

template <int DT>
__device__ __forceinline__ void store_some(void* row, int at, int n, const float (&f)[Elem<DT>::per_vec]) {
  constexpr int EPV = Elem<DT>::per_vec;
  if constexpr (DT == DT_F32) {
    float* p = static_cast<float*>(row) + at;
    if (n >= EPV) {
      *reinterpret_cast<u32x4_any*>(p) = u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                                               __float_as_uint(f[3])};
      return;
    }
#pragma unroll
    for (int e = 0; e < EPV; ++e)
      if (e < n) p[e] = f[e];
  } else {
    uint16_t* p = static_cast<uint16_t*>(row) + at;
    if (n >= EPV) {
      *reinterpret_cast<u32x4_any*>(p) = u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]),
                                               pack_bf16(f[6], f[7])};
      return;
    }
#pragma unroll
    for (int e = 0; e < EPV; ++e)
      if (e < n) p[e] = (uint16_t)pack_bf16(f[e], 0.f);
  }
}

// One head, by the lanes of a group (lane: 0 .. kRopeLanes - 1).  cs: the token's angles, at angle_at.  put(column, count, values)
// is called for every chunk, with float32 values; columns that stay are passed on unchanged, unless skip_copies.
template <int DT, bool PAIRS, class Put>
__device__ __forceinline__ void turn_head(const void* row, const RopeShape& sh, const CosSin* cs, int lane, bool skip_copies,
                                          Put&& put) {
  constexpr int EPV = Elem<DT>::per_vec;
  for (int c = lane; c < sh.turns; c += kRopeLanes) {
    const int j = c * EPV, n = min(EPV, sh.half - j);          // pairs j .. j + n - 1
    const CosSin* at_j = cs + angle_at<EPV>(j);
    const int first = PAIRS ? 2 * j : j, second = PAIRS ? 2 * j + EPV : sh.half + j;
    const int n1 = PAIRS ? min(EPV, 2 * n) : n, n2 = PAIRS ? 2 * n - n1 : n;
    float u[EPV], w[EPV];
    load_some<DT>(row, first, n1, u);
    if (n2 > 0) load_some<DT>(row, second, n2, w);
    else {
#pragma unroll
      for (int e = 0; e < EPV; ++e) w[e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      const CosSin t = at_j[min(e, n - 1)];
      float& fa = PAIRS ? (e < EPV / 2 ? u[2 * e] : w[2 * e - EPV]) : u[e];
      float& fb = PAIRS ? (e < EPV / 2 ? u[2 * e + 1] : w[2 * e + 1 - EPV]) : w[e];
      const double a = (double)fa, b = (double)fb;
      fa = (float)__builtin_fma(-b, t.s, a * t.c);
      fb = (float)__builtin_fma(a, t.s, b * t.c);
    }
    put(first, n1, u);
    if (n2 > 0) put(second, n2, w);
  }
  if (!skip_copies)
    for (int c = lane; c < sh.copies; c += kRopeLanes) {
      const int at = 2 * sh.half + c * EPV, n = min(EPV, sh.D - at);
      float u[EPV];
      load_some<DT>(row, at, n, u);
      put(at, n, u);
    }
}

}  // namespace sv
