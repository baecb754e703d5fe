// sv_sample: a token of every row under temperature, top-k, top-p and min-p, from a given random number.
//
// One workgroup per row.  Without warps, one sweep: weights relative to the largest entry of a piece of the row, in fp64; then the piece
// that holds u W, and its entries.  The warps only concern the upper tail of a row, so with them
//   sweep     the row's maximum m, and of every sixteen bytes the largest entry (its upper sixteen bits, in LDS); for a nucleus without
//             a K, the row's mass, in float32 and good to 4e-6
//   tau       a value that K entries reach: the K-th largest of the lanes' maxima, or of the vectors' (distinct entries of the
//             row), or a little less; for a nucleus a guess, and what min-p says
//   list      the entries that reach tau, by ascending token, from the few vectors that hold one
//   settle    counts and masses above the entries of the list; what is kept; its masses by token, and the one that holds u W
// up to 64 entries by one wavefront without a barrier.  A list that does not reach as far as the warps do (a deep nucleus, a K of thousands)
// is narrowed from both sides instead: a sweep counts and weighs, in float32, what lies above three values, until the stretch that holds the
// cutoff fits a list or is one value.  Where a decision lies within the float32 masses' error of its target, it is taken in fp64.
// Weights of what is drawn are fp64 (2^x as a polynomial: an error of 1e-15, where float32 exponentials would make 1 row in 300 of a flat
// 152064-entry distribution draw another token), and every sum has an order that the sizes fix, or terms that add exactly.
// What bounds it: 64 rows of 152064 bf16 entries 22 us, one row to a CU on 64 of 256 CUs (0.3 MB at what a
// workgroup can keep under way, then the chain from tau to the token); 512 rows of 128256 47 us, two rounds of the same (2.8 TB/s) with the warps' part of one
// row beside the sweep of another.
#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kDrawThreads = 512;
constexpr int kDrawWaves = kDrawThreads / kWave;
constexpr int kList = 2048;              // entries of the list
constexpr int kPieceVecs = 8;            // vectors of a lane in a piece: 4096 bfloat16 or 2048 float32 entries
constexpr int kOwn = kList / kDrawThreads;   // entries of the list that a thread owns
// Where a nucleus is guessed to end: above this many of the lanes' maxima, then above this many of the vectors'.  The first list is what one
// wavefront settles, the second what kList holds.  us, bf16, a generator's logits (one entry in a hundred 8 above the rest).  512 x 128256: T 0.7, top-p
// 0.8, 20, 40 and 80 lanes 69, 66 and 52; T 1, top-p 0.95, min-p 0.02 47.7, 47.5 and 47.3; 16 x 32000, T 0.7, top-p 0.8, 14.3, 15.4 and 19.0.  600, 1200
// and 1800 vectors, 512 x 128256, T 1, top-p 0.95 201, 110 and 202; T 1.3, top-p 0.8 250, 201 and 233; deeper ones do not fit (T 1.3, top-p
// 0.95 450 with each).
constexpr int kNucleusRank = 40;
constexpr int kDeepRank = 1200;
// The first list is passed over where the lanes' maxima above it hold less than this of the nucleus.  0.6, 0.85 and 1, us: 512 x 128256, T 1, top-p 0.95
// 117, 110 and 109, T 0.7, top-p 0.8 63, 66 and 59; 16 x 32000, T 1, top-p 0.95 32, 31 and 26.  (The maxima are not all that the list holds: it may
// do where they do not.)
constexpr double kReachedEnough = 0.85;
constexpr int kMaxKeys = 40960;          // vectors' maxima in LDS (80 KB); longer rows share one among several vectors
// Error of a float32 mass, relative: the exponent k of a weight is off by 2^-23 |k| (two roundings), which is 8.3e-8 |k| of the weight; an
// average over the mass has |k| <= 24 (2^24 entries that far down weigh as much as the first), and 25.3 where the weights refer to
// a whole number up to 1.3 above the largest entry.  v_exp_f32 adds 2^-23, and sums of eight terms 2^-21: 2.7e-6.  Nothing else adds to it: lanes'
// sums are fp64, and their references whole numbers, so that raising one scales its sum by a power of two.
constexpr double kMassError = 4e-6;

struct SampleArgs {
  const char* z;
  int64_t z_stride;                      // bytes
  int V, top_k;                          // 0: no K
  int share;                             // vectors that share a maximum in LDS
  double scale;                          // log2(e) / T
  double inv_t, top_p, min_log2;         // min_log2: log2(min_p), -inf without
  const double* u;
  int32_t* token;
  float* logprob;
  uint32_t* flags;
  // of rows that are read by more than one workgroup (null otherwise): every piece's mass and largest entry (+inf: a NaN)
  double* piece_mass;                    // [rows, pieces]
  float* piece_top;                      // [rows, pieces]
};

__device__ __forceinline__ uint32_t order_key(float f) {           // ascending
  const uint32_t u = __float_as_uint(f + 0.f);                     // (-0 is 0)
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_float(uint32_t k) { return __uint_as_float((k >> 31) ? (k & 0x7fffffffu) : ~k); }

// 2^k, k <= 1, to 1e-15: k = n + f with |f| <= 1/2, and the series of e^(f ln 2) up to the eleventh power (0.347^12 / 12! = 6e-15).
__device__ __forceinline__ double exp2_series(double k) {
  const double n = __builtin_rint(k), r = (k - n) * kLn2;
  double p = 1.0 / 39916800.0;
  p = __builtin_fma(p, r, 1.0 / 3628800.0);
  p = __builtin_fma(p, r, 1.0 / 362880.0);
  p = __builtin_fma(p, r, 1.0 / 40320.0);
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return k < -1000.0 ? 0.0 : __builtin_ldexp(p, (int)n);
}

// Weight in float32 of an entry `below` (<= 0) the largest one: hi + lo is the scale.
struct FastScale {
  float hi, lo;
  __device__ __forceinline__ float weight(float below) const {
    const float b = fmaxf(below, -1e30f);                // (-inf times lo is no -inf)
    return exp2_fast(__builtin_fmaf(b, hi, b * lo));
  }
  // The same relative to 2^ref, ref a whole number next to the exponent of the largest entry.
  __device__ __forceinline__ float whole(float top) const { return fminf(fmaxf(__builtin_ceilf(top * hi), kRefFloor), kRefCeil); }
  __device__ __forceinline__ float weight_to(float x, float ref) const {
    const float b = fmaxf(x, -1e30f);
    return exp2_fast(__builtin_fmaf(b, lo, __builtin_fmaf(b, hi, -ref)));
  }
};

struct alignas(16) DrawShared {
  uint64_t key[kList];                   // order key of a value above, token below
  double piece[kList];                   // masses of pieces of the row
  uint32_t vec[kList];                   // vectors of the list
  uint16_t lane_key[kDrawThreads];
  double d[2][kDrawWaves][4];            // sums of the wavefronts; slots alternate, so that a reduction takes one barrier
  int i[2][kDrawWaves][4];
  float wave_top[kDrawWaves];
  uint32_t wave_low[kDrawWaves];
  int n, hit, state, token;
  uint32_t found;
  double mass, value;
};

// Reductions over the workgroup.  Each writes one of two slots, so the readers of the last one are past it when it is written again.
struct Team {
  DrawShared& sh;
  int turn = 0;
  __device__ __forceinline__ int lane() const { return threadIdx.x & (kWave - 1); }
  __device__ __forceinline__ int wave() const { return threadIdx.x / kWave; }

  // The sum over eight lanes, the same in all of them.
  static_assert(kDrawWaves == 8, "eight lanes hold the wavefronts' sums");
  template <class T>
  static __device__ __forceinline__ T of_eight(T v) {
    v += lane_xor<1>(v);
    v += lane_xor<2>(v);
    return v + lane_xor<4>(v);
  }

  // Sums of up to three doubles and counts; a count is the wavefront's own already, the same in its lanes.
  template <int N, bool MASS>
  __device__ __forceinline__ void sums(double (&s)[N], int (&c)[N]) {
    turn ^= 1;
    if constexpr (MASS) {
      double w;
      if constexpr (N == 1) w = wave_scan_f64(s[0]);     // (lane 63)
      else w = wave_sum4_f64(s[0], N > 1 ? s[1 % N] : 0.0, N > 2 ? s[2 % N] : 0.0, 0.0);   // lanes 15, 31, 47
      if (N == 1 ? lane() == 63 : (lane() & 15) == 15) sh.d[turn][wave()][N == 1 ? 0 : lane() >> 4] = w;
    }
    if (lane() == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) sh.i[turn][wave()][k] = c[k];
    }
    __syncthreads();
    const int w = threadIdx.x & 7;                       // (a lane reads one wavefront's, and eight of them add up)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (MASS) s[k] = of_eight(sh.d[turn][w][k]);
      c[k] = of_eight(sh.i[turn][w][k]);
    }
  }
  __device__ __forceinline__ double sum(double v) {
    double s[1] = {v};
    int c[1] = {0};
    sums<1, true>(s, c);
    return s[0];
  }
  __device__ __forceinline__ int count(int of_wave) {
    double s[1];
    int c[1] = {of_wave};
    sums<1, false>(s, c);
    return c[0];
  }
  // Exclusive place of a thread's c items, or mass before its own, in the order of the threads; the total in every thread.
  __device__ __forceinline__ int place(int c, int* total) {
    const int incl = wave_scan_i32(c);
    turn ^= 1;
    if (lane() == kWave - 1) sh.i[turn][wave()][0] = incl;
    __syncthreads();
    const int w = threadIdx.x & 7, v = sh.i[turn][w][0];
    *total = of_eight(v);
    return of_eight(w < wave() ? v : 0) + incl - c;
  }
  __device__ __forceinline__ double place(double v, double* total) {
    const double incl = wave_scan_f64(v);
    turn ^= 1;
    if (lane() == kWave - 1) sh.d[turn][wave()][0] = incl;
    __syncthreads();
    const int w = threadIdx.x & 7;
    const double t = sh.d[turn][w][0];
    *total = of_eight(t);
    return of_eight(w < wave() ? t : 0.0) + (incl - v);
  }
};

__device__ __forceinline__ int wave_sum_i32(int c) { return __builtin_amdgcn_readlane(wave_scan_i32(c), kWave - 1); }

template <int DT>
struct Draw {
  static constexpr int EPV = Elem<DT>::per_vec;
  // the lower half of the order key of a bfloat16 value says nothing
  static constexpr uint32_t kQuantum = DT == DT_BF16 ? 1u << 16 : 1u;
  const SampleArgs& a;
  const char* row;
  DrawShared& sh;
  Team& team;
  double m;
  FastScale fast;

  __device__ __forceinline__ double weight_log2(float z) const { return ((double)z - m) * a.scale; }
  __device__ __forceinline__ double weight(float z) const { return exp2_series(weight_log2(z)); }

  // f(values, first token, entries) for every vector, in no order.
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    const int nvec = a.V / EPV;
    constexpr int U = 4;
    int i = threadIdx.x;
    for (; i + (U - 1) * kDrawThreads < nvec; i += U * kDrawThreads) {
      u32x4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = load_vec(row, i + u * kDrawThreads);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[EPV];
        unpack<DT>(q[u], x);
        f(x, (i + u * kDrawThreads) * EPV, EPV);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    for (; i < nvec; i += kDrawThreads) {
      float x[EPV];
      unpack<DT>(load_vec(row, i), x);
      f(x, i * EPV, EPV);
    }
    const int v0 = nvec * EPV, n = a.V - v0;
    if (n > 0 && threadIdx.x == 0) {
      float x[EPV];
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[e] = e < n ? load_elem<DT>(row, v0 + e) : -INFINITY;
      f(x, v0, n);
    }
  }

  // Mass of the entries with keys >= at, in fp64.
  __device__ __forceinline__ double mass_above(uint32_t at) {
    const float least = key_float(at);
    double s = 0.0;
    each([&](const float (&x)[EPV], int, int n) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < EPV; ++e) any |= x[e] >= least;
      if (!any) return;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        s += x[e] >= least && e < n ? weight(x[e]) : 0.0;
        if (e % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
    });
    return team.sum(s);
  }

  // Entries with keys >= each of three, and their masses in float32 terms.
  template <bool MASS>
  __device__ __forceinline__ void above(const uint32_t (&at)[3], int (&count)[3], double (&mass)[3]) {
    const float l0 = key_float(at[0]), l1 = key_float(at[1]), l2 = key_float(at[2]), top = (float)m;
    int c[3] = {0, 0, 0};
    double s[3] = {0.0, 0.0, 0.0};
    each([&](const float (&x)[EPV], int, int n) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < EPV; ++e) any |= x[e] >= l0;
      if (!any) return;
      float t[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const bool in = e < n, b0 = in && x[e] >= l0, b1 = in && x[e] >= l1, b2 = in && x[e] >= l2;
        c[0] += b0;
        c[1] += b1;
        c[2] += b2;
        if (MASS) {
          const float w = fast.weight(x[e] - top);
          t[0] += b0 ? w : 0.f;
          t[1] += b1 ? w : 0.f;
          t[2] += b2 ? w : 0.f;
        }
      }
      if (MASS) {
#pragma unroll
        for (int k = 0; k < 3; ++k) s[k] += (double)t[k];
      }
    });
#pragma unroll
    for (int k = 0; k < 3; ++k) count[k] = wave_sum_i32(c[k]);
    team.template sums<3, MASS>(s, count);
#pragma unroll
    for (int k = 0; k < 3; ++k) mass[k] = s[k];
  }

  // The entries with keys in [lo, hi) into sh.key, in no order; at most kList of them are there.
  __device__ __forceinline__ void collect(uint32_t lo, uint32_t hi) {
    const float least = key_float(lo);
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    each([&](const float (&x)[EPV], int v0, int n) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < EPV; ++e) any |= x[e] >= least;
      if (!any) return;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const uint32_t k = order_key(x[e]);
        if (e < n && k >= lo && k < hi) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < kList) sh.key[at] = ((uint64_t)k << 32) | (uint32_t)(v0 + e);
        }
      }
    });
    __syncthreads();
  }

  // Entries of a list that the threads own: keys (0: none) and weights.  The largest key c in [lo, hi) such that the entries >= c, with n_hi
  // and mass_hi above hi, are at least K (BY_COUNT) or weigh at least `target`; lo is such a key, hi is not.
  template <bool BY_COUNT>
  __device__ __forceinline__ uint32_t search(const uint32_t (&vk)[kOwn], const double (&w)[kOwn], uint32_t lo, uint32_t hi, int n_hi,
                                             double mass_hi, int K, double target) {
    int c_lo = 0x7fffffff, c_hi = 0;                     // entries of the list >= lo, >= hi
    while (hi - lo > kQuantum && c_lo - c_hi > 1) {
      const uint32_t quanta = (hi - lo + kQuantum - 1) / kQuantum, step = max(quanta / 4, 1u) * kQuantum;
      const uint32_t base = lo / kQuantum * kQuantum;    // (a bfloat16 key is told by its upper half)
      uint32_t p[3];
      double s[3] = {0.0, 0.0, 0.0};
      int c[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        p[k] = base + (k + 1) * step;
        int n = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
          const bool in = vk[j] >= p[k];
          n += (int)__popcll(__ballot(in));
          if (!BY_COUNT) s[k] += in ? w[j] : 0.0;
        }
        c[k] = n;
      }
      team.template sums<3, !BY_COUNT>(s, c);
#pragma unroll
      for (int k = 2; k >= 0; --k) {                     // (probes at or above hi do not count: it is not such a key)
        if (p[k] >= hi) continue;
        if (BY_COUNT ? n_hi + c[k] >= K : mass_hi + s[k] >= target) { lo = p[k]; c_lo = c[k]; break; }
        hi = p[k];
        c_hi = c[k];
      }
    }
    if (c_lo - c_hi == 1) {                              // one entry is left
#pragma unroll
      for (int j = 0; j < kOwn; ++j)
        if (vk[j] >= lo && vk[j] < hi) sh.found = vk[j];
      __syncthreads();
      lo = sh.found;
      __syncthreads();
    }
    return lo;
  }

  // The largest key c of the row such that the entries >= c are at least K, or weigh at least top_p of `all`; lo is such a key.  `all` is good
  // to kMassError, and summed again by make_exact() where a decision needs it.
  template <bool BY_COUNT, class Exact>
  __device__ __forceinline__ uint32_t narrow(int K, double& all, bool& exact, Exact&& make_exact, uint32_t lo, int n_lo) {
    uint32_t hi = order_key((float)m) + 1;               // above every entry
    int n_hi = 0;
    for (int round = 0; hi - lo > kQuantum; ++round) {
      if (n_lo - n_hi <= kList) {
        collect(lo, hi);
        const int n = min(sh.n, kList);
        const double over = BY_COUNT || n_hi == 0 ? 0.0 : mass_above(hi);
        // weights in units of 2^-41 of the largest of them: sums of 2^11 are exact, in any order
        const double unit = BY_COUNT ? 1.0 : __builtin_ldexp(1.0, max((int)__builtin_ceil(fmax(weight_log2(key_float(hi - 1)), -900.0)), -900) - 41);
        uint32_t vk[kOwn];
        double w[kOwn];
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
          const int i = threadIdx.x + j * kDrawThreads;
          vk[j] = i < n ? (uint32_t)(sh.key[i] >> 32) : 0u;
          w[j] = i < n && !BY_COUNT ? __builtin_rint(weight(key_float(vk[j])) / unit) * unit : 0.0;
        }
        const uint32_t cut = search<BY_COUNT>(vk, w, lo, hi, n_hi, over, K, a.top_p * all);
        if (BY_COUNT || exact) return cut;
        double at_cut = 0.0, past = 0.0;                 // masses of the list not below the cutoff, and above it
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
          at_cut += vk[j] >= cut ? w[j] : 0.0;
          past += vk[j] >= cut / kQuantum * kQuantum + kQuantum ? w[j] : 0.0;
        }
        at_cut = over + team.sum(at_cut) - a.top_p * all;
        past = a.top_p * all - over - team.sum(past);
        if (fmin(at_cut, past) > kMassError * all) return cut;
        make_exact();
        return search<BY_COUNT>(vk, w, lo, hi, n_hi, over, K, a.top_p * all);
      }
      uint32_t p[3];
      const uint32_t quarter = max((hi - lo) / 4, 1u);
#pragma unroll
      for (int k = 0; k < 3; ++k) p[k] = lo + min((k + 1) * quarter, hi - lo - 1);
      const float f0 = key_float(lo), f1 = key_float(hi - 1);
      if (round < 8 && f0 > -INFINITY) {                 // quarters of the values, which are nearer to quarters of the row
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          const float t = 0.25f * (k + 1);
          const uint32_t q = order_key(f0 * (1.f - t) + f1 * t);
          if (q > lo && q < hi) p[k] = q;
        }
        p[1] = max(p[1], p[0]);
        p[2] = max(p[2], p[1]);
      }
      int c[3];
      double s[3];
      above<!BY_COUNT>(p, c, s);
      for (int k = 2; k >= 0; --k) {
        bool yes;
        if (BY_COUNT) {
          yes = c[k] >= K;
        } else {
          if (fabs(s[k] - a.top_p * all) <= 2.0 * kMassError * all) {
            make_exact();
            s[k] = mass_above(p[k]);
          }
          yes = s[k] >= a.top_p * all;
        }
        if (yes) { lo = p[k]; n_lo = c[k]; break; }
        hi = p[k];
        n_hi = c[k];
      }
    }
    return lo;
  }

  // Index of the place that holds u W among places whose weights the threads own in order, w[j] that of place kOwn t + j; W; the mass before.
  __device__ __forceinline__ int place_of(const double (&w)[kOwn], double u, double* total, double* before) {
    const int i0 = threadIdx.x * kOwn;
    double mine = 0.0, W;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) mine += w[j];
    if (threadIdx.x == 0) { sh.hit = 0x7fffffff; sh.n = 0; }
    const double start = team.place(mine, &W), at = u * W;
    double run = start;
    int first = -1, last = -1;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      run += w[j];
      if (w[j] > 0.0) {
        last = i0 + j;
        if (first < 0 && run > at) first = last;
      }
    }
    if (first >= 0) atomicMin(&sh.hit, first);
    if (last >= 0) atomicMax(&sh.n, last);
    __syncthreads();
    const int i = sh.hit < kList ? sh.hit : sh.n;        // (u W rounded up to W: the last one)
    run = start;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      if (i0 + j == i) sh.mass = run;
      run += w[j];
    }
    __syncthreads();
    *total = W;
    *before = sh.mass;
    return i;
  }

  __device__ __forceinline__ double kept_weight(float z, float least) const {
    if (!(z >= least)) return 0.0;
    const double k = weight_log2(z);
    return k >= a.min_log2 ? exp2_series(k) : 0.0;
  }

  // Mass of what is kept of a piece: vectors (8 piece + j) 64 + lane.
  __device__ __forceinline__ double piece_sum(int piece, float least) const {
    const int lane = threadIdx.x & (kWave - 1), nvec = a.V / EPV;
    const int64_t base = (int64_t)piece * kPieceVecs * kWave + lane;
    u32x4 q[kPieceVecs];
#pragma unroll
    for (int j = 0; j < kPieceVecs; ++j)
      if (base + j * kWave < nvec) q[j] = load_vec(row, (int)(base + j * kWave));
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < kPieceVecs; ++j) {
      const int64_t i = base + j * kWave;
      if (i < nvec) {
        float x[EPV];
        unpack<DT>(q[j], x);
        bool any = false;
#pragma unroll
        for (int e = 0; e < EPV; ++e) any |= x[e] >= least;
        if (any) {
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            s += kept_weight(x[e], least);
            if (e % 2 == 1) __builtin_amdgcn_sched_barrier(0);
          }
        }
      } else if (i == nvec) {                            // the entries past the last vector
        for (int v = nvec * EPV; v < a.V; ++v) s += kept_weight(load_elem<DT>(row, v), least);
      }
    }
    return wave_sum_f64(s);
  }

  // From all entries not below `least` (and above min-p): masses of pieces, then the entries of one.
  __device__ __forceinline__ float draw_swept(float least, double u, int* token, double* total) {
    const int wave = threadIdx.x / kWave;
    const int pieces = a.V / EPV / (kPieceVecs * kWave) + 1;
    const int group = (pieces + kList - 1) / kList;      // pieces that share a mass
    const int groups = (pieces + group - 1) / group;
    for (int g = wave; g < groups; g += kDrawWaves) {
      double s = 0.0;
      for (int p = g * group; p < min((g + 1) * group, pieces); ++p) s += piece_sum(p, least);
      if ((threadIdx.x & (kWave - 1)) == 0) sh.piece[g] = s;
    }
    __syncthreads();
    double w[kOwn], W, begin;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) w[j] = (int)threadIdx.x * kOwn + j < groups ? sh.piece[threadIdx.x * kOwn + j] : 0.0;
    const int g = place_of(w, u, &W, &begin);
    *token = in_blocks(g * group * kPieceVecs, min((g + 1) * group, pieces) * kPieceVecs, begin, u * W, least);
    *total = W;
    return load_elem<DT>(row, *token);
  }

  // The token at which the running mass, `before` ahead of block b0, passes `at`, among blocks b0 .. b1 - 1 of 64 vectors; if it does not, the
  // last kept one.  A wavefront for each block.
  __device__ __forceinline__ int in_blocks(int b0, int b1, double before, double at, float least) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, nvec = a.V / EPV;
    int last_seen = -1;
    for (int b = b0; b < b1; b += kDrawWaves) {
      const int64_t i = b + wave < b1 ? (int64_t)(b + wave) * kWave + lane : (int64_t)nvec + 1;
      double w[EPV], s = 0.0;
      float x[EPV];
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[e] = -INFINITY;
      if (i < nvec) {
        unpack<DT>(load_vec(row, (int)i), x);
      } else if (i == nvec) {
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (i * EPV + e < a.V) x[e] = load_elem<DT>(row, (int)(i * EPV + e));
      }
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        s += w[e] = kept_weight(x[e], least);
        if (e % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
      if (threadIdx.x == 0) { sh.hit = 0x7fffffff; sh.n = -1; }
      double all;
      double run = before + team.place(s, &all);
      int first = -1, last = -1;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        run += w[e];
        if (w[e] > 0.0) {
          last = (int)(i * EPV + e);
          if (first < 0 && run > at) first = last;
        }
      }
      if (first >= 0) atomicMin(&sh.hit, first);
      if (last >= 0) atomicMax(&sh.n, last);
      __syncthreads();
      if (sh.hit != 0x7fffffff) return sh.hit;
      if (sh.n >= 0) last_seen = sh.n;
      before += all;
      __syncthreads();
    }
    return last_seen;
  }
};

template <int DT>
__device__ __forceinline__ void bad_row_out(const SampleArgs& a, int64_t r) {
  if (threadIdx.x != 0) return;
  a.token[r] = -1;
  if (a.logprob) a.logprob[r] = NAN;
  if (a.flags) a.flags[r] = SV_FLAG_BAD_ROW;
}

// A wavefront's piece of a row, vectors (PV piece + j) 64 + lane: its largest entry (+inf where a NaN is), and its mass relative to that.
template <int DT, int PV>
__device__ __forceinline__ float piece_of(const SampleArgs& a, const char* row, int piece, double* mass) {
  constexpr int EPV = Elem<DT>::per_vec;
  const int lane = threadIdx.x & (kWave - 1), nvec = a.V / EPV;
  const int64_t base = (int64_t)piece * PV * kWave + lane;
  u32x4 q[PV];
#pragma unroll
  for (int j = 0; j < PV; ++j)
    if (base + j * kWave < nvec) q[j] = load_vec(row, (int)(base + j * kWave));
  // (the entries past the last vector)
  const int past = base <= nvec && nvec < base + PV * kWave && (nvec - base) % kWave == 0 ? a.V - nvec * EPV : 0;
  float top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int j = 0; j < PV; ++j) {
    if (base + j * kWave >= nvec) continue;
    float x[EPV];
    unpack<DT>(q[j], x);
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      top = fmaxf(top, x[e]);
      nan |= x[e] != x[e];
    }
  }
  for (int e = 0; e < past; ++e) {
    const float x = load_elem<DT>(row, nvec * EPV + e);
    top = fmaxf(top, x);
    nan |= x != x;
  }
  top = wave_max_f32(top);
  // (bfloat16 unpacked again below: kept as floats they take 64 registers)
#pragma unroll
  for (int j = 0; j < PV; ++j)
    if constexpr (EPV == 8) asm volatile("" : "+v"(q[j]));
  double s = 0.0;
  if (top > -INFINITY) {
#pragma unroll
    for (int j = 0; j < PV; ++j) {
      if (base + j * kWave >= nvec) continue;
      float x[EPV];
      unpack<DT>(q[j], x);
#pragma unroll
      for (int e = 0; e < EPV; ++e) s += exp2_series(((double)x[e] - (double)top) * a.scale);
      if constexpr (EPV == 8) __builtin_amdgcn_sched_barrier(0);   // (eight weights side by side are enough; four are not)
    }
    for (int e = 0; e < past; ++e) s += exp2_series(((double)load_elem<DT>(row, nvec * EPV + e) - (double)top) * a.scale);
    s = wave_sum_f64(s);
  }
  *mass = s;
  return __ballot(nan) ? INFINITY : top;
}

// Few long rows without warps: a wavefront for each of their pieces, ahead of sample_plain_kernel.
template <int DT>
__global__ void __launch_bounds__(256) sample_pieces_kernel(SampleArgs a, int rows, int pieces) {
  const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const int r = (int)(at / pieces), piece = (int)(at - (int64_t)r * pieces);
  if (r >= rows) return;
  double mass;
  const float top = piece_of<DT, kPieceVecs>(a, a.z + r * a.z_stride, piece, &mass);
  if ((threadIdx.x & (kWave - 1)) == 0) {
    a.piece_mass[at] = mass;
    a.piece_top[at] = top;
  }
}

// No warps: masses of the pieces, from the sweep before or by the wavefronts in turn, one pass over the row; then the piece that holds u W.
// PV: vectors of a lane in a piece; two where the row is so short that pieces of eight leave wavefronts without one.
template <int DT, int PV>
__global__ void __launch_bounds__(kDrawThreads, 2) sample_plain_kernel(SampleArgs a) {
  constexpr int EPV = Elem<DT>::per_vec;
  __shared__ DrawShared sh;
  __shared__ float piece_top[kList];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  Team team{sh};
  Draw<DT> d{a, a.z + r * a.z_stride, sh, team, 0.0, {0.f, 0.f}};
  double u = a.u[r];
  const int pieces = a.V / EPV / (PV * kWave) + 1;
  const int group = (pieces + kList - 1) / kList, groups = (pieces + group - 1) / group;
  float row_top = -INFINITY;
  if (a.piece_mass) {
    for (int g = tid; g < groups; g += kDrawThreads) {
      sh.piece[g] = a.piece_mass[r * pieces + g];
      const float t = a.piece_top[r * pieces + g];
      piece_top[g] = t;
      row_top = fmaxf(row_top, t);
    }
    row_top = wave_max_f32(row_top);
  } else {
    for (int g = wave; g < groups; g += kDrawWaves) {
      float ref = -INFINITY;
      double sum = 0.0;
      for (int p = g * group; p < min((g + 1) * group, pieces); ++p) {
        double s;
        const float top = piece_of<DT, PV>(a, d.row, p, &s);
        if (top == -INFINITY) continue;
        if (top > ref) {
          sum = ref == -INFINITY ? 0.0 : sum * exp2_series(((double)ref - (double)top) * a.scale);
          ref = top;
        } else {
          s *= exp2_series(((double)top - (double)ref) * a.scale);
        }
        sum += s;
      }
      if (lane == 0) { sh.piece[g] = sum; piece_top[g] = ref; }
      row_top = fmaxf(row_top, ref);
    }
  }
  if (lane == 0) sh.wave_top[wave] = row_top;
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) top = fmaxf(top, sh.wave_top[w]);
  const double y = (double)top * a.scale;
  if (!(y >= (double)kRefFloor && y <= (double)kRefCeil) || u != u) return bad_row_out<DT>(a, r);
  u = fmin(fmax(u, 0.0), 1.0 - 0x1p-53);
  d.m = (double)top;
  double w[kOwn], W, begin;
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int i = tid * kOwn + j;
    w[j] = i < groups && sh.piece[i] > 0.0 ? sh.piece[i] * d.weight(piece_top[i]) : 0.0;
  }
  const int g = d.place_of(w, u, &W, &begin);
  const int token = d.in_blocks(g * group * PV, min((g + 1) * group, pieces) * PV, begin, u * W, -INFINITY);
  if (tid == 0) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = (float)(((double)load_elem<DT>(d.row, token) - d.m) * a.inv_t - log(W));
    if (a.flags) a.flags[r] = 0;
  }
}

template <int DT>
__global__ void __launch_bounds__(kDrawThreads, 4) sample_kernel(SampleArgs a) {
  constexpr int EPV = Elem<DT>::per_vec;
  __shared__ DrawShared sh;
  extern __shared__ __align__(16) uint16_t vec_key[];                // [n_keys rounded up to 8]
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  Team team{sh};
  Draw<DT> d{a, a.z + r * a.z_stride, sh, team, 0.0, {(float)a.scale, (float)(a.scale - (double)(float)a.scale)}};
  const bool use_k = a.top_k > 0, use_p = a.top_p < 1.0, use_min = a.min_log2 > -INFINITY;
  const int nvec = a.V / EPV, n_all = nvec + (a.V > nvec * EPV);   // the last one may be a part of a vector
  const int n_keys = (n_all + a.share - 1) / a.share;
  double u = a.u[r];

  // sweep: maxima of vectors, of the lane and the row; the row's mass relative to 2^ref of the lane
  float mine = -INFINITY, ref = kRefFloor;
  bool nan = false;
  double mass = 0.0;
  const bool weigh = use_p && !use_k;
  auto vector_at = [&](int i, float (&x)[EPV]) {         // vector i < n_all, the last one filled up with -inf
    if (i < nvec) {
      unpack<DT>(load_vec(d.row, i), x);
    } else {
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[e] = i * EPV + e < a.V ? load_elem<DT>(d.row, i * EPV + e) : -INFINITY;
    }
  };
  auto take = [&](const float (&x)[EPV]) {               // the largest of a vector's entries
    float t = x[0];
#pragma unroll
    for (int e = 1; e < EPV; ++e) t = fmaxf(t, x[e]);
#pragma unroll
    for (int e = 0; e < EPV; ++e) nan |= x[e] != x[e];
    const float m = fmaxf(mine, t);
    if (weigh && m > -INFINITY) {
      if (m > mine) {
        const float r = d.fast.whole(m);
        mass = __builtin_ldexp(mass, (int)(ref - r));
        ref = r;
      }
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < EPV; e += 2) s += d.fast.weight_to(x[e], ref) + d.fast.weight_to(x[e + 1], ref);
      mass += (double)s;
    }
    mine = m;
    return t;
  };
  if (a.share == 1) {
    // five vectors under way while the five before them are looked at
    constexpr int U = 5, kRound = U * kDrawThreads;
    auto load = [&](int i, u32x4 (&q)[U]) {
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (i + k * kDrawThreads < nvec) q[k] = load_vec(d.row, i + k * kDrawThreads);
    };
    auto look = [&](int i, const u32x4 (&q)[U]) {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int at = i + k * kDrawThreads;
        if (at >= n_all) continue;
        float x[EPV];
        if (at < nvec) unpack<DT>(q[k], x);
        else vector_at(at, x);
        vec_key[at] = (uint16_t)(order_key(take(x)) >> 16);
        __builtin_amdgcn_sched_barrier(0);               // (one at a time: their weights side by side take the registers of two more rows)
      }
    };
    u32x4 q0[U], q1[U];
    load(tid, q0);
    for (int i = tid; i < n_all; i += 2 * kRound) {
      load(i + kRound, q1);
      look(i, q0);
      if (i + kRound >= n_all) break;
      load(i + 2 * kRound, q0);
      look(i + kRound, q1);
    }
  } else {
    for (int k = tid; k < n_keys; k += kDrawThreads) {
      float all = -INFINITY;
      for (int i = k * a.share; i < min((k + 1) * a.share, n_all); ++i) {
        float x[EPV];
        vector_at(i, x);
        all = fmaxf(all, take(x));
      }
      vec_key[k] = (uint16_t)(order_key(all) >> 16);
    }
  }
  for (int k = n_keys + tid; k < ((n_keys + 7) & ~7); k += kDrawThreads) vec_key[k] = 0;
  const uint32_t lane_key = order_key(mine) >> 16;
  sh.lane_key[tid] = (uint16_t)lane_key;
  {
    const float hi = wave_max_f32(nan ? INFINITY : mine), lo = -wave_max_f32(-(float)lane_key);
    if (lane == 0) {
      sh.wave_top[wave] = __ballot(nan) ? INFINITY : hi;
      sh.wave_low[wave] = (uint32_t)lo;
    }
  }
  __syncthreads();
  float top = -INFINITY;
  uint32_t low_key = 0xffffu;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) {
    top = fmaxf(top, sh.wave_top[w]);
    low_key = min(low_key, sh.wave_low[w]);
  }
  const double y = (double)top * a.scale;
  if (!(y >= (double)kRefFloor && y <= (double)kRefCeil) || u != u) return bad_row_out<DT>(a, r);
  u = fmin(fmax(u, 0.0), 1.0 - 0x1p-53);
  d.m = (double)top;
  const uint32_t top_key = order_key(top) >> 16, none = order_key(-INFINITY);
  double all = 0.0;                                      // the row's mass
  bool exact = true;
  if (weigh) {
    const float top_ref = d.fast.whole(top);
    all = team.sum(mine == -INFINITY ? 0.0 : __builtin_ldexp(mass, (int)(ref - top_ref)));
    all *= exp2_series((double)top_ref - ((double)top * (double)d.fast.hi + (double)top * (double)d.fast.lo));
    exact = false;
  }
  auto make_exact = [&]() {
    if (!exact) all = d.mass_above(none);
    exact = true;
  };
  if (weigh && fabs(y) >= 0x1p22) make_exact();          // (the whole numbers of float32 next to it may be farther off)

  // A sixteen-bit key that at least `want` of the keys counted by count(probe) reach, and few more than that if there is such a one; the keys
  // lie between `from`, which `want` of them reach, and `to`.
  auto select = [&](uint32_t from, uint32_t to, int want, auto&& count) {
    const uint32_t differ = from ^ to;
    if (differ == 0) return from;
    int bit = 31 - __builtin_clz(differ);
    uint32_t t = from & ~((2u << bit) - 1u);
    for (; bit >= 0; --bit) {
      const uint32_t probe = t | (1u << bit);
      const int c = count(probe);
      if (c >= want) t = probe;
      if (c >= want && c <= want + (want < 40 ? 8 : want / 8)) break;
    }
    return t;
  };
  const int own = ((n_keys + kDrawThreads * 8 - 1) / (kDrawThreads * 8)) * 8;    // keys of a thread, in order
  auto each_key = [&](auto&& f) {                        // f(key, index) of the thread's keys, eight of them loaded at a time
    for (int k = tid * own; k < min((tid + 1) * own, n_keys); k += 8) {
      const u32x4 q = *reinterpret_cast<const u32x4*>(vec_key + k);
#pragma unroll
      for (int e = 0; e < 8; ++e) f((q[e / 2] >> (16 * (e % 2))) & 0xffffu, k + e);
    }
  };
  uint32_t min_key = none;
  if (use_min) {
    // (a step of a float32 below, where the weight is looked at again)
    const double zm = d.m + a.min_log2 / a.scale;
    if (zm > -3e38) min_key = max(order_key((float)zm) - 2, none);
  }

  bool done = false;
  int token = 0;
  double W = 0.0;
  float z = 0.f;
  for (int attempt = 0; attempt < 2 && !done; ++attempt) {
    // tau
    int want = use_k ? a.top_k : (use_p ? kNucleusRank : 0);
    if (attempt > 0) want = a.V <= kList ? 0 : min(kDeepRank, (n_keys * 2 + 2) / 3);
    uint32_t tau = none;
    // lanes whose maximum reaches a key: every wavefront by itself, eight of them in a lane
    const u32x4 q = *reinterpret_cast<const u32x4*>(sh.lane_key + 8 * lane);
    auto lanes = [&](uint32_t probe) {
      int c = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) c += (int)__popcll(__ballot(((q[e / 2] >> (16 * (e % 2))) & 0xffffu) >= probe));
      return c;
    };
    if (!use_k && use_min && lanes(min_key >> 16) <= kDrawThreads / 2) {
      tau = none;                                        // few entries are above what min-p drops: all of them
    } else if (want > 0 && want <= kDrawThreads && attempt == 0) {
      tau = select(low_key, top_key, want, lanes) << 16;
      if (weigh && tau > min_key) {
        // a nucleus that the lanes' maxima above tau are far from filling is deeper than their list
        const double reached = team.sum(lane_key >= (tau >> 16) ? (double)d.fast.weight(mine - top) : 0.0);
        if (reached < kReachedEnough * a.top_p * all) continue;
      }
    } else if (want > 0 && want <= n_keys) {
      // three probes a step
      uint32_t lo = low_key, hi = top_key + 1;           // `want` vectors reach lo, fewer reach hi
      for (bool first = true; hi - lo > 1; first = false) {
        const uint32_t step = max((hi - lo) / 4, 1u);
        uint32_t p[3];
        int c[3] = {0, 0, 0};
        double unused[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) p[k] = first ? (k == 0 ? lo : lo + (hi - lo) * k / 3) : min(lo + (k + 1) * step, hi);
        for (int k = 8 * tid; k < n_keys; k += 8 * kDrawThreads) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(vec_key + k);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t key = (x[e / 2] >> (16 * (e % 2))) & 0xffffu;
#pragma unroll
            for (int n = 0; n < 3; ++n) c[n] += key >= p[n];
          }
        }
        // (two counts in a word: of 64 lanes with at most 80 keys each)
        const int both = wave_sum_i32(c[0] | (c[1] << 16));
        c[0] = both & 0xffff;
        c[1] = both >> 16;
        c[2] = wave_sum_i32(c[2]);
        team.template sums<3, false>(unused, c);
        if (first && c[0] < want) { hi = lo; lo = 0; continue; }   // (not even the lowest of the lanes' maxima is reached by as many)
        int reached = n_keys;
#pragma unroll
        for (int k = 2; k >= 0; --k) {
          if (p[k] >= hi) continue;
          if (c[k] >= want) { lo = p[k]; reached = c[k]; break; }
          hi = p[k];
        }
        if (reached <= want + want / 8) break;
      }
      tau = lo << 16;
    }
    tau = max(tau, none);
    if (!use_k) tau = max(tau, min_key);                 // (the K-th value may lie below what min-p keeps)
    if (use_k && want > n_keys) break;
    // the vectors that reach it, in order
    int c = 0, n_vec, n;
    each_key([&](uint32_t key, int k) { c += key >= (tau >> 16) && k < n_keys; });
    if (a.share > 1) {
      c = 0;
      each_key([&](uint32_t key, int k) {
        if (key >= (tau >> 16) && k < n_keys) c += min(a.share, n_all - k * a.share);
      });
    }
    int at = team.place(c, &n_vec);
    if (n_vec > kList) break;
    if (c > 0)
      each_key([&](uint32_t key, int k) {
        if (key >= (tau >> 16) && k < n_keys)
          for (int i = k * a.share; i < min((k + 1) * a.share, n_all); ++i) sh.vec[at++] = (uint32_t)i;
      });
    __syncthreads();
    // their entries
    u32x4 held[kOwn];
    int v0[kOwn];
    const float least = key_float(tau);
    const int per = (n_vec + kDrawThreads - 1) / kDrawThreads;   // vectors of a thread
    c = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = tid * per + j;
      v0[j] = j < per && i < n_vec ? (int)sh.vec[i] : -1;
    }
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
      if (v0[j] >= 0 && v0[j] < nvec) held[j] = load_vec(d.row, v0[j]);
    auto entries = [&](int j, float (&x)[EPV]) {
      if (v0[j] < nvec) unpack<DT>(held[j], x);
      else vector_at(v0[j], x);
    };
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      if (v0[j] < 0) continue;
      float x[EPV];
      entries(j, x);
#pragma unroll
      for (int e = 0; e < EPV; ++e) c += x[e] >= least && v0[j] * EPV + e < a.V;
    }
    at = team.place(c, &n);
    if (n > kList) break;
    if (c > 0) {
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        if (v0[j] < 0) continue;
        float x[EPV];
        entries(j, x);
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (x[e] >= least && v0[j] * EPV + e < a.V) sh.key[at++] = ((uint64_t)order_key(x[e]) << 32) | (uint32_t)(v0[j] * EPV + e);
      }
    }
    __syncthreads();
    if (use_k && n < a.top_k) break;
    const bool whole_min = use_min && tau <= min_key;    // the list holds all that min-p keeps
    if (n <= kWave) {
      // one wavefront, a lane for each entry, by ascending token.  state: 0 settled, 1 does not reach, 2 too near a decision
      for (int pass = 0; pass < 2; ++pass) {
        if (wave == 0) {
          const uint64_t key = lane < n ? sh.key[lane] : 0;
          const uint32_t vk = (uint32_t)(key >> 32);
          const float v = key_float(vk);
          const double k2 = d.weight_log2(v);
          double w = lane < n ? exp2_series(k2) : 0.0;
          bool keep = lane < n;
          int state = 0;
          const int n4 = (n + 3) & ~3;                   // (lanes without an entry have key and weight 0)
          if (use_k) {
            int above = 0;                               // entries of a larger value
            for (int j = 0; j < n4; j += 4) {
#pragma unroll
              for (int e = 0; e < 4; ++e) above += (uint32_t)__builtin_amdgcn_readlane(vk, j + e) > vk;
            }
            keep = keep && above < a.top_k;
          }
          if (use_p) {
            if (!keep) w = 0.0;
            double above[2] = {0.0, 0.0};                // masses of larger values
            const double sum = wave_sum_f64(w);
            for (int j = 0; j < n4; j += 4) {
#pragma unroll
              for (int e = 0; e < 4; ++e) above[e & 1] += (uint32_t)__builtin_amdgcn_readlane(vk, j + e) > vk ? lane_f64(w, j + e) : 0.0;
            }
            above[0] += above[1];
            const double target = a.top_p * (use_k ? sum : all);
            const double band = use_k || exact ? 0.0 : kMassError * all;
            if (__ballot(keep && fabs(above[0] - target) < band) || fabs(sum - target) < band) state = 2;
            else if (!(sum >= target) && !use_k && !whole_min) state = 1;
            keep = keep && above[0] < target;
          } else if (!use_k && !whole_min) {
            state = 1;
          }
          keep = keep && k2 >= a.min_log2;
          w = keep ? w : 0.0;
          const double incl = wave_scan_f64(w), total = lane_f64(incl, kWave - 1);
          const uint64_t hits = __ballot(w > 0.0 && incl > u * total), any = __ballot(w > 0.0);
          const int i = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(any);
          if (lane == i) {
            sh.token = (int)(uint32_t)key;
            sh.value = (double)v;
          }
          if (lane == 0) { sh.state = state; sh.mass = total; }
        }
        __syncthreads();
        const int state = sh.state;
        if (state == 0) {
          token = sh.token;
          z = (float)sh.value;
          W = sh.mass;
          done = true;
        }
        if (state != 2) break;
        make_exact();                                    // (its barrier lets all read the state first)
      }
    } else {
      // the workgroup, up to kOwn entries a thread, by ascending token
      uint32_t vk[kOwn];
      double w[kOwn];
      const int per_n = (n + kDrawThreads - 1) / kDrawThreads;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        const int i = tid * per_n + j;
        const bool in = j < per_n && i < n;
        vk[j] = in ? (uint32_t)(sh.key[i] >> 32) : 0u;
        w[j] = in ? d.weight(key_float(vk[j])) : 0.0;
      }
      const uint32_t past = order_key(top) + 1;
      auto mass_at = [&](uint32_t probe) {
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) s += vk[j] >= probe ? w[j] : 0.0;
        return team.sum(s);
      };
      uint32_t cut = tau;
      if (use_k) cut = d.template search<true>(vk, w, tau, past, 0, 0.0, a.top_k, 0.0);
      bool settled = use_k || use_p || whole_min;
      if (use_p) {
        const double listed = mass_at(cut);
        if (use_k) all = listed;
        if (!exact && fabs(listed - a.top_p * all) < kMassError * all) make_exact();
        if (listed >= a.top_p * all) {
          const uint32_t kth = cut;
          cut = d.template search<false>(vk, w, kth, past, 0, 0.0, 0, a.top_p * all);
          if (!exact) {
            const double at_cut = mass_at(cut), over = mass_at(cut / Draw<DT>::kQuantum * Draw<DT>::kQuantum + Draw<DT>::kQuantum), target = a.top_p * all;
            if (at_cut - target < kMassError * all || target - over < kMassError * all) {
              make_exact();
              cut = d.template search<false>(vk, w, kth, past, 0, 0.0, 0, a.top_p * all);
            }
          }
        } else {
          settled = whole_min;
        }
      }
      if (settled) {
        double kept[kOwn], before;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) kept[j] = vk[j] >= cut && w[j] > 0.0 && d.weight_log2(key_float(vk[j])) >= a.min_log2 ? w[j] : 0.0;
        // (place_of counts kOwn places a thread; threads own per_n entries)
        const int i = d.place_of(kept, u, &W, &before);
        const uint64_t key = sh.key[(i / kOwn) * per_n + i % kOwn];
        token = (int)(uint32_t)key;
        z = key_float((uint32_t)(key >> 32));
        done = true;
      }
    }
    if (use_k || !use_p) break;
  }
  if (!done) {
    __syncthreads();
    uint32_t least = none;                               // keys below it are dropped
    if (use_k) {
      least = d.template narrow<true>(a.top_k, all, exact, make_exact, none, a.V);
      if (use_p) all = d.mass_above(least);
    }
    if (use_p) least = d.template narrow<false>(0, all, exact, make_exact, least, a.V);
    z = d.draw_swept(key_float(least), u, &token, &W);
  }
  if (tid == 0) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = (float)(((double)z - d.m) * a.inv_t - log(W));
    if (a.flags) a.flags[r] = 0;
  }
}

// Whether rows without warps are read by more than one workgroup each: a compute unit forms 2.2 to 2.6 weights in a nanosecond, so a second launch
// (4 us) pays for long rows that leave most of the card idle.  One launch / two, us: bf16 64 x 16384 15.4 / 17.4, 64 x 32000 17.6 / 17.3, 64 x 152064
// 58 / 26, 192 x 152064 67 / 52, 256 x 152064 69 / 68.
inline bool sample_splits(int rows, int V) { return rows <= 192 && V >= 32000 && V <= (1 << 21); }
inline int sample_pieces(int V, int e) { return V / (16 / e) / (kPieceVecs * kWave) + 1; }
inline size_t sample_top_at(int rows, int V, int e) { return ws_round((size_t)rows * sample_pieces(V, e) * 8); }

}  // namespace sv

extern "C" size_t sv_sample_workspace_bytes(int rows, int V, int dtype) {
  const int e = sv::elem_bytes(dtype);
  if (rows < 1 || V < 1 || V > (1 << 24) || e == 0) return 0;
  if (!sv::sample_splits(rows, V)) return 0;
  return sv::sample_top_at(rows, V, e) + sv::ws_round((size_t)rows * sv::sample_pieces(V, e) * 4);
}

extern "C" int sv_sample(const void* z, int64_t z_stride, int rows, int V, int dtype, float temperature, int top_k, float top_p,
                         float min_p, const double* u, int32_t* token, float* logprob_or_null, uint32_t* flags_or_null,
                         void* ws_or_null, size_t ws_bytes, sv_stream_t stream) {
  using namespace sv;
  const int e = elem_bytes(dtype);
  SV_REQUIRE(e != 0, SV_ERR_DTYPE);
  SV_REQUIRE(rows >= 0 && V >= 1 && z_stride >= V, SV_ERR_INVALID_ARG);
  Scale sc;
  SV_REQUIRE(scale_of(temperature, &sc) && top_p > 0.f && min_p >= 0.f && min_p <= 1.f, SV_ERR_INVALID_ARG);
  SV_REQUIRE(V <= (1 << 24) && z_stride < (1ll << 40), SV_ERR_TOO_LARGE);
  if (rows == 0) return SV_OK;
  SV_REQUIRE(z && u && token, SV_ERR_NULL);
  SV_REQUIRE(is_aligned(z, e) && is_aligned(u, 8) && is_aligned(token, 4) && is_aligned(logprob_or_null, 4) &&
                 is_aligned(flags_or_null, 4),
             SV_ERR_ALIGN);
  const int vectors = (V + 16 / e - 1) / (16 / e), share = (vectors + kMaxKeys - 1) / kMaxKeys;
  SampleArgs a{static_cast<const char*>(z), z_stride * e, V, top_k > 0 && top_k < V ? top_k : 0, share, kLog2e / (double)temperature,
               sc.inv_t, top_p < 1.f ? (double)top_p : 1.0, min_p > 0.f ? __builtin_log2((double)min_p) : -INFINITY, u, token,
               logprob_or_null, flags_or_null, nullptr, nullptr};
  const bool plain = a.top_k == 0 && a.top_p >= 1.0 && min_p == 0.f;
  const int pieces = sample_pieces(V, e);
  bool shorter = pieces < 2 * kDrawWaves;
  if (ws_or_null && sample_splits(rows, V)) {
    SV_REQUIRE(is_aligned(ws_or_null, kWsAlign) && ws_bytes >= sv_sample_workspace_bytes(rows, V, dtype), SV_ERR_WORKSPACE);
    if (plain) {
      a.piece_mass = static_cast<double*>(ws_or_null);
      a.piece_top = reinterpret_cast<float*>(static_cast<char*>(ws_or_null) + sample_top_at(rows, V, e));
      shorter = false;
      const dim3 grid((unsigned)(((long long)rows * pieces + 3) / 4));
      if (dtype == SV_F32) hipLaunchKernelGGL(sample_pieces_kernel<DT_F32>, grid, dim3(256), 0, as_stream(stream), a, rows, pieces);
      else hipLaunchKernelGGL(sample_pieces_kernel<DT_BF16>, grid, dim3(256), 0, as_stream(stream), a, rows, pieces);
    }
  }
  const size_t lds = plain ? 0 : ((size_t)(vectors + share - 1) / share + 7) / 8 * 16;
  in_launches(rows, kDrawThreads, [&](long long first, dim3 grid) {
    SampleArgs b = a;
    b.z += first * b.z_stride;
    b.u += first;
    b.token += first;
    if (b.logprob) b.logprob += first;
    if (b.flags) b.flags += first;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kDrawThreads), lds, as_stream(stream), b); };
    if (!plain) {
      if (dtype == SV_F32) go(sample_kernel<DT_F32>); else go(sample_kernel<DT_BF16>);
    } else if (shorter) {
      if (dtype == SV_F32) go(sample_plain_kernel<DT_F32, 2>); else go(sample_plain_kernel<DT_BF16, 2>);
    } else {
      if (dtype == SV_F32) go(sample_plain_kernel<DT_F32, kPieceVecs>); else go(sample_plain_kernel<DT_BF16, kPieceVecs>);
    }
  });
  return launch_status();
}
