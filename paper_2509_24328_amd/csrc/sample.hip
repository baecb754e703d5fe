// sv_sample: a token of every row under temperature, top-k, top-p and min-p, from a given random number.
//
// One workgroup per row.  Without warps, one sweep: weights relative to the largest entry of a piece of the row, in fp64; then the piece
// that holds u W, and its entries.  The warps only concern the upper tail of a row, so with them
//   sweep     the row's maximum m, and of every sixteen bytes the largest entry (its upper sixteen bits, in LDS); for a nucleus without
//             a K, the row's mass, in float32 and good to 4e-6
//   tau       a value that K entries reach: the K-th largest of the lanes' maxima, or of the vectors' (distinct entries of the
//             row); for a nucleus a guess, and what min-p says
//   list      the entries that reach tau, by ascending token, from the few vectors that hold one
//   settle    counts and masses above each entry of the list; what is kept; its masses by token, and the one that holds u W
// up to 64 entries by one wavefront without a barrier.  A list that does not reach as far as the warps do (a deep nucleus, a K of thousands)
// is narrowed instead: sweeps count and weigh what lies above a value, until the stretch that holds the cutoff fits a list or is one
// value.  Where a decision lies within the float32 mass's error of its target, the mass is summed again in fp64.
// Weights are fp64 (2^x as a polynomial: an error of 1e-15, where float32 exponentials would make 1 row in 300 of a flat 152064-entry
// distribution draw another token), and every sum has an order that the sizes fix.
#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kDrawThreads = 512;
constexpr int kDrawWaves = kDrawThreads / kWave;
constexpr int kList = 2048;              // entries of the list
constexpr int kPieceVecs = 8;            // vectors of a lane in a piece: 4096 bfloat16 or 2048 float32 entries
constexpr int kOwn = kList / kDrawThreads;   // entries of the list that a thread owns
constexpr int kNucleusRank = 40;         // first guess of a nucleus: the entries above this many lane maxima
constexpr int kDeepRank = 1200;          // second guess: above this many vectors' maxima
constexpr int kMaxKeys = 40960;          // vectors' maxima in LDS (80 KB); longer rows share one among several vectors
// Error of the float32 mass, relative: the exponent k of a weight is off by 2^-23 |k| (difference and product), which is 8.3e-8 |k| of the
// weight; an average over the mass has |k| <= 24 (2^24 entries that far down weigh as much as the first).  Up to six factors of v_exp_f32
// (a lane's maximum is raised a few times), 2^-23 each, and 2^-21 for sums of eight terms: 3.3e-6.
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
};

__device__ __forceinline__ uint32_t order_key(float f) {           // ascending
  const uint32_t u = __float_as_uint(f + 0.f);                     // (-0 is 0)
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_float(uint32_t k) { return __uint_as_float((k >> 31) ? (k & 0x7fffffffu) : ~k); }

// 2^k, k <= 0, to 1e-15: k = n + f with |f| <= 1/2, and the series of e^(f ln 2) up to the eleventh power (0.347^12 / 12! = 6e-15).
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

struct DrawShared {
  uint32_t vec[kList];                   // vectors of the list
  int count[2][kDrawWaves];
  uint64_t key[kList];                   // order key above, ~token below: sorted descending
  double cum[kList];                     // masses down the list, or of the kept entries up to a token
  double wave_d[kDrawWaves], out_d[2];
  int wave_i[kDrawWaves], out_i[2];
  uint32_t wave_u[kDrawWaves];
  int n, hit;
};

// Sum over the workgroup of a double and an int, in every thread.
__device__ __forceinline__ void block_sums(double& d, int& c, DrawShared& sh) {
  const int wave = threadIdx.x / kWave;
  const double dw = wave_sum_f64(d);
  const int cw = __builtin_amdgcn_readlane(wave_scan_i32(c), kWave - 1);
  if ((threadIdx.x & (kWave - 1)) == 0) { sh.wave_d[wave] = dw; sh.wave_i[wave] = cw; }
  __syncthreads();
  double ds = 0.0;
  int cs = 0;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) { ds += sh.wave_d[w]; cs += sh.wave_i[w]; }
  __syncthreads();
  d = ds;
  c = cs;
}

// Inclusive scan of the workgroup's values in the order of the threads; total in every thread.
__device__ __forceinline__ double block_scan(double v, double* total, DrawShared& sh) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const double incl = wave_scan_f64(v);
  if (lane == kWave - 1) sh.wave_d[wave] = incl;
  __syncthreads();
  double before = 0.0, all = 0.0;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) {
    if (w == wave) before = all;
    all += sh.wave_d[w];
  }
  __syncthreads();
  *total = all;
  return before + incl;
}

template <int DT>
struct Draw {
  static constexpr int EPV = Elem<DT>::per_vec;
  const SampleArgs& a;
  const char* row;
  DrawShared& sh;
  double m;

  __device__ __forceinline__ double weight_log2(float z) const { return ((double)z - m) * a.scale; }
  __device__ __forceinline__ double weight(float z) const { return exp2_series(weight_log2(z)); }

  // f(value, token) for every entry, in no order.
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

  // Entries with keys >= at: their number and, if asked for, their mass.
  __device__ __forceinline__ void above(uint32_t at, bool masses, int& count, double& mass) {
    const float least = key_float(at);
    int c = 0;
    double s = 0.0;
    each([&](const float (&x)[EPV], int, int n) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const bool in = x[e] >= least && e < n;
        c += in;
        any |= in;
      }
      if (masses && any) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) s += x[e] >= least && e < n ? weight(x[e]) : 0.0;
      }
    });
    block_sums(s, c, sh);
    count = c;
    mass = s;
  }

  // Lists the entries with keys in [lo, hi) (hi 0: no upper bound), sorted descending; their number.  (More than kList: not all.)
  __device__ __forceinline__ int list(uint32_t lo, uint32_t hi) {
    const float least = key_float(lo);
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    each([&](const float (&x)[EPV], int v0, int n) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < EPV; ++e) any |= x[e] >= least;
      if (!any || __hip_atomic_load(&sh.n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) > kList) return;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const uint32_t k = order_key(x[e]);
        if (e < n && k >= lo && (hi == 0 || k < hi)) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < kList) sh.key[at] = ((uint64_t)k << 32) | (uint32_t)~(uint32_t)(v0 + e);
        }
      }
    });
    __syncthreads();
    const int n = sh.n;
    if (n <= kList) sort(n);
    return n;
  }

  // sh.key[0 .. n) descending.
  __device__ __forceinline__ void sort(int n) {
    const int tid = threadIdx.x;
    if (n <= 256) {                                     // every key counts those above it (keys differ)
      const uint64_t mine = tid < n ? sh.key[tid] : 0;
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += sh.key[j] > mine;
      __syncthreads();
      if (tid < n) sh.key[rank] = mine;
      __syncthreads();
      return;
    }
    int n2 = 512;
    while (n2 < n) n2 <<= 1;
    for (int i = n + tid; i < n2; i += kDrawThreads) sh.key[i] = 0;
    __syncthreads();
    for (int k2 = 2; k2 <= n2; k2 <<= 1)
      for (int j = k2 >> 1; j > 0; j >>= 1) {
        const int pairs = n2 / 2;
        for (int p = tid; p < pairs; p += kDrawThreads) {
          const int i = 2 * p - (p & (j - 1)), o = i + j;
          const uint64_t x = sh.key[i], y = sh.key[o];
          if (((i & k2) == 0) == (x < y)) { sh.key[i] = y; sh.key[o] = x; }
        }
        __syncthreads();
      }
  }

  __device__ __forceinline__ float list_value(int i) const { return key_float((uint32_t)(sh.key[i] >> 32)); }

  // Masses down the list: sh.cum[i] = before + the weights of entries 0 .. i.
  __device__ __forceinline__ void masses(int n, double before) {
    const int i0 = threadIdx.x * kOwn;
    double w[kOwn], mine = 0.0, total;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) mine += w[j] = i0 + j < n ? weight(list_value(i0 + j)) : 0.0;
    double run = before + (block_scan(mine, &total, sh) - mine);
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      run += w[j];
      if (i0 + j < n) sh.cum[i0 + j] = run;
    }
    __syncthreads();
  }

  // First index whose mass reaches `target`, or n.
  __device__ __forceinline__ int reach(int n, double target) {
    if (threadIdx.x == 0) sh.hit = n;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kDrawThreads)
      if (sh.cum[i] >= target && (i == 0 || !(sh.cum[i - 1] >= target))) atomicMin(&sh.hit, i);
    __syncthreads();
    return sh.hit;
  }

  // The largest key c such that the entries >= c are at least K (by_count) or weigh at least `target`; lo is such a key, hi (0: none) is
  // not, with n_hi entries and a mass of mass_hi not below it.
  __device__ __forceinline__ uint32_t narrow(bool by_count, int K, double target, uint32_t lo, int n_lo, uint32_t hi, int n_hi,
                                             double mass_hi) {
    const uint32_t top = order_key((float)m) + 1;        // above every entry
    if (hi == 0) hi = top;
    for (int round = 0; hi - lo > 1; ++round) {
      if (n_lo - n_hi <= kList) {
        const int n = list(lo, hi);
        int i = 0;
        if (by_count) {
          i = K - n_hi - 1;
        } else {
          masses(n, mass_hi);
          i = reach(n, target);
        }
        // (not reached by rounding: the lowest)
        const uint32_t c = (uint32_t)(sh.key[max(min(i, n - 1), 0)] >> 32);
        __syncthreads();
        return c;
      }
      uint32_t mid = lo + (hi - lo) / 2;
      if (round < 12) {                                  // halves of the values first, which are nearer to halves of the row
        const float v = 0.5f * key_float(lo) + 0.5f * key_float(hi);
        const uint32_t k = order_key(v);
        if (v > -INFINITY && k > lo && k < hi) mid = k;
      }
      int c;
      double s;
      above(mid, !by_count, c, s);
      if (by_count ? c >= K : s >= target) { lo = mid; n_lo = c; }
      else { hi = mid; n_hi = c; mass_hi = s; }
    }
    return lo;
  }

  // Index of the place that holds u W among n places whose weights the threads own in order, w[j] that of place kOwn t + j; W; the mass before.
  __device__ __forceinline__ int place_of(const double (&w)[kOwn], int n, double u, double* total, double* before) {
    const int i0 = threadIdx.x * kOwn;
    double mine = 0.0, W;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) mine += w[j];
    if (threadIdx.x == 0) { sh.hit = 0x7fffffff; sh.n = 0; }
    const double start = block_scan(mine, &W, sh) - mine, at = u * W;
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
    const int i = sh.hit < n ? sh.hit : sh.n;            // (u W rounded up to W: the last one)
    run = start;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      if (i0 + j == i) sh.out_d[0] = run;
      run += w[j];
    }
    __syncthreads();
    *total = W;
    *before = sh.out_d[0];
    return i;
  }

  __device__ __forceinline__ double kept_weight(float z, float least) const {
    if (!(z >= least)) return 0.0;
    const double k = weight_log2(z);
    return k >= a.min_log2 ? exp2_series(k) : 0.0;
  }

  // Weights of a piece, entry e of vector j of this lane: entries (piece * 8 + j) * 64 + lane, EPV of them.  sums[j]: of a vector.
  __device__ __forceinline__ double piece_sum(int piece, float least) const {
    const int lane = threadIdx.x & (kWave - 1), nvec = a.V / EPV;
    const int64_t base = (int64_t)piece * kPieceVecs * kWave + lane;
    u32x4 q[kPieceVecs];
#pragma unroll
    for (int j = 0; j < kPieceVecs; ++j) {
      const int64_t i = base + j * kWave;
      if (i < nvec) q[j] = load_vec(row, (int)i);
    }
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
          for (int e = 0; e < EPV; ++e) s += kept_weight(x[e], least);
        }
      } else if (i == nvec) {                            // the entries past the last vector
        for (int v = nvec * EPV; v < a.V; ++v) s += kept_weight(load_elem<DT>(row, v), least);
      }
    }
    return wave_sum_f64(s);
  }

  // From all entries not below `least` (and above min-p): masses of pieces, then the entries of one.
  __device__ __forceinline__ float draw_swept(float least, double u, int* token, double* total) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int pieces = a.V / EPV / (kPieceVecs * kWave) + 1;
    double* mass = sh.cum;                               // (the list's places: pieces are gathered so that there are at most kList of them)
    const int group = (pieces + kList - 1) / kList;      // pieces that share a mass
    const int groups = (pieces + group - 1) / group;
    for (int gI = wave; gI < groups; gI += kDrawWaves) {
      double s = 0.0;
      for (int p = gI * group; p < min((gI + 1) * group, pieces); ++p) s += piece_sum(p, least);
      if (lane == 0) mass[gI] = s;
    }
    __syncthreads();
    double w[kOwn], W, begin;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) w[j] = (int)threadIdx.x * kOwn + j < groups ? mass[threadIdx.x * kOwn + j] : 0.0;
    const int gI = place_of(w, groups, u, &W, &begin);
    *token = in_pieces(gI * group, min((gI + 1) * group, pieces), begin, u * W, least);
    *total = W;
    return load_elem<DT>(row, *token);
  }

  // The token at which the running mass, `before` ahead of piece p0, passes `at`, among pieces p0 .. p1 - 1; if it does not, the last kept one.
  // A wavefront for each vector of 64 lanes, eight of them at a time.
  __device__ __forceinline__ int in_pieces(int p0, int p1, double before, double at, float least) {
    static_assert(kPieceVecs == kDrawWaves, "a wavefront for each vector of a piece");
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, nvec = a.V / EPV;
    int last_seen = -1;
    for (int p = p0; p < p1; ++p) {
      const int64_t i = ((int64_t)p * kPieceVecs + wave) * kWave + lane;
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
      for (int e = 0; e < EPV; ++e) s += w[e] = kept_weight(x[e], least);
      const double incl = wave_scan_f64(s);
      if (lane == kWave - 1) sh.wave_d[wave] = incl;
      if (threadIdx.x == 0) { sh.hit = 0x7fffffff; sh.n = -1; }
      __syncthreads();
      double run = before, all = before;
#pragma unroll
      for (int k = 0; k < kDrawWaves; ++k) {
        if (k == wave) run = all;
        all += sh.wave_d[k];
      }
      run += incl - s;
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
      before = all;
      __syncthreads();
    }
    return last_seen;
  }
};
// Sum over the workgroup of a small count (at most 2^16 a wavefront); slots alternate, so that one barrier is enough.
__device__ __forceinline__ int block_count(int c, int& turn, DrawShared& sh) {
  // c: the wavefront's own, the same in its lanes
  if ((threadIdx.x & (kWave - 1)) == 0) sh.count[turn][threadIdx.x / kWave] = c;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) all += sh.count[turn][w];
  turn ^= 1;
  return all;
}
__device__ __forceinline__ int wave_sum_i32(int c) { return __builtin_amdgcn_readlane(wave_scan_i32(c), kWave - 1); }

// Exclusive place of a thread's c items in the order of the threads; their number in every thread.
__device__ __forceinline__ int block_place(int c, int* total, DrawShared& sh) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, incl = wave_scan_i32(c);
  if (lane == kWave - 1) sh.wave_i[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) {
    if (w == wave) before = all;
    all += sh.wave_i[w];
  }
  __syncthreads();
  *total = all;
  return before + incl - c;
}

template <int DT>
__device__ __forceinline__ void bad_row_out(const SampleArgs& a, int64_t r) {
  if (threadIdx.x != 0) return;
  a.token[r] = -1;
  if (a.logprob) a.logprob[r] = NAN;
  if (a.flags) a.flags[r] = SV_FLAG_BAD_ROW;
}

// No warps: a piece of the row for each wavefront in turn, weights relative to the piece's largest entry; one pass over the row.
template <int DT>
__global__ void __launch_bounds__(kDrawThreads) sample_plain_kernel(SampleArgs a) {
  constexpr int EPV = Elem<DT>::per_vec;
  __shared__ DrawShared sh;
  __shared__ float piece_top[kList];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  Draw<DT> d{a, a.z + r * a.z_stride, sh, 0.0};
  double u = a.u[r];
  const int nvec = a.V / EPV, pieces = nvec / (kPieceVecs * kWave) + 1;
  const int group = (pieces + kList - 1) / kList, groups = (pieces + group - 1) / group;
  bool nan = false;
  float row_top = -INFINITY;
  for (int gI = wave; gI < groups; gI += kDrawWaves) {
    float ref = -INFINITY;
    double sum = 0.0;
    for (int p = gI * group; p < min((gI + 1) * group, pieces); ++p) {
      const int64_t base = (int64_t)p * kPieceVecs * kWave + lane;
      u32x4 q[kPieceVecs];
#pragma unroll
      for (int j = 0; j < kPieceVecs; ++j)
        if (base + j * kWave < nvec) q[j] = load_vec(d.row, (int)(base + j * kWave));
      float tail[EPV], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < EPV; ++e) tail[e] = -INFINITY;
#pragma unroll
      for (int j = 0; j < kPieceVecs; ++j) {
        const int64_t i = base + j * kWave;
        float x[EPV];
        if (i < nvec) {
          unpack<DT>(q[j], x);
        } else if (i == nvec) {                          // the entries past the last vector
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            if (i * EPV + e < a.V) tail[e] = load_elem<DT>(d.row, (int)(i * EPV + e));
        }
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const float v = i < nvec ? x[e] : tail[e];
          nan |= v != v;
          top = fmaxf(top, v);
        }
      }
      top = wave_max_f32(top);
      if (top == -INFINITY) continue;
      if (top > ref) {
        sum = ref == -INFINITY ? 0.0 : sum * exp2_series(((double)ref - (double)top) * a.scale);
        ref = top;
      }
      d.m = (double)ref;
      double s = 0.0;
#pragma unroll
      for (int j = 0; j < kPieceVecs; ++j) {
        const int64_t i = base + j * kWave;
        if (i >= nvec) continue;
        float x[EPV];
        unpack<DT>(q[j], x);
#pragma unroll
        for (int e = 0; e < EPV; ++e) s += d.weight(x[e]);
      }
      if (base <= nvec && nvec < base + kPieceVecs * kWave && (nvec - base) % kWave == 0) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) s += d.weight(tail[e]);
      }
      sum += wave_sum_f64(s);
    }
    if (lane == 0) { sh.cum[gI] = sum; piece_top[gI] = ref; }
    row_top = fmaxf(row_top, ref);
  }
  if (__ballot(nan)) row_top = INFINITY;
  if (lane == 0) sh.wave_u[wave] = __float_as_uint(row_top);
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) top = fmaxf(top, __uint_as_float(sh.wave_u[w]));
  const double y = (double)top * a.scale;
  if (!(y >= (double)kRefFloor && y <= (double)kRefCeil) || u != u) return bad_row_out<DT>(a, r);
  u = fmin(fmax(u, 0.0), 1.0 - 0x1p-53);
  d.m = (double)top;
  double w[kOwn], W, begin;
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int i = tid * kOwn + j;
    w[j] = i < groups && sh.cum[i] > 0.0 ? sh.cum[i] * d.weight(piece_top[i]) : 0.0;
  }
  const int gI = d.place_of(w, groups, u, &W, &begin);
  const int token = d.in_pieces(gI * group, min((gI + 1) * group, pieces), begin, u * W, -INFINITY);
  if (tid == 0) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = (float)(((double)load_elem<DT>(d.row, token) - d.m) * a.inv_t - log(W));
    if (a.flags) a.flags[r] = 0;
  }
}

// Weight in float32 of an entry `below` (<= 0) the largest one: L_hi + L_lo is the scale.
struct FastScale {
  float hi, lo;
  __device__ __forceinline__ float weight(float below) const {
    const float b = fmaxf(below, -1e30f);                // (-inf times lo is no -inf)
    return exp2_fast(__builtin_fmaf(b, hi, b * lo));
  }
};

template <int DT>
__global__ void __launch_bounds__(kDrawThreads) sample_kernel(SampleArgs a) {
  constexpr int EPV = Elem<DT>::per_vec;
  __shared__ DrawShared sh;
  extern __shared__ uint16_t vec_key[];                  // [n_keys rounded up to 8]
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  Draw<DT> d{a, a.z + r * a.z_stride, sh, 0.0};
  const bool use_k = a.top_k > 0, use_p = a.top_p < 1.0, use_min = a.min_log2 > -INFINITY;
  const int nvec = a.V / EPV, n_all = nvec + (a.V > nvec * EPV);   // the last one may be a part of a vector
  const int n_keys = (n_all + a.share - 1) / a.share;
  int turn = 0;
  double u = a.u[r];
  const FastScale fast{(float)a.scale, (float)(a.scale - (double)(float)a.scale)};

  // sweep: maxima of vectors, of the lane and the row; the row's mass relative to the lane's maximum
  float mine = -INFINITY;
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
  auto take = [&](const float (&x)[EPV], float top) {    // (top: of these entries)
    if (!weigh) return;
    const float m = fmaxf(mine, top);
    if (m == -INFINITY) return;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < EPV; e += 2) s += fast.weight(x[e] - m) + fast.weight(x[e + 1] - m);
    if (m > mine) mass *= mine == -INFINITY ? 0.0 : (double)fast.weight(mine - m);
    mass += (double)s;
  };
  auto top_in = [&](const float (&x)[EPV]) {
    float t = x[0];
#pragma unroll
    for (int e = 1; e < EPV; ++e) t = fmaxf(t, x[e]);
#pragma unroll
    for (int e = 0; e < EPV; ++e) nan |= x[e] != x[e];
    return t;
  };
  if (a.share == 1) {
    constexpr int U = 8;
    int i = tid;
    for (; i + (U - 1) * kDrawThreads < nvec; i += U * kDrawThreads) {
      u32x4 q[U];
#pragma unroll
      for (int k = 0; k < U; ++k) q[k] = load_vec(d.row, i + k * kDrawThreads);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        float x[EPV];
        unpack<DT>(q[k], x);
        const float t = top_in(x);
        take(x, t);
        mine = fmaxf(mine, t);
        vec_key[i + k * kDrawThreads] = (uint16_t)(order_key(t) >> 16);
      }
    }
    u32x4 q[U];                                          // what is left, all of it under way together
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (i + k * kDrawThreads < nvec) q[k] = load_vec(d.row, i + k * kDrawThreads);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int at = i + k * kDrawThreads;
      if (at >= n_all) continue;
      float x[EPV];
      if (at < nvec) unpack<DT>(q[k], x);
      else vector_at(at, x);
      const float t = top_in(x);
      take(x, t);
      mine = fmaxf(mine, t);
      vec_key[at] = (uint16_t)(order_key(t) >> 16);
    }
  } else {
    for (int k = tid; k < n_keys; k += kDrawThreads) {
      float all = -INFINITY;
      for (int i = k * a.share; i < min((k + 1) * a.share, n_all); ++i) {
        float x[EPV];
        vector_at(i, x);
        const float t = top_in(x);
        take(x, t);
        mine = fmaxf(mine, t);
        all = fmaxf(all, t);
      }
      vec_key[k] = (uint16_t)(order_key(all) >> 16);
    }
  }
  for (int k = n_keys + tid; k < ((n_keys + 7) & ~7); k += kDrawThreads) vec_key[k] = 0;
  const uint32_t lane_key = order_key(mine) >> 16;
  {
    const float hi = wave_max_f32(nan ? INFINITY : mine), lo = -wave_max_f32(-mine);
    if (lane == 0) {
      sh.wave_u[wave] = __float_as_uint(hi);
      sh.count[0][wave] = (int)(order_key(lo) >> 16);
    }
  }
  __syncthreads();
  float top = -INFINITY;
  uint32_t low_key = 0xffffu;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) {
    top = fmaxf(top, __uint_as_float(sh.wave_u[w]));
    low_key = min(low_key, (uint32_t)sh.count[0][w]);
  }
  turn = 1;                                              // (slot 0 may still be read)
  const double y = (double)top * a.scale;
  if (!(y >= (double)kRefFloor && y <= (double)kRefCeil) || u != u) return bad_row_out<DT>(a, r);
  u = fmin(fmax(u, 0.0), 1.0 - 0x1p-53);
  d.m = (double)top;
  const uint32_t top_key = order_key(top) >> 16, none = order_key(-INFINITY);
  double all = 0.0;                                      // the row's mass
  bool exact = true;
  if (weigh) {
    all = mine == -INFINITY ? 0.0 : mass * (double)fast.weight(mine - top);
    int zero = 0;
    block_sums(all, zero, sh);
    exact = false;
  }
  auto make_exact = [&]() {
    if (exact) return;
    int count;
    d.above(none, true, count, all);
    exact = true;
  };

  // The largest sixteen-bit key that at least `want` of the keys counted by count(probe) reach; `from` to `to` hold it.
  auto select = [&](uint32_t from, uint32_t to, int want, auto&& count) {
    const uint32_t differ = from ^ to;
    if (differ == 0) return from;
    int bit = 31 - __builtin_clz(differ);
    uint32_t t = from & ~((2u << bit) - 1u);
    for (; bit >= 0; --bit) {
      const uint32_t probe = t | (1u << bit);
      if (block_count(count(probe), turn, sh) >= want) t = probe;
    }
    return t;
  };
  auto lanes_at = [&](uint32_t probe) { return (int)__popcll(__ballot(lane_key >= probe)); };
  const int own = ((n_keys + kDrawThreads * 8 - 1) / (kDrawThreads * 8)) * 8;    // keys of a thread, in order
  auto each_key = [&](auto&& f) {                        // f(key, index) of the thread's keys, eight of them loaded at a time
    for (int k = tid * own; k < min((tid + 1) * own, n_keys); k += 8) {
      const u32x4 q = *reinterpret_cast<const u32x4*>(vec_key + k);
#pragma unroll
      for (int e = 0; e < 8; ++e) f((q[e / 2] >> (16 * (e % 2))) & 0xffffu, k + e);
    }
  };
  auto vectors_at = [&](uint32_t probe) {
    int c = 0;
    each_key([&](uint32_t key, int) { c += key >= probe; });
    return wave_sum_i32(c);
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
    if (want > 0 && want <= kDrawThreads && attempt == 0) {
      tau = select(low_key, top_key, want, lanes_at) << 16;
    } else if (want > 0 && want <= n_keys) {
      tau = select(0, top_key, want, vectors_at) << 16;
    }
    tau = max(tau, none);
    if (!use_k) tau = max(tau, min_key);                 // (the K-th value may lie below what min-p keeps)
    if (use_k && want > n_keys) break;
    // the vectors that reach it, in order
    int c = 0, n_vec, n;
    each_key([&](uint32_t key, int k) {
      if (key >= (tau >> 16) && k < n_keys) c += min(a.share, n_all - k * a.share);
    });
    int at = block_place(c, &n_vec, sh);
    if (n_vec > kList) break;
    each_key([&](uint32_t key, int k) {
      if (key >= (tau >> 16) && k < n_keys)
        for (int i = k * a.share; i < min((k + 1) * a.share, n_all); ++i) sh.vec[at++] = (uint32_t)i;
    });
    __syncthreads();
    // their entries
    float x[kOwn][EPV];
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
    for (int j = 0; j < kOwn; ++j) {
      if (v0[j] < 0) continue;
      vector_at(v0[j], x[j]);
    }
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      if (v0[j] < 0) continue;
#pragma unroll
      for (int e = 0; e < EPV; ++e) c += x[j][e] >= least && v0[j] * EPV + e < a.V;
    }
    at = block_place(c, &n, sh);
    if (n > kList) break;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      if (v0[j] < 0) continue;
#pragma unroll
      for (int e = 0; e < EPV; ++e)
        if (x[j][e] >= least && v0[j] * EPV + e < a.V)
          sh.key[at++] = ((uint64_t)order_key(x[j][e]) << 32) | (uint32_t)(v0[j] * EPV + e);
    }
    __syncthreads();
    if (use_k && n < a.top_k) break;
    const bool whole_min = use_min && tau <= min_key;    // the list holds all that min-p keeps
    if (n <= kWave) {
      // one wavefront, a lane for each entry, by ascending token.  out_i[0]: 0 settled, 1 does not reach, 2 too near a decision
      for (int pass = 0; pass < 2; ++pass) {
        if (wave == 0) {
          const uint64_t key = lane < n ? sh.key[lane] : 0;
          const uint32_t vk = (uint32_t)(key >> 32);
          const float v = key_float(vk);
          const double k2 = d.weight_log2(v);
          double w = lane < n ? exp2_series(k2) : 0.0;
          bool keep = lane < n;
          int state = 0;
          if (use_k) {
            int above = 0;                               // entries of a larger value
            for (int j = 0; j < n; ++j) above += (uint32_t)__builtin_amdgcn_readlane(vk, j) > vk;
            keep = keep && above < a.top_k;
          }
          if (use_p) {
            if (!keep) w = 0.0;
            double above = 0.0, sum = 0.0;               // masses of larger values, of all
            for (int j = 0; j < n; ++j) {
              const double wj = lane_f64(w, j);
              sum += wj;
              above += (uint32_t)__builtin_amdgcn_readlane(vk, j) > vk ? wj : 0.0;
            }
            const double target = a.top_p * (use_k ? sum : all);
            const double band = use_k || exact ? 0.0 : kMassError * all;
            if (__ballot(keep && fabs(above - target) < band) || fabs(sum - target) < band) state = 2;
            else if (!(sum >= target) && !use_k && !whole_min) state = 1;
            keep = keep && above < target;
          } else if (!use_k && !whole_min) {
            state = 1;
          }
          keep = keep && k2 >= a.min_log2;
          w = keep ? w : 0.0;
          const double incl = wave_scan_f64(w), total = lane_f64(incl, kWave - 1);
          const uint64_t hits = __ballot(w > 0.0 && incl > u * total), any = __ballot(w > 0.0);
          const int i = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(any);
          if (lane == i) {
            sh.out_i[1] = (int)(uint32_t)key;
            sh.out_d[1] = (double)v;
          }
          if (lane == 0) { sh.out_i[0] = state; sh.out_d[0] = total; }
        }
        __syncthreads();
        const int state = sh.out_i[0];
        if (state == 0) {
          token = sh.out_i[1];
          z = (float)sh.out_d[1];
          W = sh.out_d[0];
          done = true;
        }
        __syncthreads();
        if (state != 2) break;
        make_exact();
      }
    } else {
      // the workgroup, kOwn entries a thread, by ascending token
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
      const uint32_t top32 = order_key(top);
      // the largest key that satisfies f; the lower half of a bfloat16 key says nothing
      constexpr int stop = DT == DT_BF16 ? 16 : 0;
      auto search = [&](uint32_t from, auto&& f) {
        const uint32_t differ = from ^ top32;
        if (differ == 0) return from;
        int bit = 31 - __builtin_clz(differ);
        uint32_t t = from & ~((2u << bit) - 1u);
        for (; bit >= stop; --bit) {
          const uint32_t probe = t | (1u << bit);
          if (f(probe)) t = probe;
        }
        return t;
      };
      auto mass_at = [&](uint32_t probe) {
        double s = 0.0;
        int c2 = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) s += vk[j] >= probe ? w[j] : 0.0;
        block_sums(s, c2, sh);
        return s;
      };
      uint32_t cut = tau;
      if (use_k)
        cut = search(tau, [&](uint32_t probe) {
          int c2 = 0;
#pragma unroll
          for (int j = 0; j < kOwn; ++j) c2 += (int)__popcll(__ballot(vk[j] >= probe));
          return block_count(c2, turn, sh) >= a.top_k;
        });
      bool settled = use_k || use_p || whole_min;
      if (use_p) {
        const double listed = mass_at(use_k ? cut : 1u);
        if (use_k) all = listed;
        if (!use_k && !exact && fabs(listed - a.top_p * all) < kMassError * all) make_exact();
        if (listed >= a.top_p * all) {
          const uint32_t kth = cut;
          auto nearest = [&](double target) { return search(kth, [&](uint32_t probe) { return mass_at(probe) >= target; }); };
          cut = max(nearest(a.top_p * all), kth);
          if (!use_k && !exact) {
            const double at_cut = mass_at(cut), over = mass_at(cut + (1u << stop)), target = a.top_p * all;
            if (at_cut - target < kMassError * all || target - over < kMassError * all) {
              make_exact();
              cut = max(nearest(a.top_p * all), kth);
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
        // (place_of counts places of kOwn a thread; threads own per_n of them)
        const int i = d.place_of(kept, kList, u, &W, &before);
        const uint64_t key = sh.key[(i / kOwn) * per_n + i % kOwn];
        token = (int)(uint32_t)key;
        z = key_float((uint32_t)(key >> 32));
        done = true;
        __syncthreads();
      }
    }
    if (use_k || !use_p) break;
  }
  if (!done) {
    uint32_t least = none;                               // keys below it are dropped
    int count = a.V;
    if (use_k) {
      least = d.narrow(true, a.top_k, 0.0, none, a.V, 0, 0, 0.0);
      if (use_p) d.above(least, true, count, all);
    } else if (use_p) {
      make_exact();
    }
    if (use_p) least = d.narrow(false, 0, a.top_p * all, least, count, 0, 0, 0.0);
    z = d.draw_swept(key_float(least), u, &token, &W);
  }
  if (tid == 0) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = (float)(((double)z - d.m) * a.inv_t - log(W));
    if (a.flags) a.flags[r] = 0;
  }
}

}  // namespace sv

extern "C" int sv_sample(const void* z, int64_t z_stride, int rows, int V, int dtype, float temperature, int top_k, float top_p,
                         float min_p, const double* u, int32_t* token, float* logprob_or_null, uint32_t* flags_or_null,
                         sv_stream_t stream) {
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
               logprob_or_null, flags_or_null};
  const bool plain = a.top_k == 0 && a.top_p >= 1.0 && min_p == 0.f;
  const size_t lds = plain ? 0 : ((size_t)(vectors + share - 1) / share + 7) / 8 * 16;
  in_launches(rows, kDrawThreads, [&](long long first, dim3 grid) {
    SampleArgs b = a;
    b.z += first * b.z_stride;
    b.u += first;
    b.token += first;
    if (b.logprob) b.logprob += first;
    if (b.flags) b.flags += first;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kDrawThreads), lds, as_stream(stream), b); };
    if (dtype == SV_F32) { if (plain) go(sample_plain_kernel<DT_F32>); else go(sample_kernel<DT_F32>); }
    else { if (plain) go(sample_plain_kernel<DT_BF16>); else go(sample_kernel<DT_BF16>); }
  });
  return launch_status();
}
